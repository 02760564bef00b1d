// Products in 8 bits in tiles of 256 x 256 or 256 x 128 (BN): the scheme of gemm_wide.h, whose phases, halves and slots these are; a step
// of the contraction is 128 codes, a matrix instruction takes 64 of them and twice the time of a bf16 one.
//
// The scales of a step are requested with its first halves, in phase X, and read into registers in the phase before the step (Y), so
// that the two slots of theirs do.  One word per row and step: some 2 % of what LDS receives and gives.
#pragma once
#include "q8_gemm.h"

namespace tfla {

// The pair's results, 32 rows at a time: bias, a and u where wanted, h = act(a) u, its scale and codes.  The 128 columns that share a scale
// are this tile's: two wavefronts hold 64 each and meet in `meet` (two areas in turn, so that one meeting per 32 rows is enough).
template <bool FULL>
__device__ __forceinline__ void q8_gated_epilogue(const Q8GemmArgs& q, long row0, int col0, int wm, int wn, f32x16 (&acc)[4][4], int lane,
                                                  uint32_t (*meet)[2][2][32]) {
    const GemmArgs& a = q.g;
    const int c = lane & 31, g = lane >> 5;
    int rows = 4;
    asm("" : "+s"(rows));
#pragma unroll 1
    for (int mb = 0; mb < rows; ++mb) {
        f32x16 cur[4];
#define TFLA_PICK(I)                                                          \
    case I:                                                                   \
        _Pragma("unroll") for (int j = 0; j < 4; ++j) cur[j] = acc[I][j];     \
        break;
        switch (mb) {
            TFLA_PICK(0) TFLA_PICK(1) TFLA_PICK(2) TFLA_PICK(3)
            default: __builtin_unreachable();
        }
#undef TFLA_PICK
        float v[4][8], u[4][8];
#pragma unroll
        for (int j = 0; j < 4; j += 2) {
            eight_columns(cur[j], v[j], v[j + 1]);
            eight_columns(cur[j + 1], u[j], u[j + 1]);
        }
        // group i: row m + 16 (i & 1), columns n + 32 (i >> 1) ...
        const long m = row0 + mb * 32 + (c & 15);
        const int n = col0 + wn * 64 + (c >> 4) * 16 + 8 * g;
        auto left = [&](int i) { return FULL ? 8 : (m + (i & 1) * 16 < a.M ? min(8, a.N - n - (i >> 1) * 32) : 0); };
        auto at = [&](int i) { return (m + (i & 1) * 16) * a.N + n + (i >> 1) * 32; };
        auto ready = [&](float (&x)[4][8], const float* bias, void* keep) {
            if (bias) {
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    float t[8];
                    load8<float>(bias, n + k * 32, FULL ? 8 : a.N - n - k * 32).get(t);
#pragma unroll
                    for (int e = 0; e < 8; ++e) { x[2 * k][e] += t[e]; x[2 * k + 1][e] += t[e]; }
                }
            }
            if (keep) {
#pragma unroll
                for (int i = 0; i < 4; ++i) store8<bf16_t>(keep, at(i), left(i), x[i]);
            }
        };
        ready(v, a.bias[0], a.z[0]);
        ready(u, a.bias[1], a.z[1]);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float h = act_value<bf16_t>(v[i][e], a.act) * u[i][e];
                v[i][e] = FULL || e < left(i) ? h : 0.0f;
            }
        if (q.hc) {
#pragma unroll
            for (int i = 0; i < 4; ++i) store8<bf16_t>(q.hc, at(i), left(i), v[i]);
        }
        uint32_t most[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            uint32_t x = max(q8_magnitude8(v[r]), q8_magnitude8(v[r + 2]));
            // the other columns of the row are those of the lanes 16 and 32 further
            const auto p = __builtin_amdgcn_permlane16_swap(x, x, false, false);
            const uint32_t p0 = p[0], p1 = p[1];
            x = max(p0, p1);
            const auto h = __builtin_amdgcn_permlane32_swap(x, x, false, false);
            const uint32_t h0 = h[0], h1 = h[1];
            most[r] = max(h0, h1);
        }
        uint32_t (*area)[2][32] = meet[mb & 1];
        if (lane < 16) {
            area[wm][wn][lane] = most[0];
            area[wm][wn][lane + 16] = most[1];
        }
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const uint32_t s = q8_scale(max(most[r], area[wm][wn ^ 1][(c & 15) + 16 * r]));
            const float inv = q8_inverse(s);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int i = 2 * k + r, l = left(i);
                if (l > 0) q8_store8(q.h.q + at(i), q8_codes8(v[i], inv), l);
            }
            if (wn == 0 && lane < 16 && (FULL || m + 16 * r < a.M)) q.h.s[(long)(col0 >> 7) * a.M + m + 16 * r] = (uint8_t)s;
        }
    }
}

template <int BN, bool PAIR, int EPI>
__global__ void __launch_bounds__(256, 1) gemm_q8_wide_kernel(Q8GemmArgs q, int tms, int tns) {
    static_assert(EPI != EPI_GATED || (PAIR && BN == 256), "the tile holds the 128 columns of a scale");
    const GemmArgs& a = q.g;
    constexpr int HB = BN / 2;                              // rows of a half of B
    constexpr int NB = HB / 64;                             // its 32-wide blocks per wavefront
    constexpr int AHALF = 16384, BHALF = HB * 128, ASLOT = 2 * AHALF, BSLOT = 2 * BHALF;
    typedef ScaleStream<256, BN, 4, PAIR> Scales;
    constexpr int SSLOT = Scales::BYTES, SN = Scales::N;
    __shared__ __align__(1024) char lds[2 * (ASLOT + BSLOT + SSLOT)];
    __shared__ uint32_t meet[EPI == EPI_GATED ? 2 : 1][2][2][32];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave >> 1, wn = wave & 1, l32 = lane & 31;
    OperandStream<128, false, 64, 256, 2, false> oa;
    OperandStream<HB, false, PAIR ? HB : HB / 2, 256, 2, PAIR> ob;
    Scales sc;
    constexpr int NA = oa.N, NBQ = ob.N, LOADS = NA + NBQ;  // requests of a wavefront per phase, beside those of scales
    Q8StepStream<PAIR, 1> qs;
    auto& st = qs.st;
    st.ksteps = (a.K + 63) / 64;
    const int all = st.ksteps * a.segs, per = (all + a.split - 1) / a.split;
    const unsigned total = (unsigned)tms * tns * a.split * a.batch;
    GemmWork w;
    long row0;
    int col0, k_begin;
    auto take = [&](unsigned id) {
        w = gemm_work(xcd_range(id, total), tms, tns, a.split);
        row0 = (long)w.tm * 256;
        col0 = w.tn * (PAIR ? HB : BN);
        k_begin = w.part * per;
        st.k_end = min(all, k_begin + per);
    };
    oa.init(a.lda, tid);
    ob.init(a.ldb, tid);
    const uint32_t la = lds_addr(lds) + wave * 1024, lb = la + 2 * ASLOT, ls = lds_addr(lds) + 2 * (ASLOT + BSLOT) + wave * 256;
    uint32_t slot;              // of the step to request, 0 or 1
    KFragReader<64> kf;
    kf.init(l32, lane >> 5);
    const char* la_p = lds + wm * 64 * 128;
    const char* lb_p = lds + 2 * ASLOT + wn * NB * 32 * 128;
    const char* ls_p = lds + 2 * (ASLOT + BSLOT) + l32 * 4;
    // piece n of half H in slot SL: block n / 4, 16 codes of four pieces each
#define TFLA_PIECE(DST, P, n)                                                                                                \
    do {                                                                                                                      \
        const u32x4 w_ = __builtin_bit_cast(u32x4, kf.load(P, (n) % 4, (n) / 4));                                             \
        _Pragma("unroll") for (int e_ = 0; e_ < 4; ++e_) DST[(n) / 4][(n) % 4 / 2][(n) % 2 * 4 + e_] = (int)w_[e_];           \
    } while (0)
#define TFLA_FRAG_A(DST, H, SL, n) TFLA_PIECE(DST, la_p + (SL) * ASLOT + (H) * AHALF, n)
#define TFLA_FRAG_B(DST, H, SL, n) TFLA_PIECE(DST, lb_p + (SL) * BSLOT + (H) * BHALF, n)
    // matrix instruction m of a product of halves; the scheduler keeps what stands around it on its side
#define TFLA_MUL(A, B, HA, HB_, m)                                                                                            \
    do {                                                                                                                      \
        const int ks_ = (m) / (2 * NB), i_ = (m) / NB % 2, j_ = (m) % NB, c_ = PAIR ? j_ * 2 + (HB_) : (HB_) * NB + j_;        \
        __builtin_amdgcn_sched_barrier(0);                                                                                    \
        acc[(HA) * 2 + i_][c_] = mma_q8<EPI>(A[i_][ks_], B[j_][ks_], acc[(HA) * 2 + i_][c_], sa[(HA) * 2 + i_], sb[(HB_) * NB + j_]); \
    } while (0)
#define TFLA_REQUEST(H, r)                                                                                                    \
    do {                                                                                                                      \
        if ((r) < NA) oa.template issue<H>(r, la + slot * ASLOT + (H) * AHALF);                                               \
        else if ((r) < LOADS) ob.template issue<H>((r) - NA, lb + slot * BSLOT + (H) * BHALF);                                \
    } while (0)
#define TFLA_PHASE()                                                     \
    do {                                                                 \
        if (landed > 0) --landed;                                        \
        else wait_vmcnt<2 * LOADS + SN>();                               \
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); \
    } while (0)
    f32x16 acc[4][2 * NB];
    // the compiler takes these matrix instructions for ones that it may move behind the phase's branches: their results are wanted here
    auto hold = [&]() {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 2 * NB; ++j) asm volatile("" : "+a"(acc[i][j]));
    };
    int sa[4], sb[2 * NB], na[4], nb[2 * NB];
    // scales of the step in slot SL
    auto scales = [&](uint32_t sl) {
        const char* p = ls_p + sl * SSLOT;
#pragma unroll
        for (int i = 0; i < 4; ++i) na[i] = *reinterpret_cast<const int*>(p + (wm * 128 + i * 32) * 4);
#pragma unroll
        for (int j = 0; j < 2 * NB; ++j) {
            const int h = j / NB, r = PAIR ? h * HB + wn * NB * 32 + j % NB * 32 : wn * HB + h * (HB / 2) + j % NB * 32;
            nb[j] = *reinterpret_cast<const int*>(p + (256 + r) * 4);
        }
    };
    auto turn = [&]() {
#pragma unroll
        for (int i = 0; i < 4; ++i) sa[i] = na[i];
#pragma unroll
        for (int j = 0; j < 2 * NB; ++j) sb[j] = nb[j];
    };
    // the first two steps of a tile
    auto start = [&]() {
        st.at = k_begin;
        slot = 0;
        qs.find(q, w, row0, col0, oa, ob, sc, tid);
#pragma unroll
        for (int p = 0; p < 2; ++p) {
#pragma unroll
            for (int r = 0; r < LOADS; ++r) TFLA_REQUEST(0, r);
#pragma unroll
            for (int r = 0; r < LOADS; ++r) TFLA_REQUEST(1, r);
            sc.issue_all(ls + slot * SSLOT);
            qs.next(q, w, row0, col0, oa, ob, sc, tid);
            slot ^= 1;
        }
    };
    i32x8 a0[2][2], a1[2][2], b0[NB][2], b1[NB][2];
    take(blockIdx.x);
    start();
    wait_vmcnt<0>();
    // One workgroup per CU takes tile after tile; the next one's first steps are requested before the epilogue of the last.
    for (unsigned id = blockIdx.x;;) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 2 * NB; ++j)
#pragma unroll
                for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.0f;
        barrier_nofence();
#pragma unroll
        for (int n = 0; n < 8; ++n) TFLA_FRAG_A(a0, 0, 0, n);
#pragma unroll
        for (int n = 0; n < 4 * NB; ++n) TFLA_FRAG_B(b0, 0, 0, n);
        scales(0);
        uint32_t at = 0;        // slot of the step that is multiplied
        int landed = 3;         // phases that need nothing but the first two steps, which have arrived
        constexpr int Q = 4 * NB;       // matrix instructions of a product of halves
        for (int t = k_begin; t < st.k_end; ++t) {
            // X: first b1, which the second half of the phase needs, then a1 and the requests in turn, the scales' last
            TFLA_PHASE();
            turn();
#pragma unroll
            for (int m = 0; m < 2 * Q; ++m) {
                if (m < Q) TFLA_MUL(a0, b0, 0, 0, m);
                else TFLA_MUL(a0, b1, 0, 1, m - Q);
                if (NB == 2) {
                    if (m < 4) {
                        TFLA_FRAG_B(b1, 1, at, 2 * m);
                        TFLA_FRAG_B(b1, 1, at, 2 * m + 1);
                    } else if (m < 12) {
                        TFLA_FRAG_A(a1, 1, at, m - 4);
                        TFLA_REQUEST(0, m - 4);
                    } else if (m - 12 < SN) sc.issue(m - 12, ls + slot * SSLOT);
                } else {
                    if (m < 2) {
                        TFLA_FRAG_B(b1, 1, at, 2 * m);
                        TFLA_FRAG_B(b1, 1, at, 2 * m + 1);
                    } else if (m < 6) {
                        TFLA_FRAG_A(a1, 1, at, 2 * m - 4);
                        TFLA_REQUEST(0, 2 * m - 4);
                        TFLA_FRAG_A(a1, 1, at, 2 * m - 3);
                        TFLA_REQUEST(0, 2 * m - 3);
                    } else if (m - 6 < SN) sc.issue(m - 6, ls + slot * SSLOT);
                }
            }
            hold();
            at ^= 1;
            // Y: the next step's a0 and the requests in turn, then its b0, which the first half of the phase still needed, and its scales
            TFLA_PHASE();
#pragma unroll
            for (int m = 0; m < 2 * Q; ++m) {
                if (m < Q) TFLA_MUL(a1, b0, 1, 0, m);
                else TFLA_MUL(a1, b1, 1, 1, m - Q);
                if (NB == 2) {
                    if (m < 8) {
                        TFLA_FRAG_A(a0, 0, at, m);
                        TFLA_REQUEST(1, m);
                    } else if (m < 12) {
                        TFLA_FRAG_B(b0, 0, at, 2 * m - 16);
                        TFLA_FRAG_B(b0, 0, at, 2 * m - 15);
                    }
                } else {
                    if (m < 4) {
                        TFLA_FRAG_A(a0, 0, at, 2 * m);
                        TFLA_REQUEST(1, 2 * m);
                        TFLA_FRAG_A(a0, 0, at, 2 * m + 1);
                        TFLA_REQUEST(1, 2 * m + 1);
                    } else if (m < 6) {
                        TFLA_FRAG_B(b0, 0, at, 2 * m - 8);
                        TFLA_FRAG_B(b0, 0, at, 2 * m - 7);
                    }
                }
                if (m == 2 * Q - 2) scales(at);
            }
            hold();
            qs.next(q, w, row0, col0, oa, ob, sc, tid);
            slot ^= 1;
        }
        // what was requested of steps behind the end has to have arrived before the memory is used anew
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        const GemmWork done = w;
        const long drow = row0 + wm * 128;
        const int dcol = col0;
        id += gridDim.x;
        const bool more = id < total;
        if (more) {
            take(id);
            start();
        }
        bool full;
        if constexpr (EPI == EPI_GATED) {
            full = drow - wm * 128 + 256 <= a.M && dcol + HB <= a.N;       // (the same for the wavefronts, which meet)
            if (full) q8_gated_epilogue<true>(q, drow, dcol, wm, wn, acc, lane, meet);
            else q8_gated_epilogue<false>(q, drow, dcol, wm, wn, acc, lane, meet);
        } else {
            full = wave_epilogue<bf16_t, EPI, PAIR, 4, 2 * NB>(a, done, drow, dcol + wn * (PAIR ? NB * 32 : NB * 64), acc, lane);
        }
        if (!more) break;
        // the requests are older than the epilogue's operations, so its last stores need not have arrived.  Of a whole tile every lane
        // stores 4 x 2 NB blocks in 16 bytes of two rows, partial results in 16 words, or a pair's codes in 4 x 4 pieces, at the least.
        constexpr int STORES = EPI == EPI_GATED ? 16 : 4 * 2 * NB * (EPI == EPI_PART ? 16 : 2), NEWER = 8;
        static_assert(STORES >= NEWER, "what may be under way is stores alone");
        if (full) wait_vmcnt<NEWER>();
        else wait_vmcnt<0>();
    }
#undef TFLA_REQUEST
#undef TFLA_FRAG_A
#undef TFLA_FRAG_B
#undef TFLA_PIECE
#undef TFLA_MUL
#undef TFLA_PHASE
}

}  // namespace tfla
