// Products in 8 bits in tiles of 256 x 256 or 256 x 128 (BN): the scheme of gemm_wide.h, whose phases, halves and slots these are; a step
// of the contraction is 128 codes, a matrix instruction takes 64 of them and twice the time of a bf16 one.
//
// The scales of a step are requested with its first halves, in phase X, and read into registers in the phase before the step (Y), so
// that the two slots of theirs do.  One word per row and step: some 2 % of what LDS receives and gives.
//
// Measured: 8192 x 4096 x 4096 113 us (2.4 PFLOP/s), 8192 x 4096 x 21888 580 (2.5 PFLOP/s, matrix unit 71 % busy at the clock that its power
// leaves), pair 8192 x 4096 x 2 10944 with its gate 614 (2.4 PFLOP/s), with a, u and h besides 683.
// Scratch: none, but for the linear epilogue of 256 x 256 (30 vector registers, 124 bytes a lane; as calls, 8192 x 4096 x 4096 takes 117 us, with bias
// and residual 134, with silu and z besides 148, where the bytes alone would add 13 each) and the parts of a divided pair (47).
#pragma once
#include "q8_gemm.h"

namespace tfla {

// Results.  The matrix unit leaves a lane one column of a block of 32, rows in its registers.  Which column of the tile that is, the rows of
// B in LDS decide: of a wavefront's W blocks lane n has the columns W n ... W n + W - 1, so that a row leaves as 32 neighbouring lanes with W
// columns each, whole cache lines (16 lanes on one line a clock; with 16 rows of 16 bytes side by side, as gemm.h turns its blocks, a store
// took 64 clocks of the address unit, 7 us of a pair's tile with a, u and h).
//
// One wavefront's MB x W blocks, 32 rows at a time; row0, col0: its first row and column.  Of the rows' registers a switch picks those of
// a block: unrolled, what follows a product is code that a wavefront waits for line by line.
template <int W> struct Columns { float v[W]; };
template <int W> __device__ __forceinline__ Columns<W> load_columns(const float* p, long at, int left) {
    Columns<W> r;
    if (left >= W) __builtin_memcpy(&r, p + at, 4 * W);
    else {
#pragma unroll
        for (int c = 0; c < W; ++c) r.v[c] = c < left ? p[at + c] : 0.0f;
    }
    return r;
}
template <int W> struct Packed { uint32_t w[W / 2]; };
template <int W> __device__ __forceinline__ void store_columns(uint16_t* base, uint32_t at, int left, const float (&x)[W]) {
    uint16_t* p = base + at;
    Packed<W> k;
#pragma unroll
    for (int c = 0; c < W / 2; ++c) k.w[c] = pack_bf16x2(x[2 * c], x[2 * c + 1]);
    if (left >= W) __builtin_memcpy(p, &k, 2 * W);
    else {
#pragma unroll
        for (int c = 0; c < W; ++c)
            if (c < left) p[c] = (uint16_t)(k.w[c / 2] >> (16 * (c & 1)));
    }
}
// f(kind) with the activation as a constant: one branch for all values of a block
template <typename F> __device__ __forceinline__ void by_activation(int act, F f) {
    struct None { __device__ constexpr int operator()() const { return ACT_NONE; } };
    struct Silu { __device__ constexpr int operator()() const { return ACT_SILU; } };
    struct Gelu { __device__ constexpr int operator()() const { return ACT_GELU; } };
    struct Relu { __device__ constexpr int operator()() const { return ACT_RELU; } };
    if (act == ACT_SILU) f(Silu());
    else if (act == ACT_GELU) f(Gelu());
    else if (act == ACT_RELU) f(Relu());
    else f(None());
}
#define TFLA_PICK(I)                                                            \
    case I:                                                                     \
        _Pragma("unroll") for (int j = 0; j < NA; ++j) cur[j] = acc[I][j];      \
        break;
#define TFLA_PICK_BLOCK(mb)                                        \
    switch (mb) {                                                  \
        TFLA_PICK(0) TFLA_PICK(1) TFLA_PICK(2) TFLA_PICK(3)        \
        default: __builtin_unreachable();                          \
    }

// EPI_LINEAR, EPI_STORE, EPI_PART.  NA: blocks of columns, those of a pair's two matrices in turn (EPI_PART)
template <int EPI, bool PAIR, int NA, bool FULL>
__device__ __forceinline__ void q8_epilogue(const GemmArgs& a, const GemmWork& w, long row0, int col0, f32x16 (&acc)[4][NA], int lane) {
    constexpr int W = PAIR ? NA / 2 : NA;
    const int n = col0 + (lane & 31) * W, g = lane >> 5, left = FULL ? W : a.N - n;
    // where register v's row begins, the same for all lanes, and a lane's place behind that: one address register, not one per row
    const uint32_t place = (uint32_t)(4 * g * a.N + (lane & 31) * W), place_part = (uint32_t)(4 * g * a.ld_part + (lane & 31) * W);
    Columns<W> bias;
    if (EPI == EPI_LINEAR && a.bias[0]) bias = load_columns<W>(a.bias[0], n, left);
    int blocks = 4;
    asm("" : "+s"(blocks));
#pragma unroll 1
    for (int mb = 0; mb < blocks; ++mb) {
        f32x16 cur[NA];
        TFLA_PICK_BLOCK(mb)
        const long m0 = row0 + mb * 32;
        auto exists = [&](int v) { return FULL || (left > 0 && m0 + acc_row(v, g) < a.M); };
        if constexpr (EPI == EPI_PART) {
            const int planes = PAIR ? 2 : a.batch;
#pragma unroll
            for (int p = 0; p < (PAIR ? 2 : 1); ++p) {
                float* to = partial_plane(a, planes, w.part, PAIR ? p : w.b) + m0 * a.ld_part + col0;
#pragma unroll
                for (int v = 0; v < 16; ++v) {
                    Columns<W> x;
#pragma unroll
                    for (int c = 0; c < W; ++c) x.v[c] = cur[PAIR ? 2 * c + p : c][v];
                    if (exists(v)) {
                        float* d = to + acc_row(v, 0) * a.ld_part + place_part;
                        if (left >= W) __builtin_memcpy(d, &x, 4 * W);
                        else {
#pragma unroll
                            for (int c = 0; c < W; ++c)
                                if (c < left) d[c] = x.v[c];
                        }
                    }
                }
            }
        } else {
            auto at = [&](int v) { return (m0 + acc_row(v, 0)) * a.N + col0; };
            auto put = [&](void* p, int v0, int v1) {
#pragma unroll
                for (int v = v0; v < v1; ++v) {
                    float x[W];
#pragma unroll
                    for (int c = 0; c < W; ++c) x[c] = cur[c][v];
                    if (exists(v)) store_columns<W>(reinterpret_cast<uint16_t*>(p) + at(v), place, left, x);
                }
            };
            if constexpr (EPI == EPI_LINEAR) {
                if (a.bias[0]) {
#pragma unroll
                    for (int c = 0; c < W; ++c)
#pragma unroll
                        for (int v = 0; v < 16; ++v) cur[c][v] += bias.v[c];
                }
                if (a.z[0]) put(a.z[0], 0, 16);
                if (a.act != ACT_NONE)
                    by_activation(a.act, [&](auto kind) {
#pragma unroll
                        for (int c = 0; c < W; ++c)
#pragma unroll
                            for (int v = 0; v < 16; ++v) cur[c][v] = act_value<bf16_t>(cur[c][v], kind());
                    });
                if (a.residual) {
                    // (eight rows at a time: the registers hold no more beside the results)
#pragma unroll
                    for (int v0 = 0; v0 < 16; v0 += 8) {
                        Packed<W> r[8];
#pragma unroll
                        for (int v = 0; v < 8; ++v) {
                            const uint16_t* p = reinterpret_cast<const uint16_t*>(a.residual) + at(v0 + v) + place;
#pragma unroll
                            for (int c = 0; c < W / 2; ++c) r[v].w[c] = 0;
                            if (exists(v0 + v)) {
                                if (left >= W) __builtin_memcpy(&r[v], p, 2 * W);
                                else {
#pragma unroll
                                    for (int c = 0; c < W; ++c)
                                        if (c < left) r[v].w[c / 2] |= (uint32_t)p[c] << (16 * (c & 1));
                                }
                            }
                        }
#pragma unroll
                        for (int c = 0; c < W; ++c)
#pragma unroll
                            for (int v = 0; v < 8; ++v) cur[c][v0 + v] += c & 1 ? bf16_hi_to_f32(r[v].w[c / 2]) : bf16_lo_to_f32(r[v].w[c / 2]);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
            }
            put(a.out[EPI == EPI_STORE ? w.b : 0], 0, 16);
        }
    }
}

// A pair's results, 32 rows at a time, in transposed blocks as gemm.h turns them: bias, a and u where wanted, h = act(a) u, its scale and
// codes.  (Two columns a lane, as above, are four times the stores: 8192 x 4096 x 10944 651 -> 725 us.  Four columns, two rows exchanged between lanes
// 16 apart, are whole lines and half the exchanges, but twice the stores: 677 -> 716, without a, u and h 625 -> 617.  Stores past the caches:
// 683 -> 724, where inputs change from call to call.)  The 128 columns that share a scale are this tile's: two wavefronts hold 64 each and meet
// in `meet` (two areas in turn, so that one meeting per 32 rows is enough).
template <bool FULL>
__device__ __forceinline__ void q8_gated_epilogue(const Q8GemmArgs& q, long row0, int col0, int wm, int wn, f32x16 (&acc)[4][4], int lane,
                                                  uint32_t (*meet)[2][2][32]) {
    constexpr int NA = 4;
    const GemmArgs& a = q.g;
    const int c = lane & 31, g = lane >> 5;
    int rows = 4;
    asm("" : "+s"(rows));
#pragma unroll 1
    for (int mb = 0; mb < rows; ++mb) {
        f32x16 cur[NA];
        TFLA_PICK_BLOCK(mb)
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
        // (with a branch for each value the epilogue of a tile took 11 us of 55)
        by_activation(a.act, [&](auto kind) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float h = act_value<bf16_t>(v[i][e], kind()) * u[i][e];
                    v[i][e] = FULL || e < left(i) ? h : 0.0f;
                }
        });
        if (q.hc) {
#pragma unroll
            for (int i = 0; i < 4; ++i) store8<bf16_t>(q.hc, at(i), left(i), v[i]);
        }
        uint32_t most[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            uint32_t x = max(q8_largest(v[r]), q8_largest(v[r + 2]));
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
            const float power = q8_power(s);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int i = 2 * k + r, l = left(i);
                if (l > 0) q8_store8(q.h.q + at(i), q8_codes8(v[i], power), l);
            }
            if (wn == 0 && lane < 16 && (FULL || m + 16 * r < a.M)) q.h.s[(long)(col0 >> 7) * a.M + m + 16 * r] = (uint8_t)s;
        }
    }
}

#undef TFLA_PICK
#undef TFLA_PICK_BLOCK

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
    // Row r of half H of B stands for the column of the tile that its place in the results has: of block j = r / 32 % NB of wavefront
    // r / (32 NB) lane r % 32's column j (a pair's) or NB H + j among the W that are the lane's.  (A gate's blocks: rows in their order.)
    constexpr int W = PAIR ? NB : 2 * NB;
    constexpr bool TURNED = EPI == EPI_GATED;
    OperandStream<HB, false, PAIR ? HB : NB, 256, 2, PAIR> ob;
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
#pragma unroll
    for (int j = 0; j < (TURNED ? 0 : NBQ); ++j) {
        const int r = (wave + j * 4) * 8 + (lane >> 3), col = ((lane & 7) ^ swz_mask<SWZ_K, 8>(r)) * 8;
        ob.goff[j] = (uint32_t)(((r / (32 * NB) * 32 * W + r % 32 * W + r / 32 % NB) * a.ldb + col) * 2);
    }
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
        acc[(HA) * 2 + i_][c_] = mma_q8<TURNED ? EPI_GATED : EPI_PART>(A[i_][ks_], B[j_][ks_], acc[(HA) * 2 + i_][c_], sa[(HA) * 2 + i_], sb[(HB_) * NB + j_]); \
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
            const int r = (PAIR ? j / NB * HB : 0) + wn * 32 * W + (PAIR ? j % NB : j) * (TURNED ? 32 : 1);
            nb[j] = *reinterpret_cast<const int*>(p + (256 + r) * 4 + (TURNED ? 0 : l32 * 4 * (W - 1)));
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
            const int col = dcol + wn * 32 * W;
            full = drow + 128 <= a.M && col + 32 * W <= a.N;
            if (full) q8_epilogue<EPI, PAIR, 2 * NB, true>(a, done, drow, col, acc, lane);
            else q8_epilogue<EPI, PAIR, 2 * NB, false>(a, done, drow, col, acc, lane);
        }
        if (!more) break;
        // the requests are older than the epilogue's operations, so its last stores need not have arrived: of a whole tile every lane stores
        // 4 x 16 pieces at the least, a gate's codes 4 x 4.
        constexpr int NEWER = EPI == EPI_GATED ? 16 : 32;
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
