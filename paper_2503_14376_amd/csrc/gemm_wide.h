// bf16 products in tiles of 256 x 256 or 256 x 128 (BN): four wavefronts, one per SIMD, each with 128 x BN / 2 results in its
// accumulation registers.
// (Eight wavefronts of 128 x 64 read half as much again from LDS; under load the clock goes by the power that is drawn.)
// The matrix unit bounds it, busy in 76 - 83 % of the CUs' clocks, at a clock that falls with the operands' toggling (zeros take
// 1 / 1.35 of the time of random values): 8192^3 1439 TFLOP/s, pair 8192 x 4096 x 10944 1.10 - 1.19 ms (1234 - 1330).
//
// A step of the contraction is 64 wide.  Each operand's tile is kept as two halves (half h: of every wavefront's 128 rows or
// columns the first or second half; of a pair's columns: matrix h), in two slots each: 128 KB for BN = 256.  A step has two phases
// of BN / 8 matrix instructions per wavefront, with one barrier each:
//   X: A0 B0, then A0 B1, while the fragments of B1 and A1 are read;      requests A0, B0 of the step after the next
//   Y: A1 B0, then A1 B1, while those of the next step's A0 and B0 are;   requests A1, B1 of the step after the next
// so that a half's memory is requested anew the phase after its last read, and requests have three phases (some 3000 clocks
// for BN = 256) to arrive: at every phase's start those of two phases may be under way.  Steps behind the last request nothing
// (bounds of zero bytes), which keeps the counts.  One LDS read or request stands between any two matrix instructions.
#pragma once
#include "gemm.h"

namespace tfla {

template <int BN, bool ATR, bool BTR, bool PAIR, int EPI>
__global__ void __launch_bounds__(256, 1) gemm_bf16_wide_kernel(GemmArgs a, int tms, int tns) {
    static_assert(!PAIR || !BTR, "pairs are plain operands");
    constexpr int HB = BN / 2;                              // rows of a half of B
    constexpr int NB = HB / 64;                             // its 32-wide blocks per wavefront
    constexpr int AHALF = 16384, BHALF = HB * 128, ASLOT = 2 * AHALF, BSLOT = 2 * BHALF;
    __shared__ __align__(1024) char lds[2 * (ASLOT + BSLOT)];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave >> 1, wn = wave & 1;
    OperandStream<128, ATR, 64, 256, 2, false> oa;
    OperandStream<HB, BTR, PAIR ? HB : HB / 2, 256, 2, PAIR> ob;
    constexpr int NA = oa.N, NBQ = ob.N, LOADS = NA + NBQ;  // requests of a wavefront per phase
    StepStream<PAIR, 1> st;
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
    const uint32_t la = lds_addr(lds) + wave * 1024, lb = la + 2 * ASLOT;
    uint32_t slot;              // of the step to request, 0 or 1

    // fragments: per lane offsets into a half
    KFragReader<64> kf;
    uint32_t ta[2], tb[NB];
    if constexpr (!ATR || !BTR) kf.init(lane & 31, lane >> 5);
#pragma unroll
    for (int i = 0; i < 2; ++i)
        if constexpr (ATR) ta[i] = TFragReader<128>::offset_of(lane, 8, wm * 2 + i);
#pragma unroll
    for (int i = 0; i < NB; ++i)
        if constexpr (BTR) tb[i] = TFragReader<HB>::offset_of(lane, 8, wn * NB + i);
    const char* la_p = lds + (ATR ? 0 : wm * 64 * 128);
    const char* lb_p = lds + 2 * ASLOT + (BTR ? 0 : wn * NB * 32 * 128);
    // fragment n = (contraction steps 16 (n / blocks) ..., block n % blocks) of half H in slot SL
#define TFLA_FRAG_A(DST, H, SL, n)                                                                                            \
    do {                                                                                                                      \
        const int ks_ = (n) / 2, i_ = (n) % 2;                                                                                \
        const char* p_ = la_p + (SL) * ASLOT + (H) * AHALF;                                                                   \
        if constexpr (ATR) DST[i_][ks_] = TFragReader<128>::load_at(p_, ta[i_], ks_ * 16, ks_ * 16 + 4);                      \
        else DST[i_][ks_] = kf.load(p_, ks_, i_);                                                                             \
    } while (0)
#define TFLA_FRAG_B(DST, H, SL, n)                                                                                            \
    do {                                                                                                                      \
        const int ks_ = (n) / NB, i_ = (n) % NB;                                                                              \
        const char* p_ = lb_p + (SL) * BSLOT + (H) * BHALF;                                                                   \
        if constexpr (BTR) DST[i_][ks_] = TFragReader<HB>::load_at(p_, tb[i_], ks_ * 16, ks_ * 16 + 4);                       \
        else DST[i_][ks_] = kf.load(p_, ks_, i_);                                                                             \
    } while (0)
    // matrix instruction m of a product of halves; the scheduler keeps what stands around it on its side.  (Blocks of a pair
    // alternate.)
#define TFLA_MUL(A, B, HA, HB_, m)                                                                                            \
    do {                                                                                                                      \
        const int ks_ = (m) / (2 * NB), i_ = (m) / NB % 2, j_ = (m) % NB, c_ = PAIR ? j_ * 2 + (HB_) : (HB_) * NB + j_;        \
        __builtin_amdgcn_sched_barrier(0);                                                                                    \
        acc[(HA) * 2 + i_][c_] = mma_bf16<EPI>(A[i_][ks_], B[j_][ks_], acc[(HA) * 2 + i_][c_]);                               \
    } while (0)
    // request r of the A or B half H
#define TFLA_REQUEST(H, r)                                                                                                    \
    do {                                                                                                                      \
        if ((r) < NA) oa.template issue<H>(r, la + slot * ASLOT + (H) * AHALF);                                               \
        else if ((r) < LOADS) ob.template issue<H>((r) - NA, lb + slot * BSLOT + (H) * BHALF);                                \
    } while (0)
#define TFLA_PHASE()                                                     \
    do {                                                                 \
        if (landed > 0) --landed;                                        \
        else wait_vmcnt<2 * LOADS>();                                    \
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); \
    } while (0)

    // the first two steps of a tile
    auto start = [&]() {
        st.at = k_begin;
        slot = 0;
        st.find(a, w, row0, col0, oa, ob, tid);
#pragma unroll
        for (int q = 0; q < 2; ++q) {
#pragma unroll
            for (int r = 0; r < LOADS; ++r) TFLA_REQUEST(0, r);
#pragma unroll
            for (int r = 0; r < LOADS; ++r) TFLA_REQUEST(1, r);
            st.next(a, w, row0, col0, oa, ob, tid);
            slot ^= 1;
        }
    };
    f32x16 acc[4][2 * NB];
    bf16x8 a0[2][4], a1[2][4], b0[NB][4], b1[NB][4];
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
        uint32_t at = 0;        // slot of the step that is multiplied
        int landed = 3;         // phases that need nothing but the first two steps, which have arrived
        constexpr int Q = 8 * NB;       // matrix instructions of a product of halves
        for (int t = k_begin; t < st.k_end; ++t) {
            // X: first b1, which the second half of the phase needs, then a1 and the requests in turn
            TFLA_PHASE();
#pragma unroll
            for (int m = 0; m < 2 * Q; ++m) {
                if (m < Q) TFLA_MUL(a0, b0, 0, 0, m);
                else TFLA_MUL(a0, b1, 0, 1, m - Q);
                if (NB == 2) {
                    if (m < 8) TFLA_FRAG_B(b1, 1, at, m);
                    else if (m < 24 && m % 2 == 0) TFLA_FRAG_A(a1, 1, at, (m - 8) / 2);
                    else if (m < 24) TFLA_REQUEST(0, (m - 9) / 2);
                } else {
                    if (m < 4) TFLA_FRAG_B(b1, 1, at, m);
                    else if (m < 12) {
                        TFLA_FRAG_A(a1, 1, at, m - 4);
                        TFLA_REQUEST(0, m - 4);
                    }
                }
            }
            at ^= 1;
            // Y: the next step's a0 and the requests in turn, then its b0, which the first half of the phase still needed
            TFLA_PHASE();
#pragma unroll
            for (int m = 0; m < 2 * Q; ++m) {
                if (m < Q) TFLA_MUL(a1, b0, 1, 0, m);
                else TFLA_MUL(a1, b1, 1, 1, m - Q);
                if (NB == 2) {
                    if (m < 16 && m % 2 == 0) TFLA_FRAG_A(a0, 0, at, m / 2);
                    else if (m < 16) TFLA_REQUEST(1, m / 2);
                    else if (m < 24) TFLA_FRAG_B(b0, 0, at, m - 16);
                } else {
                    if (m < 8) {
                        TFLA_FRAG_A(a0, 0, at, m);
                        TFLA_REQUEST(1, m);
                    } else if (m < 12) TFLA_FRAG_B(b0, 0, at, m - 8);
                }
                if (m == 2 * Q - 4) {
                    st.next(a, w, row0, col0, oa, ob, tid);
                    slot ^= 1;
                }
            }
        }
        // what was requested of steps behind the end has to have arrived before the memory is used anew
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        const GemmWork done = w;
        const long drow = row0 + wm * 128;
        const int dcol = col0 + wn * (PAIR ? NB * 32 : NB * 64);
        id += gridDim.x;
        const bool more = id < total;
        if (more) {
            take(id);
            start();
        }
        const bool full = wave_epilogue<bf16_t, EPI, PAIR, 4, 2 * NB>(a, done, drow, dcol, acc, lane);
        if (!more) break;
        // the requests are older than the epilogue's operations, so its last stores need not have arrived.  Of a whole tile every lane
        // stores 4 x 2 NB blocks (a pair's two make one) in 16 bytes of two rows, or partial results in 16 words, at the least: a pair of
        // BN = 128 without a and u has no store to spare.
        constexpr int STORES = 4 * 2 * NB * (EPI == EPI_PART ? 16 : 2) / (PAIR && EPI != EPI_PART ? 2 : 1), NEWER = 8;
        static_assert(STORES >= NEWER, "what may be under way is stores alone");
        if (full) wait_vmcnt<NEWER>();
        else wait_vmcnt<0>();
    }
#undef TFLA_REQUEST
#undef TFLA_FRAG_A
#undef TFLA_FRAG_B
#undef TFLA_MUL
#undef TFLA_PHASE
}

}  // namespace tfla
