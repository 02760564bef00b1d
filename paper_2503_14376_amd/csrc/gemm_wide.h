// bf16 products in tiles of 256 x 256: four wavefronts, one per SIMD, each with 128 x 128 results in its accumulation registers.
// (Eight wavefronts of 128 x 64 read half as much again from LDS; under load the clock goes by the power that is drawn.)
//
// A step of the contraction is 64 wide.  Each operand's tile is kept as two halves (half h: of every wavefront's 128 rows or
// columns the 64 from 64 h on; of a pair's columns: matrix h), in two slots each: 128 KB.  A step has two phases of 32 matrix
// instructions per wavefront, with one barrier each:
//   X: A0 B0, then A0 B1, while the fragments of B1 and A1 are read;      requests A0, B0 of the step after the next
//   Y: A1 B0, then A1 B1, while those of the next step's A0 and B0 are;   requests A1, B1 of the step after the next
// so that a half's memory is requested anew the phase after its last read, and requests have three phases (some 3000 clocks)
// to arrive: at every phase's start sixteen requests per wavefront may be under way.  Steps behind the last request nothing
// (bounds of zero bytes), which keeps the counts.  One LDS read or request stands between any two matrix instructions.
#pragma once
#include "gemm.h"

namespace tfla {

// One operand's requests.  A half is 128 output rows (or columns) x 64 steps, 16 KB, four requests of each of 256 threads; its
// local row r stands for row (r / G) 2 G + r % G of the operand behind the half's first row.  The buffer descriptors of both
// halves are kept ready and moved on by a step at a time; everything else about them is found anew only at the steps where
// it changes (the last step of a contraction that is no multiple of 64, the second segment, the end).
template <bool TR, int G, bool PAIR> struct WideOperand {
    typedef DmaTile<TR ? 64 : 128, TR ? 128 : 64, 256, TR ? SWZ_T : SWZ_K> Shape;
    static constexpr int CPR = Shape::CPR, N = 4;
    static constexpr uint32_t BEHIND = 0x40000000u;       // an offset beyond every bound
    static_assert(Shape::N == N, "four requests per half");
    u32x4 d[2];                 // descriptors of the halves at the next step
    uint32_t goff[N], hop;      // byte offsets of this lane; bytes from step to step
    __device__ __forceinline__ void init(long ld, int tid) {
        const int lane = tid & 63, wave = tid >> 6;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int q = (wave + j * 4) * 64 + lane, r = q / CPR, c = ((q % CPR) ^ swz_mask<TR ? SWZ_T : SWZ_K, CPR>(r)) * 8;
            const int row = TR ? r : (r / G) * 2 * G + r % G, col = TR ? (c / G) * 2 * G + c % G : c;
            goff[j] = (uint32_t)((row * ld + col) * 2);
        }
        hop = (uint32_t)(TR ? 128 * ld : 128);
    }
    // p0, p1: the matrices of the halves; first: the operand's first row in the tile, of `extent`; K: contraction length; steps from k0 on.
    // Columns behind the end of a transposed operand's rows are other rows' values: they meet results that are not stored.
    __device__ __forceinline__ void set(const void* p0, const void* p1, long ld, long first, long extent, int K, int k0, bool exists, int tid) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const long at = first + (PAIR ? 0 : h * G), left = extent - at;
            const long rows = TR ? (K - k0 < 64 ? K - k0 : 64) : (left < 256 ? left : 256);
            const int K8 = (K + 7) & ~7, cols = TR ? (int)(left < 256 ? (left + 7) & ~7l : 256) : (K8 - k0 < 64 ? K8 - k0 : 64);
            const uint64_t b = reinterpret_cast<uint64_t>(h ? p1 : p0) + 2 * (TR ? k0 * ld + at : at * ld + k0);
            d[h][0] = (uint32_t)b;
            d[h][1] = (uint32_t)(b >> 32) & 0xffffu;
            d[h][2] = exists && rows > 0 && cols > 0 ? (uint32_t)((rows - 1) * ld * 2) + 2u * (uint32_t)cols : 0u;
            d[h][3] = 0x00020000u;
        }
        if constexpr (!TR) {
            const int lane = tid & 63, wave = tid >> 6, left = ((K + 7) & ~7) - k0;
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const int q = (wave + j * 4) * 64 + lane, c = ((q % CPR) ^ swz_mask<SWZ_K, CPR>(q / CPR)) * 8;
                goff[j] = (goff[j] & (BEHIND - 1)) | (c < left ? 0u : BEHIND);
            }
        }
    }
    __device__ __forceinline__ void advance() {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint64_t b = ((uint64_t)d[h][1] << 32 | d[h][0]) + hop;
            d[h][0] = (uint32_t)b;
            d[h][1] = (uint32_t)(b >> 32);
        }
    }
    // request j of half H into the half at LDS address `half` (of this wavefront's part of it)
    template <int H> __device__ __forceinline__ void issue(int j, uint32_t half) const {
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                     :: "s"(half + j * 4096), "v"(goff[j]), "s"(d[H]) : "m0");
    }
};

template <bool ATR, bool BTR, bool PAIR, int EPI>
__global__ void __launch_bounds__(256, 1) gemm_bf16_wide_kernel(GemmArgs a, int tms, int tns) {
    static_assert(!PAIR || !BTR, "pairs are plain operands");
    constexpr int HALF = 16384, SLOT = 2 * HALF, OPERAND = 2 * SLOT;
    __shared__ __align__(1024) char lds[2 * OPERAND];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave >> 1, wn = wave & 1;
    const int ksteps = (a.K + 63) / 64, all = ksteps * a.segs, per = (all + a.split - 1) / a.split;
    const unsigned total = (unsigned)tms * tns * a.split * a.batch;
    GemmWork w;
    long row0;
    int col0, k_begin, k_end;
    auto take = [&](unsigned id) {
        w = gemm_work(xcd_range(id, total), tms, tns, a.split);
        row0 = (long)w.tm * 256;
        col0 = w.tn * (PAIR ? 128 : 256);
        k_begin = w.part * per;
        k_end = min(all, k_begin + per);
    };
    WideOperand<ATR, 64, false> oa;
    WideOperand<BTR, PAIR ? 128 : 64, PAIR> ob;
    oa.init(a.lda, tid);
    ob.init(a.ldb, tid);
    // the next step to request, and the next at which its descriptors change by more than a step
    int rt, change;
    auto find = [&]() {
        const bool on = rt < k_end, second = rt >= ksteps;
        const int k0 = on ? (second ? rt - ksteps : rt) * 64 : 0;
        oa.set(a.A[second ? 1 : w.b], a.A[second ? 1 : w.b], a.lda, row0, a.M, a.K, k0, on, tid);
        ob.set(PAIR ? a.B[0] : a.B[second ? 1 : 0], PAIR ? a.B[1] : a.B[second ? 1 : 0], a.ldb, col0, a.N, a.K, k0, on, tid);
        const int seg_end = second ? 2 * ksteps : ksteps, whole = seg_end - (a.K % 64 != 0);
        change = !on ? 0x7fffffff : min(k_end, rt < whole ? whole : seg_end);
    };
    const uint32_t la = lds_addr(lds) + wave * 1024, lb = la + OPERAND;
    uint32_t rslot;             // slot of the step to request
#define TFLA_NEXT()                                        \
    do {                                                   \
        ++rt;                                              \
        rslot ^= SLOT;                                     \
        oa.advance();                                      \
        ob.advance();                                      \
        if (rt == change) find();                          \
    } while (0)
#define TFLA_REQUEST(H)                                                                                  \
    _Pragma("unroll") for (int j = 0; j < 4; ++j) oa.template issue<H>(j, la + rslot + (H) * HALF);    \
    _Pragma("unroll") for (int j = 0; j < 4; ++j) ob.template issue<H>(j, lb + rslot + (H) * HALF);

    // fragments: per lane offsets into a half
    KFragReader<64> kf;
    uint32_t ta[2], tb[2];
    if constexpr (!ATR || !BTR) kf.init(lane & 31, lane >> 5);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if constexpr (ATR) ta[i] = TFragReader<128>::offset_of(lane, 8, wm * 2 + i);
        if constexpr (BTR) tb[i] = TFragReader<128>::offset_of(lane, 8, wn * 2 + i);
    }
    const char* la_p = lds + (ATR ? 0 : wm * 64 * 128);
    const char* lb_p = lds + OPERAND + (BTR ? 0 : wn * 64 * 128);
    // fragment of block i (32 rows or columns), contraction steps 16 ks ..., of half H in slot offset SO
#define TFLA_FRAG_A(DST, H, SO, i, ks)                                                                        \
    if constexpr (ATR) DST[i][ks] = TFragReader<128>::load_at(la_p + (SO) + (H) * HALF, ta[i], (ks) * 16, (ks) * 16 + 4); \
    else DST[i][ks] = kf.load(la_p + (SO) + (H) * HALF, ks, i);
#define TFLA_FRAG_B(DST, H, SO, i, ks)                                                                        \
    if constexpr (BTR) DST[i][ks] = TFragReader<128>::load_at(lb_p + (SO) + (H) * HALF, tb[i], (ks) * 16, (ks) * 16 + 4); \
    else DST[i][ks] = kf.load(lb_p + (SO) + (H) * HALF, ks, i);
    // one matrix instruction; the scheduler keeps what stands around it on its side.  (Blocks of a pair alternate.)
#define TFLA_MUL(A, B, HA, HB, i, j, ks)                                                                      \
    __builtin_amdgcn_sched_barrier(0);                                                                        \
    acc[(HA) * 2 + i][PAIR ? (j) * 2 + HB : (HB) * 2 + j] =                                                   \
        __builtin_amdgcn_mfma_f32_32x32x16_bf16(B[j][ks], A[i][ks], acc[(HA) * 2 + i][PAIR ? (j) * 2 + HB : (HB) * 2 + j], 0, 0, 0);
#define TFLA_PHASE()                                                     \
    do {                                                                 \
        if (landed > 0) --landed;                                        \
        else wait_vmcnt<16>();                                           \
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); \
    } while (0)

    // the first two steps of a tile
    auto start = [&]() {
        rt = k_begin;
        rslot = 0;
        find();
        TFLA_REQUEST(0)
        TFLA_REQUEST(1)
        TFLA_NEXT();
        TFLA_REQUEST(0)
        TFLA_REQUEST(1)
        TFLA_NEXT();
    };
    f32x16 acc[4][4];
    bf16x8 a0[2][4], a1[2][4], b0[2][4], b1[2][4];
    take(blockIdx.x);
    start();
    wait_vmcnt<0>();
    // One workgroup per CU takes tile after tile; the next one's first steps are requested before the epilogue of the last.
    for (unsigned id = blockIdx.x;;) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.0f;
        barrier_nofence();
#pragma unroll
        for (int ks = 0; ks < 4; ++ks)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                TFLA_FRAG_A(a0, 0, 0, i, ks)
                TFLA_FRAG_B(b0, 0, 0, i, ks)
            }
        uint32_t so = 0;
        int landed = 3;         // phases that need nothing but the first two steps, which have arrived
        for (int t = k_begin; t < k_end; ++t) {
            TFLA_PHASE();
            TFLA_MUL(a0, b0, 0, 0, 0, 0, 0)
            TFLA_FRAG_B(b1, 1, so, 0, 0)
            TFLA_MUL(a0, b0, 0, 0, 0, 1, 0)
            TFLA_FRAG_B(b1, 1, so, 1, 0)
            TFLA_MUL(a0, b0, 0, 0, 1, 0, 0)
            TFLA_FRAG_B(b1, 1, so, 0, 1)
            TFLA_MUL(a0, b0, 0, 0, 1, 1, 0)
            TFLA_FRAG_B(b1, 1, so, 1, 1)
            TFLA_MUL(a0, b0, 0, 0, 0, 0, 1)
            TFLA_FRAG_B(b1, 1, so, 0, 2)
            TFLA_MUL(a0, b0, 0, 0, 0, 1, 1)
            TFLA_FRAG_B(b1, 1, so, 1, 2)
            TFLA_MUL(a0, b0, 0, 0, 1, 0, 1)
            TFLA_FRAG_B(b1, 1, so, 0, 3)
            TFLA_MUL(a0, b0, 0, 0, 1, 1, 1)
            TFLA_FRAG_B(b1, 1, so, 1, 3)
            TFLA_MUL(a0, b0, 0, 0, 0, 0, 2)
            TFLA_FRAG_A(a1, 1, so, 0, 0)
            TFLA_MUL(a0, b0, 0, 0, 0, 1, 2)
            oa.template issue<0>(0, la + rslot);
            TFLA_MUL(a0, b0, 0, 0, 1, 0, 2)
            TFLA_FRAG_A(a1, 1, so, 1, 0)
            TFLA_MUL(a0, b0, 0, 0, 1, 1, 2)
            oa.template issue<0>(1, la + rslot);
            TFLA_MUL(a0, b0, 0, 0, 0, 0, 3)
            TFLA_FRAG_A(a1, 1, so, 0, 1)
            TFLA_MUL(a0, b0, 0, 0, 0, 1, 3)
            oa.template issue<0>(2, la + rslot);
            TFLA_MUL(a0, b0, 0, 0, 1, 0, 3)
            TFLA_FRAG_A(a1, 1, so, 1, 1)
            TFLA_MUL(a0, b0, 0, 0, 1, 1, 3)
            oa.template issue<0>(3, la + rslot);
            TFLA_MUL(a0, b1, 0, 1, 0, 0, 0)
            TFLA_FRAG_A(a1, 1, so, 0, 2)
            TFLA_MUL(a0, b1, 0, 1, 0, 1, 0)
            ob.template issue<0>(0, lb + rslot);
            TFLA_MUL(a0, b1, 0, 1, 1, 0, 0)
            TFLA_FRAG_A(a1, 1, so, 1, 2)
            TFLA_MUL(a0, b1, 0, 1, 1, 1, 0)
            ob.template issue<0>(1, lb + rslot);
            TFLA_MUL(a0, b1, 0, 1, 0, 0, 1)
            TFLA_FRAG_A(a1, 1, so, 0, 3)
            TFLA_MUL(a0, b1, 0, 1, 0, 1, 1)
            ob.template issue<0>(2, lb + rslot);
            TFLA_MUL(a0, b1, 0, 1, 1, 0, 1)
            TFLA_FRAG_A(a1, 1, so, 1, 3)
            TFLA_MUL(a0, b1, 0, 1, 1, 1, 1)
            ob.template issue<0>(3, lb + rslot);
            TFLA_MUL(a0, b1, 0, 1, 0, 0, 2)
            TFLA_MUL(a0, b1, 0, 1, 0, 1, 2)
            TFLA_MUL(a0, b1, 0, 1, 1, 0, 2)
            TFLA_MUL(a0, b1, 0, 1, 1, 1, 2)
            TFLA_MUL(a0, b1, 0, 1, 0, 0, 3)
            TFLA_MUL(a0, b1, 0, 1, 0, 1, 3)
            TFLA_MUL(a0, b1, 0, 1, 1, 0, 3)
            TFLA_MUL(a0, b1, 0, 1, 1, 1, 3)
            so ^= SLOT;
            TFLA_PHASE();
            TFLA_MUL(a1, b0, 1, 0, 0, 0, 0)
            TFLA_FRAG_A(a0, 0, so, 0, 0)
            TFLA_MUL(a1, b0, 1, 0, 0, 1, 0)
            oa.template issue<1>(0, la + rslot + HALF);
            TFLA_MUL(a1, b0, 1, 0, 1, 0, 0)
            TFLA_FRAG_A(a0, 0, so, 1, 0)
            TFLA_MUL(a1, b0, 1, 0, 1, 1, 0)
            oa.template issue<1>(1, la + rslot + HALF);
            TFLA_MUL(a1, b0, 1, 0, 0, 0, 1)
            TFLA_FRAG_A(a0, 0, so, 0, 1)
            TFLA_MUL(a1, b0, 1, 0, 0, 1, 1)
            oa.template issue<1>(2, la + rslot + HALF);
            TFLA_MUL(a1, b0, 1, 0, 1, 0, 1)
            TFLA_FRAG_A(a0, 0, so, 1, 1)
            TFLA_MUL(a1, b0, 1, 0, 1, 1, 1)
            oa.template issue<1>(3, la + rslot + HALF);
            TFLA_MUL(a1, b0, 1, 0, 0, 0, 2)
            TFLA_FRAG_A(a0, 0, so, 0, 2)
            TFLA_MUL(a1, b0, 1, 0, 0, 1, 2)
            ob.template issue<1>(0, lb + rslot + HALF);
            TFLA_MUL(a1, b0, 1, 0, 1, 0, 2)
            TFLA_FRAG_A(a0, 0, so, 1, 2)
            TFLA_MUL(a1, b0, 1, 0, 1, 1, 2)
            ob.template issue<1>(1, lb + rslot + HALF);
            TFLA_MUL(a1, b0, 1, 0, 0, 0, 3)
            TFLA_FRAG_A(a0, 0, so, 0, 3)
            TFLA_MUL(a1, b0, 1, 0, 0, 1, 3)
            ob.template issue<1>(2, lb + rslot + HALF);
            TFLA_MUL(a1, b0, 1, 0, 1, 0, 3)
            TFLA_FRAG_A(a0, 0, so, 1, 3)
            TFLA_MUL(a1, b0, 1, 0, 1, 1, 3)
            ob.template issue<1>(3, lb + rslot + HALF);
            TFLA_MUL(a1, b1, 1, 1, 0, 0, 0)
            TFLA_FRAG_B(b0, 0, so, 0, 0)
            TFLA_MUL(a1, b1, 1, 1, 0, 1, 0)
            TFLA_FRAG_B(b0, 0, so, 1, 0)
            TFLA_MUL(a1, b1, 1, 1, 1, 0, 0)
            TFLA_FRAG_B(b0, 0, so, 0, 1)
            TFLA_MUL(a1, b1, 1, 1, 1, 1, 0)
            TFLA_FRAG_B(b0, 0, so, 1, 1)
            TFLA_MUL(a1, b1, 1, 1, 0, 0, 1)
            TFLA_FRAG_B(b0, 0, so, 0, 2)
            TFLA_MUL(a1, b1, 1, 1, 0, 1, 1)
            TFLA_FRAG_B(b0, 0, so, 1, 2)
            TFLA_MUL(a1, b1, 1, 1, 1, 0, 1)
            TFLA_FRAG_B(b0, 0, so, 0, 3)
            TFLA_MUL(a1, b1, 1, 1, 1, 1, 1)
            TFLA_FRAG_B(b0, 0, so, 1, 3)
            TFLA_MUL(a1, b1, 1, 1, 0, 0, 2)
            TFLA_MUL(a1, b1, 1, 1, 0, 1, 2)
            TFLA_MUL(a1, b1, 1, 1, 1, 0, 2)
            TFLA_MUL(a1, b1, 1, 1, 1, 1, 2)
            TFLA_NEXT();
            TFLA_MUL(a1, b1, 1, 1, 0, 0, 3)
            TFLA_MUL(a1, b1, 1, 1, 0, 1, 3)
            TFLA_MUL(a1, b1, 1, 1, 1, 0, 3)
            TFLA_MUL(a1, b1, 1, 1, 1, 1, 3)
        }
        // what was requested of steps behind the end has to have arrived before the memory is used anew
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        const GemmWork done = w;
        const long drow = row0 + wm * 128;
        const int dcol = col0 + wn * (PAIR ? 64 : 128);
        id += gridDim.x;
        const bool more = id < total;
        if (more) {
            take(id);
            start();
        }
        const bool full = wave_epilogue<bf16_t, EPI, PAIR, 4, 4>(a, done, drow, dcol, acc, lane);
        if (!more) break;
        // the requests are older than the epilogue's operations, so its last stores need not have arrived
        if (full) wait_vmcnt<16>();
        else wait_vmcnt<0>();
    }
#undef TFLA_NEXT
#undef TFLA_REQUEST
#undef TFLA_FRAG_A
#undef TFLA_FRAG_B
#undef TFLA_MUL
#undef TFLA_PHASE
}

}  // namespace tfla
