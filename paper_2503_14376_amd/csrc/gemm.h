// Matrix products of the residual block for gfx950: bf16 (v_mfma_f32_32x32x16_bf16) and fp32 (v_mfma_f32_32x32x2_f32), fp32
// accumulation.  See block_internal.h for what a product is and gemm_epilogue.h for what follows it.
#pragma once
#include "gemm_epilogue.h"
#include "lds_tiles.h"

namespace tfla {

// Workgroups go to the 8 XCDs in turn by their id; here every XCD gets a contiguous range of work, whatever the total.
__device__ __forceinline__ unsigned xcd_range(unsigned hw, unsigned total) {
    const unsigned x = hw & 7u, i = hw >> 3, q = total >> 3, r = total & 7u;
    return x * q + (x < r ? x : r) + i;
}
// Work item -> output tile, part of the contraction and result of a batch.  Within a band of GROUP tile rows the rows run
// fastest, so that the workgroups that run together on an XCD read few different rows and columns.
struct GemmWork { int tm, tn, part, b; };
template <int GROUP = 8> __device__ __forceinline__ GemmWork gemm_work(unsigned id, int tms, int tns, int split) {
    GemmWork w;
    const unsigned tiles = (unsigned)tms * tns;
    const unsigned pb = id / tiles, t = id % tiles;
    w.part = pb % split; w.b = pb / split;
    const unsigned band = t / (GROUP * tns), in = t % (GROUP * tns);
    const int rows = min(GROUP, tms - (int)band * GROUP);
    w.tm = band * GROUP + in % rows;
    w.tn = in / rows;
    return w;
}

// An accumulator block (32 rows x 32 columns per 16 registers) goes through LDS so that the epilogue has eight consecutive
// columns in a lane.  One wavefront's area: 32 rows of C + 4 floats.
template <int C> struct EpiStage {
    static constexpr int LD = C + 4, FLOATS = 32 * LD;
    static __device__ __forceinline__ void put(float* area, const f32x16& acc, int col0, int lane) {
        const int c = lane & 31, g = lane >> 5;
#pragma unroll
        for (int v = 0; v < 16; ++v) area[acc_row(v, g) * LD + col0 + c] = acc[v];
    }
    static __device__ __forceinline__ void get(const float* area, int row, int col, float (&x)[8]) {
        const f32x4 a = *reinterpret_cast<const f32x4*>(area + row * LD + col), b = *reinterpret_cast<const f32x4*>(area + row * LD + col + 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) { x[e] = a[e]; x[4 + e] = b[e]; }
    }
};

// One wavefront's MB x NB blocks of 32 x 32 through the epilogue.  row0, col0: first row and (without PAIR) first column;
// PAIR: blocks 0, 2, ... hold the first matrix's columns col0, col0 + 32, ..., blocks 1, 3, ... the second's.
template <typename DT, int EPI, bool PAIR, int MB, int NB>
__device__ __forceinline__ void wave_epilogue(const GemmArgs& a, const GemmWork& w, long row0, int col0, f32x16 (&acc)[MB][NB], float* area,
                                              int lane) {
    constexpr int C = NB * 32;
    typedef EpiStage<C> S;
    constexpr int OC = PAIR ? C / 2 : C, LPR = OC / 8, RPP = 64 / LPR;      // output columns, lanes per row, rows per pass
    const int planes = PAIR ? 2 : a.batch;
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) S::put(area, acc[mb][nb], nb * 32, lane);
        // (the area is this wavefront's own: only its own writes have to have arrived)
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll 1
        for (int p = 0; p < 32 / RPP; ++p) {        // (a loop: unrolled, the activations alone are thousands of instructions)
            const int r = p * RPP + lane / LPR, c = (lane % LPR) * 8;
            float v[8], u[8];
            if constexpr (PAIR) {
                const int lc = (c / 32) * 64 + (c % 32);
                S::get(area, r, lc, v);
                S::get(area, r, lc + 32, u);
            } else {
                S::get(area, r, c, v);
            }
            const long m = row0 + mb * 32 + r;
            if constexpr (EPI == EPI_PART) {
                partial8(a, planes, w.part, PAIR ? 0 : w.b, m, col0 + c, v);
                if constexpr (PAIR) partial8(a, planes, w.part, 1, m, col0 + c, u);
            } else {
                epilogue8<DT, EPI>(a, w.b, m, col0 + c, v, u);
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
}

// Bytes of a tile (rows_left x cols_left of the tensor from its first element on, at most ROWS rows) that may be read.
template <int ROWS> __device__ __forceinline__ uint32_t tile_bytes(long rows_left, int cols_left, long ld) {
    const int r = rows_left < ROWS ? (int)rows_left : ROWS;
    return (r > 0 && cols_left > 0) ? (uint32_t)((r - 1) * ld * 2) + 2u * (uint32_t)cols_left : 0u;
}

// One operand of a bf16 product: tiles of ROWS output rows (or columns) x 64 contraction steps.  Plain: [ROWS][64] in LDS;
// transposed: [64][ROWS], read by the transposing LDS reads.
template <int ROWS, bool TR, int NT> struct OperandTile {
    typedef DmaTile<TR ? 64 : ROWS, TR ? ROWS : 64, NT, TR ? SWZ_T : SWZ_K> Dma;
    Dma dma;
    const bf16_t* base; long ld; long rows_left; int K8; int cols_left;
    // base: element (row0, 0) or, transposed, (0, row0); extent: rows of the operand; K: contraction length
    __device__ __forceinline__ void init(const void* p, long ld_, long row0, long extent, int K, int tid) {
        ld = ld_;
        base = reinterpret_cast<const bf16_t*>(p) + (TR ? row0 : row0 * ld);
        // whole groups of eight: what lies behind the extent belongs to the row's padding
        rows_left = extent - row0; K8 = TR ? K : (K + 7) & ~7;
        cols_left = TR ? (int)((rows_left + 7) & ~7l) : 0;
        dma.init(ld, tid);
        if (TR) dma.bound_columns(cols_left, tid);
    }
    __device__ __forceinline__ void issue(int k0, uint32_t lds, int tid) const {
        if constexpr (TR) {
            const uint32_t bytes = tile_bytes<64>(K8 - k0, cols_left, ld);
            dma.template issue_bounded<false>(base + (long)k0 * ld, bytes, ROWS, lds, tid);
        } else {
            const uint32_t bytes = tile_bytes<ROWS>(rows_left, K8 - k0, ld);
            dma.template issue_bounded<false>(base + k0, bytes, K8 - k0, lds, tid);
        }
    }
};

// Fragments of an operand tile for one wavefront: block b = rows 32 b ... of the wavefront's part, which starts at row0 (a
// multiple of 32).
template <int ROWS, bool TR> struct OperandFrags;
template <int ROWS> struct OperandFrags<ROWS, false> {
    KFragReader<64> r;
    __device__ __forceinline__ void init(int lane) { r.init(lane & 31, lane >> 5); }
    __device__ __forceinline__ bf16x8 load(const char* tile, int ks, int row0) const { return r.load(tile + row0 * 128, ks, 0); }
};
template <int ROWS> struct OperandFrags<ROWS, true> {
    int lane;
    __device__ __forceinline__ void init(int l) { lane = l; }
    __device__ __forceinline__ bf16x8 load(const char* tile, int ks, int row0) const {
        return TFragReader<ROWS>::load_at(tile, TFragReader<ROWS>::offset_of(lane, 8, row0 >> 5), ks * 16, ks * 16 + 4);
    }
};

// Tile BM x BN, WM x WN wavefronts, contraction in steps of 64 through two LDS stages filled asynchronously.
// PAIR: the columns of a tile are BN / 2 of B[0] and the same BN / 2 of B[1], wavefront by wavefront.
template <int BM, int BN, int WM, int WN, bool ATR, bool BTR, bool PAIR, int EPI>
__global__ void __launch_bounds__(WM* WN * 64) gemm_bf16_kernel(GemmArgs a, int tms, int tns) {
    constexpr int NT = WM * WN * 64, TM = BM / WM, TN = BN / WN, MB = TM / 32, NB = TN / 32, BNO = PAIR ? BN / 2 : BN;
    static_assert(!PAIR || !BTR, "pairs are plain operands");
    constexpr int ABYTES = BM * 128, BBYTES = BN * 128, STAGE = ABYTES + BBYTES;
    constexpr int EPIB = WM * WN * EpiStage<TN>::FLOATS * 4, LDS = 2 * STAGE > EPIB ? 2 * STAGE : EPIB;
    __shared__ __align__(1024) char lds[LDS];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / WN, wn = wave % WN;
    const GemmWork w = gemm_work(xcd_range(blockIdx.x, gridDim.x), tms, tns, a.split);
    const long row0 = (long)w.tm * BM;
    const int col0 = w.tn * BNO;

    const int ksteps = (a.K + 63) / 64, all = ksteps * a.segs;
    const int per = (all + a.split - 1) / a.split, k_begin = w.part * per, k_end = min(all, k_begin + per);

    OperandTile<BM, ATR, NT> ta;
    OperandTile<BNO, BTR, NT> tb, tb2;
    ta.init(a.A[w.b], a.lda, row0, a.M, a.K, tid);
    tb.init(a.B[0], a.ldb, col0, a.N, a.K, tid);
    if constexpr (PAIR) tb2.init(a.B[1], a.ldb, col0, a.N, a.K, tid);
    // the second segment's operands lie this many bytes away from the first's
    const uintptr_t hopA = reinterpret_cast<uintptr_t>(a.A[1]) - reinterpret_cast<uintptr_t>(a.A[0]);
    const uintptr_t hopB = reinterpret_cast<uintptr_t>(a.B[1]) - reinterpret_cast<uintptr_t>(a.B[0]);
    const uint32_t la = lds_addr(lds);
    int kt = k_begin;           // next step to request
    auto request = [&](int stage) {
        const bool second = kt >= ksteps;
        const int k0 = (second ? kt - ksteps : kt) * 64;
        OperandTile<BM, ATR, NT> xa = ta;
        OperandTile<BNO, BTR, NT> xb = tb;
        if (second) {
            xa.base = reinterpret_cast<const bf16_t*>(reinterpret_cast<uintptr_t>(xa.base) + hopA);
            xb.base = reinterpret_cast<const bf16_t*>(reinterpret_cast<uintptr_t>(xb.base) + hopB);
        }
        xa.issue(k0, la + stage * STAGE, tid);
        xb.issue(k0, la + stage * STAGE + ABYTES, tid);
        if constexpr (PAIR) tb2.issue(k0, la + stage * STAGE + ABYTES + BBYTES / 2, tid);
        ++kt;
    };

    f32x16 acc[MB][NB];
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.0f;
    OperandFrags<BM, ATR> fa;
    OperandFrags<BNO, BTR> fb;
    fa.init(lane);
    fb.init(lane);

    if (kt < k_end) request(0);
    for (int k = k_begin, stage = 0; k < k_end; ++k, stage ^= 1) {
        wait_vmcnt<0>();
        barrier_nofence();
        if (kt < k_end) request(stage ^ 1);
        const char* A = lds + stage * STAGE;
        const char* B = A + ABYTES;
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
            bf16x8 af[MB], bf[NB];
#pragma unroll
            for (int i = 0; i < MB; ++i) af[i] = fa.load(A, ks, wm * TM + i * 32);
#pragma unroll
            for (int j = 0; j < NB; ++j)
                bf[j] = PAIR ? fb.load(B + (j & 1) * (BBYTES / 2), ks, wn * (TN / 2) + (j >> 1) * 32) : fb.load(B, ks, wn * TN + j * 32);
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int j = 0; j < NB; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(af[i], bf[j], acc[i][j], 0, 0, 0);
        }
    }
    wait_vmcnt<0>();
    __syncthreads();
    wave_epilogue<bf16_t, EPI, PAIR, MB, NB>(a, w, row0 + wm * TM, col0 + wn * (PAIR ? TN / 2 : TN), acc,
                                             reinterpret_cast<float*>(lds) + wave * EpiStage<TN>::FLOATS, lane);
}

// fp32 products: tiles through registers into LDS, contraction steps of 32, the contraction index contiguous per LDS row
// (transposed operands are turned on the way).
template <int ROWS, bool TR, int NT> struct OperandTileF32;
template <int ROWS, int NT> struct OperandTileF32<ROWS, false, NT> {
    RowsPrefetch<float, ROWS, 32, NT> r;
    __device__ __forceinline__ void load(const float* p, long ld, long row0, long extent, int k0, int K, int tid) {
        const long left = extent - row0;
        r.template load<true>(p + row0 * ld + k0, ld, tid, left < ROWS ? (int)left : ROWS, K - k0);
    }
    __device__ __forceinline__ void store(float* lds, int tid) const { r.store(lds, 36, tid); }
};
template <int ROWS, int NT> struct OperandTileF32<ROWS, true, NT> {
    TrPrefetch<float, 32, ROWS, NT, false> r;
    __device__ __forceinline__ void load(const float* p, long ld, long row0, long extent, int k0, int K, int tid) {
        const long left = extent - row0;
        r.template load<true>(p + (long)k0 * ld + row0, ld, tid, K - k0, left < ROWS ? (int)left : ROWS);
    }
    __device__ __forceinline__ void store(float* lds, int tid) const { r.store(lds, 36, tid); }
};

template <int BM, int BN, int WM, int WN, bool ATR, bool BTR, bool PAIR, int EPI>
__global__ void __launch_bounds__(WM* WN * 64) gemm_f32_kernel(GemmArgs a, int tms, int tns) {
    constexpr int NT = WM * WN * 64, TM = BM / WM, TN = BN / WN, MB = TM / 32, NB = TN / 32, BNO = PAIR ? BN / 2 : BN, LD = 36;
    static_assert(!PAIR || !BTR, "pairs are plain operands");
    constexpr int STAGE = (BM + BN) * LD, EPIF = WM * WN * EpiStage<TN>::FLOATS;
    __shared__ __align__(16) float lds[2 * STAGE > EPIF ? 2 * STAGE : EPIF];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / WN, wn = wave % WN, l32 = lane & 31, g = lane >> 5;
    const GemmWork w = gemm_work(xcd_range(blockIdx.x, gridDim.x), tms, tns, a.split);
    const long row0 = (long)w.tm * BM;
    const int col0 = w.tn * BNO;
    const int ksteps = (a.K + 31) / 32, all = ksteps * a.segs;
    const int per = (all + a.split - 1) / a.split, k_begin = w.part * per, k_end = min(all, k_begin + per);
    // (plain operands are read in groups of four: what lies behind K is the row's padding)
    const int K4 = (a.K + 3) & ~3;

    OperandTileF32<BM, ATR, NT> ta;
    OperandTileF32<BNO, BTR, NT> tb, tb2;
    auto load = [&](int kt) {
        const int seg = kt >= ksteps ? 1 : 0, k0 = (kt - seg * ksteps) * 32;
        ta.load(reinterpret_cast<const float*>(seg ? a.A[1] : a.A[w.b]), a.lda, row0, a.M, k0, ATR ? a.K : K4, tid);
        tb.load(reinterpret_cast<const float*>(a.B[seg]), a.ldb, col0, a.N, k0, BTR ? a.K : K4, tid);
        if constexpr (PAIR) tb2.load(reinterpret_cast<const float*>(a.B[1]), a.ldb, col0, a.N, k0, K4, tid);
    };
    auto store = [&](int stage) {
        float* p = lds + stage * STAGE;
        ta.store(p, tid);
        tb.store(p + BM * LD, tid);
        if constexpr (PAIR) tb2.store(p + (BM + BNO) * LD, tid);
    };
    f32x16 acc[MB][NB];
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.0f;
    if (k_begin < k_end) {
        load(k_begin);
        store(0);
    }
    __syncthreads();
    for (int k = k_begin, stage = 0; k < k_end; ++k, stage ^= 1) {
        const bool more = k + 1 < k_end;
        if (more) load(k + 1);
        const float* A = lds + stage * STAGE;
        const float* B = A + BM * LD;
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            Elem<float>::frag af[MB], bf[NB];
#pragma unroll
            for (int i = 0; i < MB; ++i) af[i] = Elem<float>::load(A + (wm * TM + i * 32 + l32) * LD + ks * 16 + g * 8);
#pragma unroll
            for (int j = 0; j < NB; ++j) {
                const int r = PAIR ? (j & 1) * BNO + wn * (TN / 2) + (j >> 1) * 32 : wn * TN + j * 32;
                bf[j] = Elem<float>::load(B + (r + l32) * LD + ks * 16 + g * 8);
            }
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int j = 0; j < NB; ++j) acc[i][j] = Elem<float>::mma(af[i], bf[j], acc[i][j]);
        }
        if (more) store(stage ^ 1);
        __syncthreads();
    }
    wave_epilogue<float, EPI, PAIR, MB, NB>(a, w, row0 + wm * TM, col0 + wn * (PAIR ? TN / 2 : TN), acc, lds + wave * EpiStage<TN>::FLOATS,
                                            lane);
}

}  // namespace tfla
