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

// Results.  The kernels compute the transposed blocks (weights as the first operand), so that lane (c = lane & 31, g = lane >> 5)
// holds of row c of a block the columns 8 q + 4 g + {0 .. 3} in registers 4 q ... 4 q + 3.  Two exchanges between the halves of
// a wavefront give lane (c, g) the eight consecutive columns 8 (q + g) ... of row c, for even q: no LDS, 16-byte stores.
__device__ __forceinline__ void eight_columns(const f32x16& acc, int q, float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float x = acc[4 * q + e], y = acc[4 * q + 4 + e];     // (a bit cast of a vector's element takes the first one)
        const auto p = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, y), false, false);
        const unsigned lo = p[0], hi = p[1];
        v[e] = __builtin_bit_cast(float, lo);
        v[4 + e] = __builtin_bit_cast(float, hi);
    }
}

// One wavefront's MB x NB blocks of 32 x 32 through the epilogue, 32 rows at a time.  row0, col0: first row and column of the
// results; PAIR: blocks 0, 2, ... hold the first matrix's columns col0, col0 + 32, ..., blocks 1, 3, ... the second's.
// The rows go round a loop that picks its registers by a switch: unrolled, the activations alone are 400 KB of code, and a
// wavefront that runs through it once waits for every line.
template <typename DT, int EPI, bool PAIR, int MB, int NB, bool FULL>
__device__ __forceinline__ void wave_epilogue_as(const GemmArgs& a, const GemmWork& w, long row0, int col0, f32x16 (&acc)[MB][NB], int lane) {
    constexpr int NG = PAIR ? NB : 2 * NB;
    const int planes = PAIR ? 2 : a.batch, c = lane & 31, g = lane >> 5;
    int rows = MB;
    asm("" : "+s"(rows));
#pragma unroll 1
    for (int mb = 0; mb < rows; ++mb) {
        f32x16 cur[NB];
#define TFLA_PICK(I)                                            \
    case I:                                                     \
        if constexpr (I < MB) {                                 \
            _Pragma("unroll") for (int j = 0; j < NB; ++j) cur[j] = acc[I][j]; \
        }                                                       \
        break;
        switch (mb) {
            TFLA_PICK(0) TFLA_PICK(1) TFLA_PICK(2) TFLA_PICK(3)
            default: __builtin_unreachable();
        }
#undef TFLA_PICK
        float v[NG][8], u[NG][8];
#pragma unroll
        for (int i = 0; i < NG; ++i) {
            const int nb = PAIR ? (i >> 1) * 2 : i >> 1, q = (i & 1) * 2;
            eight_columns(cur[nb], q, v[i]);
            if constexpr (PAIR) eight_columns(cur[nb + 1], q, u[i]);
        }
        const long m = row0 + mb * 32 + c;
        const int n = col0 + 8 * g;
        auto step = [](int i) { return (i >> 1) * 32 + (i & 1) * 16; };
        if constexpr (EPI == EPI_PART) {
#pragma unroll
            for (int i = 0; i < NG; ++i) {
                partial8<FULL>(a, planes, w.part, PAIR ? 0 : w.b, m, n + step(i), v[i]);
                if constexpr (PAIR) partial8<FULL>(a, planes, w.part, 1, m, n + step(i), u[i]);
            }
        } else {
            epilogue_groups<DT, EPI, NG, FULL>(a, w.b, m, n, step, v, u);
        }
    }
}
// (whole tiles without the checks of every row and column, so that loads and stores are not held up by branches)
// Returns whether that was so: at least 16 vector memory operations have been issued then.
template <typename DT, int EPI, bool PAIR, int MB, int NB>
__device__ __forceinline__ bool wave_epilogue(const GemmArgs& a, const GemmWork& w, long row0, int col0, f32x16 (&acc)[MB][NB], int lane) {
    const bool full = row0 + MB * 32 <= a.M && col0 + NB * (PAIR ? 16 : 32) <= a.N;
    if (full) wave_epilogue_as<DT, EPI, PAIR, MB, NB, true>(a, w, row0, col0, acc, lane);
    else wave_epilogue_as<DT, EPI, PAIR, MB, NB, false>(a, w, row0, col0, acc, lane);
    return full;
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
    __shared__ __align__(1024) char lds[2 * STAGE];
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
                for (int j = 0; j < NB; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(bf[j], af[i], acc[i][j], 0, 0, 0);
        }
    }
    wave_epilogue<bf16_t, EPI, PAIR, MB, NB>(a, w, row0 + wm * TM, col0 + wn * (PAIR ? TN / 2 : TN), acc, lane);
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
    constexpr int STAGE = (BM + BN) * LD;
    __shared__ __align__(16) float lds[2 * STAGE];
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
                for (int j = 0; j < NB; ++j) acc[i][j] = Elem<float>::mma(bf[j], af[i], acc[i][j]);
        }
        if (more) store(stage ^ 1);
        __syncthreads();
    }
    wave_epilogue<float, EPI, PAIR, MB, NB>(a, w, row0 + wm * TM, col0 + wn * (PAIR ? TN / 2 : TN), acc, lane);
}

}  // namespace tfla
