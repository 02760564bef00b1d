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

// Results.  Partial results are stored as they leave the matrix unit: lane (c = lane & 31, g = lane >> 5) holds of column c of a
// block the rows acc_row(v, g), so that a store writes whole rows of 32 floats.  For everything else the kernels compute the
// transposed blocks (the second operand first), so that the lane holds of row c the columns 8 q + 4 g + {0 .. 3} in registers
// 4 q ... 4 q + 3.  Exchanges between the halves, then between the quarters of a wavefront give it eight consecutive columns:
// x: row c % 16, y: row c % 16 + 16, columns 16 (c / 16) + 8 g ...; a store writes 64 consecutive bytes of 16 rows in bf16.
// (Without the second exchange 32 bytes of 32 rows, without any, 16-byte pieces; through LDS the turn took longer than the stores.)
template <bool WIDE> __device__ __forceinline__ void lane_swap(float& x, float& y) {
    const unsigned a = __builtin_bit_cast(unsigned, x), b = __builtin_bit_cast(unsigned, y);
    const auto p = WIDE ? __builtin_amdgcn_permlane32_swap(a, b, false, false) : __builtin_amdgcn_permlane16_swap(a, b, false, false);
    const unsigned lo = p[0], hi = p[1];
    x = __builtin_bit_cast(float, lo);
    y = __builtin_bit_cast(float, hi);
}
__device__ __forceinline__ void eight_columns(const f32x16& acc, float (&x)[8], float (&y)[8]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        x[e] = acc[e]; x[4 + e] = acc[4 + e];
        y[e] = acc[8 + e]; y[4 + e] = acc[12 + e];
        lane_swap<true>(x[e], x[4 + e]);
        lane_swap<true>(y[e], y[4 + e]);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) lane_swap<false>(x[e], y[e]);
}
// the product of two fragments in the orientation that the epilogue wants
template <int EPI> __device__ __forceinline__ f32x16 mma_bf16(const bf16x8& a, const bf16x8& b, const f32x16& c) {
    return EPI == EPI_PART ? __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0) : __builtin_amdgcn_mfma_f32_32x32x16_bf16(b, a, c, 0, 0, 0);
}

// One wavefront's MB x NB blocks of 32 x 32 through the epilogue, 32 rows at a time.  row0, col0: first row and column of the
// results; PAIR: blocks 0, 2, ... hold the first matrix's columns col0, col0 + 32, ..., blocks 1, 3, ... the second's.
// The rows go round a loop that picks its registers by a switch: unrolled, the activations alone are 400 KB of code, and a
// wavefront that runs through it once waits for every line.
template <typename DT, int EPI, bool PAIR, int MB, int NB, bool FULL>
__device__ __forceinline__ void wave_epilogue_as(const GemmArgs& a, const GemmWork& w, long row0, int col0, f32x16 (&acc)[MB][NB], int lane) {
    constexpr int NG = PAIR ? NB : 2 * NB;
    const int c = lane & 31, g = lane >> 5;
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
        const long m0 = row0 + mb * 32;
        if constexpr (EPI == EPI_PART) {
            const int planes = PAIR ? 2 : a.batch;
#pragma unroll
            for (int j = 0; j < NB; ++j) {
                const int n = col0 + (PAIR ? j / 2 : j) * 32 + c;
                float* p = partial_plane(a, planes, w.part, PAIR ? j & 1 : w.b) + m0 * a.ld_part + n;
#pragma unroll
                for (int v = 0; v < 16; ++v) {
                    const int r = acc_row(v, g);
                    if (FULL || (m0 + r < a.M && n < a.N)) p[r * a.ld_part] = cur[j][v];
                }
            }
        } else {
            float v[NG][8], u[NG][8];
#pragma unroll
            for (int j = 0; j < NB; j += PAIR ? 2 : 1) {
                constexpr int F = PAIR ? 1 : 2;
                eight_columns(cur[j], v[j * F], v[j * F + 1]);
                if constexpr (PAIR) eight_columns(cur[j + 1], u[j], u[j + 1]);
            }
            epilogue_groups<DT, EPI, NG, FULL>(a, w.b, m0 + (c & 15), col0 + (c >> 4) * 16 + 8 * g, [](int i) { return (i & 1) * 16; },
                                               [](int i) { return (i >> 1) * 32; }, v, u);
        }
    }
}
// (whole tiles without the checks of every row and column, so that loads and stores are not held up by branches)
// Returns whether that was so: every lane has stored MB * NB (PAIR: half that) times 32 bytes or more then.
template <typename DT, int EPI, bool PAIR, int MB, int NB>
__device__ __forceinline__ bool wave_epilogue(const GemmArgs& a, const GemmWork& w, long row0, int col0, f32x16 (&acc)[MB][NB], int lane) {
    const bool full = row0 + MB * 32 <= a.M && col0 + NB * (PAIR ? 16 : 32) <= a.N;
    if (full) wave_epilogue_as<DT, EPI, PAIR, MB, NB, true>(a, w, row0, col0, acc, lane);
    else wave_epilogue_as<DT, EPI, PAIR, MB, NB, false>(a, w, row0, col0, acc, lane);
    return full;
}

// The stream of one operand's tiles into LDS: HALVES parts of ROWS output rows (or columns) x 64 contraction steps each, filled by
// requests of NT threads.  Plain: [ROWS][64] in LDS; transposed: [64][ROWS], read by the transposing LDS reads.  Local row r of
// a part stands for row (r / G) 2 G + r % G behind the part's first row (G = ROWS: itself); part h starts at row h G, or with
// PAIR at the first row of matrix h.  The buffer descriptors are kept ready and moved on by a step at a time; everything else
// about them is found anew (set) only at the steps where it changes: the last step of a contraction that is no multiple of 64,
// the second segment, the end, behind which nothing is requested (bounds of zero bytes) and LDS receives zeros.
template <int ROWS, bool TR, int G, int NT, int HALVES, bool PAIR> struct OperandStream {
    typedef DmaTile<TR ? 64 : ROWS, TR ? ROWS : 64, NT, TR ? SWZ_T : SWZ_K> Shape;
    static constexpr int CPR = Shape::CPR, N = Shape::N, NW = NT / 64, BYTES = ROWS * 128;
    static constexpr long SPAN = G == ROWS ? ROWS : 2 * ROWS;
    static constexpr uint32_t BEHIND = 0x40000000u;       // an offset beyond every bound
    u32x4 d[HALVES];            // descriptors of the parts at the next step
    uint32_t goff[N], hop;      // byte offsets of this lane; bytes from step to step
    __device__ __forceinline__ void init(long ld, int tid) {
        const int lane = tid & 63, wave = tid >> 6;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int q = (wave + j * NW) * 64 + lane, r = q / CPR, c = ((q % CPR) ^ swz_mask<TR ? SWZ_T : SWZ_K, CPR>(r)) * 8;
            const int row = TR || G == ROWS ? r : (r / G) * 2 * G + r % G, col = TR && G != ROWS ? (c / G) * 2 * G + c % G : c;
            goff[j] = (uint32_t)((row * ld + col) * 2);
        }
        hop = (uint32_t)(TR ? 128 * ld : 128);
    }
    // p0, p1: the matrices of the parts; first: the operand's first row in the tile, of `extent`; K: contraction length; steps from
    // k0 on.  Columns behind the end of a transposed operand's rows are other rows' values: they meet results that are not
    // stored.
    __device__ __forceinline__ void set(const void* p0, const void* p1, long ld, long first, long extent, int K, int k0, bool exists, int tid) {
#pragma unroll
        for (int h = 0; h < HALVES; ++h) {
            const long at = first + (PAIR ? 0 : h * G), left = extent - at;
            const long rows = TR ? (K - k0 < 64 ? K - k0 : 64) : (left < SPAN ? left : SPAN);
            // whole groups of eight columns: what lies behind the extent belongs to the row's padding
            const int K8 = (K + 7) & ~7, cols = TR ? (int)(left < SPAN ? (left + 7) & ~7l : SPAN) : (K8 - k0 < 64 ? K8 - k0 : 64);
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
                const int q = (wave + j * NW) * 64 + lane, c = ((q % CPR) ^ swz_mask<SWZ_K, CPR>(q / CPR)) * 8;
                goff[j] = (goff[j] & (BEHIND - 1)) | (c < left ? 0u : BEHIND);
            }
        }
    }
    template <int STEPS> __device__ __forceinline__ void advance() {
#pragma unroll
        for (int h = 0; h < HALVES; ++h) {
            const uint64_t b = ((uint64_t)d[h][1] << 32 | d[h][0]) + (uint64_t)hop * STEPS;
            d[h][0] = (uint32_t)b;
            d[h][1] = (uint32_t)(b >> 32);
        }
    }
    // request j of part H; lds: LDS address of the part plus 1024 times the wavefront
    template <int H> __device__ __forceinline__ void issue(int j, uint32_t lds) const {
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                     :: "s"(lds + j * NW * 1024), "v"(goff[j]), "s"(d[H]) : "m0");
    }
    template <int H> __device__ __forceinline__ void issue_all(uint32_t lds) const {
#pragma unroll
        for (int j = 0; j < N; ++j) issue<H>(j, lds);
    }
};

// Which step of a tile's contraction the operands' streams stand at.
// STRIDE: steps from one that is requested to the next.
template <bool PAIR, int STRIDE> struct StepStream {
    int at, change, k_end, ksteps;      // next step, the first at which the descriptors change by more than a stride
    template <typename OA, typename OB>
    __device__ __forceinline__ void find(const GemmArgs& a, const GemmWork& w, long row0, int col0, OA& oa, OB& ob, int tid) {
        const bool on = at < k_end, second = at >= ksteps;
        const int k0 = on ? (second ? at - ksteps : at) * 64 : 0;
        const void* pa = a.A[second ? 1 : w.b];
        const void* pb = a.B[second && !PAIR ? 1 : 0];
        oa.set(pa, pa, a.lda, row0, a.M, a.K, k0, on, tid);
        ob.set(pb, PAIR ? a.B[1] : pb, a.ldb, col0, a.N, a.K, k0, on, tid);
        const int seg_end = second ? 2 * ksteps : ksteps, whole = seg_end - (a.K % 64 != 0);
        change = !on ? 0x7fffffff : min(k_end, at < whole ? whole : seg_end);
    }
    template <typename OA, typename OB>
    __device__ __forceinline__ void next(const GemmArgs& a, const GemmWork& w, long row0, int col0, OA& oa, OB& ob, int tid) {
        at += STRIDE;
        oa.template advance<STRIDE>();
        ob.template advance<STRIDE>();
        if (at >= change) find(a, w, row0, col0, oa, ob, tid);
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

// Joining the sums of wavefronts that divide a contraction: wavefront `slot` (-1: none) leaves its blocks, another adds them.
template <int MB, int NB> __device__ __forceinline__ void join_put(f32x4* area, const f32x16 (&acc)[MB][NB], int slot, int lane) {
    if (slot < 0) return;
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                area[((slot * MB + i) * NB + j) * 256 + q * 64 + lane] =
                    f32x4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
}
template <int MB, int NB> __device__ __forceinline__ void join_add(const f32x4* area, f32x16 (&acc)[MB][NB], int slot, int lane) {
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const f32x4 t = area[((slot * MB + i) * NB + j) * 256 + q * 64 + lane];
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i][j][4 * q + e] += t[e];
            }
}

// Tile BM x BN, WM x WN wavefronts, contraction in steps of 64 through S LDS stages, S - 1 of them under way.  KG such groups of
// wavefronts take the steps in turn, each through stages of its own, and meet in LDS at the end: where a launch has no more
// than one workgroup per CU, a wavefront per SIMD spends a step on issuing its instructions (64 x 64 tiles: 0.29 us, with two
// wavefronts per SIMD 0.2).  PAIR: the columns of a tile are BN / 2 of B[0] and the same BN / 2 of B[1], wavefront by wavefront.
// id, total: which of the product's workgroups this is.
template <int BM, int BN, int WM, int WN, int S, int KG> constexpr int gemm_bf16_lds = KG * S * (BM + BN) * 128;
template <int BM, int BN, int WM, int WN, int S, int KG, bool ATR, bool BTR, bool PAIR, int EPI>
__device__ __forceinline__ void gemm_bf16(const GemmArgs& a, int tms, int tns, unsigned id, unsigned total, char* lds) {
    constexpr int NT = WM * WN * 64, TM = BM / WM, TN = BN / WN, MB = TM / 32, NB = TN / 32, BNO = PAIR ? BN / 2 : BN;
    static_assert(!PAIR || !BTR, "pairs are plain operands");
    constexpr int ABYTES = BM * 128, BBYTES = BN * 128, STAGE = ABYTES + BBYTES;
    constexpr int JOIN = (KG - 1) * WM * WN * MB * NB * 4096;
    static_assert(JOIN <= KG * S * STAGE, "the groups' results fit the stages");
    const int tid = threadIdx.x % NT, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int group = KG == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / NT);
    const int wm = wave / WN, wn = wave % WN;
    const GemmWork w = gemm_work(xcd_range(id, total), tms, tns, a.split);
    const long row0 = (long)w.tm * BM;
    const int col0 = w.tn * BNO;

    OperandStream<BM, ATR, BM, NT, 1, false> oa;
    OperandStream<BNO, BTR, BNO, NT, PAIR ? 2 : 1, PAIR> ob;
    constexpr int LOADS = oa.N + (PAIR ? 2 : 1) * ob.N;     // requests of a wavefront per step
    StepStream<PAIR, KG> st;
    oa.init(a.lda, tid);
    ob.init(a.ldb, tid);
    st.ksteps = (a.K + 63) / 64;
    const int all = st.ksteps * a.segs, per = (all + a.split - 1) / a.split;
    const int k_begin = w.part * per;
    st.at = k_begin + group;
    st.k_end = min(all, k_begin + per);
    st.find(a, w, row0, col0, oa, ob, tid);
    char* ring = lds + group * S * STAGE;
    const uint32_t la = lds_addr(ring) + wave * 1024, lb = la + ABYTES;
    auto request = [&](uint32_t off) {
        oa.template issue_all<0>(la + off);
        ob.template issue_all<0>(lb + off);
        if constexpr (PAIR) ob.template issue_all<1>(lb + BBYTES / 2 + off);
        st.next(a, w, row0, col0, oa, ob, tid);
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

#pragma unroll
    for (int q = 0; q < S - 1; ++q) request(q * STAGE);
    uint32_t off = 0, next = (S - 1) * STAGE;
    for (int k = k_begin; k < st.k_end; k += KG) {
        wait_vmcnt<(S - 2) * LOADS>();
        // (the reads of the stage that is requested next have to be over, not only begun, when the wavefronts meet)
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        const char* A = ring + off;
        const char* B = A + ABYTES;
        bf16x8 af[4][MB], bf[4][NB];
        auto read = [&](int ks) {
#pragma unroll
            for (int i = 0; i < MB; ++i) af[ks][i] = fa.load(A, ks, wm * TM + i * 32);
#pragma unroll
            for (int j = 0; j < NB; ++j)
                bf[ks][j] = PAIR ? fb.load(B + (j & 1) * (BBYTES / 2), ks, wn * (TN / 2) + (j >> 1) * 32) : fb.load(B, ks, wn * TN + j * 32);
        };
        auto multiply = [&](int ks) {
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int j = 0; j < NB; ++j) acc[i][j] = mma_bf16<EPI>(af[ks][i], bf[ks][j], acc[i][j]);
        };
        // Plain operands: all fragments are on their way while the requests are issued (2000 x 4096 x 4096 in 128 x 128 tiles
        // 87 -> 64 us).  Transposed ones take twice the reads: a quarter of the step at a time (2048 x 2048 x 1024, both
        // backward products, 50.6 -> 44.9).
        if constexpr (!ATR && !BTR) {
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) read(ks);
            __builtin_amdgcn_sched_barrier(0);
            request(next);
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) multiply(ks);
        } else {
            request(next);
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) {
                read(ks);
                multiply(ks);
            }
        }
        next = off;
        off = off == (S - 1) * STAGE ? 0 : off + STAGE;
    }
    wait_vmcnt<0>();        // (what was requested of steps behind the end writes LDS too)
    if constexpr (KG > 1) {
        // the other groups' sums, in the order of the groups
        __syncthreads();
        f32x4* area = reinterpret_cast<f32x4*>(lds);
        join_put<MB, NB>(area, acc, group > 0 ? (group - 1) * WM * WN + wave : -1, lane);
        __syncthreads();
        if (group > 0) return;
#pragma unroll
        for (int p = 0; p < KG - 1; ++p) join_add<MB, NB>(area, acc, p * WM * WN + wave, lane);
    }
    wave_epilogue<bf16_t, EPI, PAIR, MB, NB>(a, w, row0 + wm * TM, col0 + wn * (PAIR ? TN / 2 : TN), acc, lane);
}

template <int BM, int BN, int WM, int WN, int S, int KG, bool ATR, bool BTR, bool PAIR, int EPI>
__global__ void __launch_bounds__(KG* WM* WN * 64, 2) gemm_bf16_kernel(GemmArgs a, int tms, int tns) {
    __shared__ __align__(1024) char lds[gemm_bf16_lds<BM, BN, WM, WN, S, KG>];
    gemm_bf16<BM, BN, WM, WN, S, KG, ATR, BTR, PAIR, EPI>(a, tms, tns, blockIdx.x, gridDim.x, lds);
}
// Both products of a small backward pass, dx = dz W and dw = dz^T x, in one launch: nx workgroups from x0 on take dx.  Those
// with the longer contraction come first, so that the shorter ones fill the end (2392 x 656 x 800 25.5 us against 27.1).
struct BothGrid { int xms, xns, wms, wns; unsigned nx, x0; };
template <int BM, int BN, int WM, int WN, int S, int KG>
__global__ void __launch_bounds__(KG* WM* WN * 64, 2) gemm_bf16_both_kernel(GemmArgs x, GemmArgs w, BothGrid n) {
    __shared__ __align__(1024) char lds[gemm_bf16_lds<BM, BN, WM, WN, S, KG>];
    const unsigned i = blockIdx.x;
    if (i >= n.x0 && i < n.x0 + n.nx) gemm_bf16<BM, BN, WM, WN, S, KG, false, true, false, EPI_STORE>(x, n.xms, n.xns, i - n.x0, n.nx, lds);
    else gemm_bf16<BM, BN, WM, WN, S, KG, true, true, false, EPI_STORE>(w, n.wms, n.wns, i < n.x0 ? i : i - n.nx, gridDim.x - n.nx, lds);
}

// fp32 products: tiles through registers into two LDS stages, contraction steps of STEP.  The matrix unit takes 64 clocks for
// 2 x 32 x 32 products of fp32, a sixteenth of its bf16 rate, so LDS never bounds it: what does is how many other instructions
// its wavefronts have to issue (4096^3: 993 us, 138 TFLOP/s; backward 2060).  So tiles keep the order that they have in memory (plain: rows of STEP, fragments by 16-byte reads;
// transposed: rows of ROWS, fragments value by value), and loads go through buffer descriptors, whose bounds give the zeros
// behind the ends.  WM x WN wavefronts with WK each: those divide a step's contraction and meet in LDS at the end, for products
// of few tiles.
template <int ROWS, bool TR, int STEP, int NT> struct OperandTileF32 {
    static constexpr int R = TR ? STEP : ROWS, C = TR ? ROWS : STEP, CPR = C / 4, N = R * CPR / NT, LD = C + 4, FLOATS = R * LD;
    static_assert(R * CPR % NT == 0, "whole loads per thread");
    struct Regs { u32x4 r[N]; };
    uint32_t goff[N];
    __device__ __forceinline__ void init(long ld, int tid) {
#pragma unroll
        for (int i = 0; i < N; ++i) goff[i] = (uint32_t)(((tid + i * NT) / CPR * ld + (tid + i * NT) % CPR * 4) * 4);
    }
    // p: the matrix; first: its first row (column) in the tile, of `extent`; K: contraction length.  Rows may begin at any
    // element: these loads want no more than 4 bytes' alignment, and their bounds hold word by word.  Columns behind the end of a
    // transposed operand's rows are other rows' values: they meet results that are not stored.
    __device__ __forceinline__ void load(Regs& to, const void* p, long ld, long first, long extent, int k0, int K, int tid) const {
        const long left = extent - first, rows = TR ? (K - k0 < STEP ? K - k0 : STEP) : (left < ROWS ? left : ROWS);
        const int cols = TR ? (int)(left < ROWS ? left : ROWS) : (K - k0 < STEP ? K - k0 : STEP);
        const float* base = reinterpret_cast<const float*>(p) + (TR ? k0 * ld + first : first * ld + k0);
        const int bytes = rows > 0 && cols > 0 ? (int)((rows - 1) * ld * 4) + 4 * cols : 0;
        const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(base), 0, bytes, 0x00020000);
        const bool ends = !TR && cols < STEP;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint32_t at = ends && (tid + i * NT) % CPR * 4 >= cols ? 0x7ffffff0u : goff[i];
            to.r[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, at, 0, 0));
        }
    }
    static __device__ __forceinline__ void store(const Regs& from, float* lds, int tid) {
#pragma unroll
        for (int i = 0; i < N; ++i) *reinterpret_cast<u32x4*>(lds + (tid + i * NT) / CPR * LD + (tid + i * NT) % CPR * 4) = from.r[i];
    }
    // A plain operand's last group of four can end in the next row: zeros in the place of columns k ... of that group
    static __device__ __forceinline__ void clear(float* lds, int k, int tid) {
        if constexpr (!TR)
            for (int i = tid; i < ROWS * 4; i += NT)
                if ((k & ~3) + i % 4 >= k) lds[i / 4 * LD + (k & ~3) + i % 4] = 0.0f;
    }
    // the eight values k = k0 + 8 g ... of row `row`
    static __device__ __forceinline__ Elem<float>::frag frag(const float* lds, int row, int k0, int g) {
        if constexpr (TR) {
            Elem<float>::frag f;
#pragma unroll
            for (int e = 0; e < 8; ++e) f.v[e] = lds[(k0 + 8 * g + e) * LD + row];
            return f;
        } else {
            return Elem<float>::load(lds + row * LD + k0 + 8 * g);
        }
    }
};

template <int BM, int BN, int STEP, bool ATR, bool BTR> constexpr int gemm_f32_lds = 2 * ((ATR ? STEP * (BM + 4) : BM * (STEP + 4)) + (BTR ? STEP * (BN + 4) : BN * (STEP + 4)));
// AHEAD: steps that are loaded ahead in registers.  64 x 64 tiles take two: a pair's 1500 x 1024 x 2048 107 us against 128,
// 2048 x 1024 x 1024 37.2 against 38.5.  32 x 32 tiles, whose work-groups are short, lose by it (333 x 1000 x 777 17.8 us
// against 16.7), and 128 x 128 tiles have no registers left for it.
template <int BM, int BN, int WM, int WN, int WK, int STEP, int AHEAD, bool ATR, bool BTR, bool PAIR, int EPI>
__device__ __forceinline__ void gemm_f32(const GemmArgs& a, int tms, int tns, unsigned id, unsigned total, float* lds) {
    constexpr int NW = WM * WN, NT = NW * WK * 64, TM = BM / WM, TN = BN / WN, MB = TM / 32, NB = TN / 32, BNO = PAIR ? BN / 2 : BN;
    static_assert(AHEAD == 1 || AHEAD == 2, "the loop's steps");
    static_assert(!PAIR || !BTR, "pairs are plain operands");
    typedef OperandTileF32<BM, ATR, STEP, NT> TileA;
    typedef OperandTileF32<BNO, BTR, STEP, NT> TileB;
    constexpr int STAGE = TileA::FLOATS + (PAIR ? 2 : 1) * TileB::FLOATS, KS = STEP / 16 / WK;      // 16 contraction steps per fragment
    static_assert((WK - 1) * NW * MB * NB * 1024 <= 2 * STAGE, "the wavefronts' results fit the stages");
    static_assert(2 * STAGE == gemm_f32_lds<BM, BN, STEP, ATR, BTR>, "two stages");
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wk = wave / NW, wm = wave % NW / WN, wn = wave % WN, l32 = lane & 31, g = lane >> 5;
    const GemmWork w = gemm_work(xcd_range(id, total), tms, tns, a.split);
    const long row0 = (long)w.tm * BM;
    const int col0 = w.tn * BNO;
    const int ksteps = (a.K + STEP - 1) / STEP, all = ksteps * a.segs;
    const int per = (all + a.split - 1) / a.split, k_begin = w.part * per, k_end = min(all, k_begin + per);

    TileA ta;
    TileB tb;
    ta.init(a.lda, tid);
    tb.init(a.ldb, tid);
    struct { typename TileA::Regs a; typename TileB::Regs b, b2; } regs[AHEAD];
    auto load = [&](int kt, auto& to) {
        // (behind the last step zeros, which cost no traffic: with loads in every step it is known how many are in flight)
        const int seg = kt < k_end && kt >= ksteps ? 1 : 0, k0 = (kt < k_end ? kt - seg * ksteps : ksteps) * STEP;
        ta.load(to.a, seg ? a.A[1] : a.A[w.b], a.lda, row0, a.M, k0, a.K, tid);
        tb.load(to.b, a.B[seg], a.ldb, col0, a.N, k0, a.K, tid);
        if constexpr (PAIR) tb.load(to.b2, a.B[1], a.ldb, col0, a.N, k0, a.K, tid);
    };
    auto store = [&](int stage, const auto& from) {
        float* p = lds + stage * STAGE;
        TileA::store(from.a, p, tid);
        TileB::store(from.b, p + TileA::FLOATS, tid);
        if constexpr (PAIR) TileB::store(from.b2, p + TileA::FLOATS + TileB::FLOATS, tid);
    };
    f32x16 acc[MB][NB];
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.0f;
#pragma unroll
    for (int p = 0; p < AHEAD; ++p) load(k_begin + p, regs[p]);
    store(0, regs[0]);
    load(k_begin + AHEAD, regs[0]);
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    int stage = 0;
    // the next step whose plain operands end inside a group
    int ends = (ATR && BTR) || a.K % 4 == 0 ? -1 : (k_begin / ksteps + 1) * ksteps - 1;
    // step k, whose successor lies in regs[next]
    auto step = [&](int k, auto& next) {
        float* A = lds + stage * STAGE;
        float* B = A + TileA::FLOATS;
        if (k == ends) {
            TileA::clear(A, a.K % STEP, tid);
            TileB::clear(B, a.K % STEP, tid);
            if constexpr (PAIR) TileB::clear(B + TileB::FLOATS, a.K % STEP, tid);
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
            ends += ksteps;
        }
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            const int kk = (wk * KS + ks) * 16;
            Elem<float>::frag af[MB], bf[NB];
#pragma unroll
            for (int i = 0; i < MB; ++i) af[i] = TileA::frag(A, wm * TM + i * 32 + l32, kk, g);
#pragma unroll
            for (int j = 0; j < NB; ++j)
                bf[j] = PAIR ? TileB::frag(B + (j & 1) * TileB::FLOATS, wn * (TN / 2) + (j >> 1) * 32 + l32, kk, g)
                             : TileB::frag(B, wn * TN + j * 32 + l32, kk, g);
            // (blocks in turn within a product index, so that no instruction waits for the one before it)
#pragma unroll
            for (int e = 0; e < 8; ++e)
#pragma unroll
                for (int i = 0; i < MB; ++i)
#pragma unroll
                    for (int j = 0; j < NB; ++j)
                        acc[i][j] = EPI == EPI_PART ? __builtin_amdgcn_mfma_f32_32x32x2f32(af[i].v[e], bf[j].v[e], acc[i][j], 0, 0, 0)
                                                    : __builtin_amdgcn_mfma_f32_32x32x2f32(bf[j].v[e], af[i].v[e], acc[i][j], 0, 0, 0);
        }
        stage ^= 1;
        store(stage, next);
        load(k + 1 + AHEAD, next);
        // (without the fence of __syncthreads, which would wait for the loads)
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    };
    // (one way back to the loop's start, or the compiler would count the loads in flight there as none)
    for (int k = k_begin;;) {
        if (k++ >= k_end) break;
        step(k - 1, regs[AHEAD - 1]);
        if constexpr (AHEAD > 1) {
            if (k++ >= k_end) break;
            step(k - 1, regs[0]);
        }
    }
    if constexpr (WK > 1) {
        f32x4* area = reinterpret_cast<f32x4*>(lds);
        join_put<MB, NB>(area, acc, wk > 0 ? (wk - 1) * NW + wave % NW : -1, lane);
        __syncthreads();
        if (wk > 0) return;
#pragma unroll
        for (int p = 0; p < WK - 1; ++p) join_add<MB, NB>(area, acc, p * NW + wave, lane);
    }
    wave_epilogue<float, EPI, PAIR, MB, NB>(a, w, row0 + wm * TM, col0 + wn * (PAIR ? TN / 2 : TN), acc, lane);
}

template <int BM, int BN, int WM, int WN, int WK, int STEP, int AHEAD, bool ATR, bool BTR, bool PAIR, int EPI>
__global__ void __launch_bounds__(WM* WN* WK * 64, 2) gemm_f32_kernel(GemmArgs a, int tms, int tns) {
    __shared__ __align__(16) float lds[gemm_f32_lds<BM, BN, STEP, ATR, BTR>];
    gemm_f32<BM, BN, WM, WN, WK, STEP, AHEAD, ATR, BTR, PAIR, EPI>(a, tms, tns, blockIdx.x, gridDim.x, lds);
}
template <int BM, int BN, int WM, int WN, int WK, int STEP, int AHEAD>
__global__ void __launch_bounds__(WM* WN* WK * 64, 2) gemm_f32_both_kernel(GemmArgs x, GemmArgs w, BothGrid n) {
    constexpr int LX = gemm_f32_lds<BM, BN, STEP, false, true>, LW = gemm_f32_lds<BM, BN, STEP, true, true>;
    __shared__ __align__(16) float lds[LX > LW ? LX : LW];
    const unsigned i = blockIdx.x;
    if (i >= n.x0 && i < n.x0 + n.nx) gemm_f32<BM, BN, WM, WN, WK, STEP, AHEAD, false, true, false, EPI_STORE>(x, n.xms, n.xns, i - n.x0, n.nx, lds);
    else gemm_f32<BM, BN, WM, WN, WK, STEP, AHEAD, true, true, false, EPI_STORE>(w, n.wms, n.wns, i < n.x0 ? i : i - n.nx, gridDim.x - n.nx, lds);
}

}  // namespace tfla
