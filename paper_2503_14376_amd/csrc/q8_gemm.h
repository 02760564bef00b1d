// Products of two matrices of e4m3 codes with power-of-two scales for every 128 of the contraction, for gfx950:
// v_mfma_scale_f32_32x32x64_f8f6f4, fp32 accumulation.  128 codes of a row are as many bytes as 64 elements of bf16, so that tiles
// come and lie in LDS as the bf16 products' do (gemm.h), and a step is worth twice the contraction.  The scales go the same way:
// one byte per row and step, widened to a word of LDS by the load, which the matrix unit takes as it is.
//
// Within an instruction the matrix unit adds the products of eight consecutive codes with the bits that lie no more than 13 below
// the largest one's, and everything else in fp32: 1.3e-5 of a random sum's size, a 130th of what its rounding to bf16 costs.
#pragma once
#include "gemm.h"
#include "q8.h"
#include "q8_internal.h"

namespace tfla {

template <int EPI> __device__ __forceinline__ f32x16 mma_q8(const i32x8& a, const i32x8& b, const f32x16& c, int sa, int sb) {
    return EPI == EPI_PART ? __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 0, 0, 0, sa, 0, sb)
                           : __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(b, a, c, 0, 0, 0, sb, 0, sa);
}
// Two pieces of 16 codes.  (Which codes of a step a lane's registers hold does not matter: it is the same for both operands, and
// they share the step's scale.)
__device__ __forceinline__ i32x8 q8_frag(const bf16x8& lo, const bf16x8& hi) {
    const u32x4 a = __builtin_bit_cast(u32x4, lo), b = __builtin_bit_cast(u32x4, hi);
    return i32x8{(int)a[0], (int)a[1], (int)a[2], (int)a[3], (int)b[0], (int)b[1], (int)b[2], (int)b[3]};
}

// The stream of a tile's scales into LDS, a word for each of the AR rows of A and, behind them, the BR rows of B (PAIR: BR / 2 of
// either matrix).  A request brings those of 64 rows; a wavefront issues N of them per step, some of which bring nothing.
template <int AR, int BR, int NW, bool PAIR> struct ScaleStream {
    static constexpr int REQUESTS = (AR + BR) / 64, N = (REQUESTS + NW - 1) / NW, BYTES = N * NW * 256;
    u32x4 d[N];
    uint32_t off[N], hop[N];
    // second: of the second segment; block: of the contraction
    __device__ __forceinline__ void set(const Q8GemmArgs& a, const GemmWork& w, long row0, int col0, int block, bool second, bool exists, int tid) {
        const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int q = wave + j * NW;
            const bool ofa = q < AR / 64;
            const int r = (ofa ? q : q - AR / 64) * 64, m = PAIR && !ofa ? r / (BR / 2) : 0;
            const int sh = ofa ? 0 : a.shb;
            const long first = ofa ? row0 + r : (long)col0 + r - m * (BR / 2), extent = ofa ? a.g.M : a.g.N, ld = ofa ? a.lsa : a.lsb;
            // (members by constant indices: with others the compiler keeps the arguments in memory, where a descriptor cannot be)
            const uint8_t* p = ofa ? (second || w.b ? a.sa[1] : a.sa[0]) : ((PAIR ? m != 0 : second) ? a.sb[1] : a.sb[0]);
            const uint64_t b = reinterpret_cast<uint64_t>(p) + (uint64_t)(block * ld + (first >> sh));
            d[j][0] = (uint32_t)b;
            d[j][1] = (uint32_t)(b >> 32) & 0xffffu;
            d[j][2] = exists && q < REQUESTS && first < extent ? (uint32_t)min(64l, ((extent - 1) >> sh) - (first >> sh) + 1) : 0u;
            d[j][3] = 0x00020000u;
            off[j] = (uint32_t)(((first + lane) >> sh) - (first >> sh));
            hop[j] = (uint32_t)ld;
        }
    }
    template <int STEPS> __device__ __forceinline__ void advance() {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const uint64_t b = ((uint64_t)d[j][1] << 32 | d[j][0]) + (uint64_t)hop[j] * STEPS;
            d[j][0] = (uint32_t)b;
            d[j][1] = (uint32_t)(b >> 32);
        }
    }
    // lds: LDS address of the scales plus 256 times the wavefront
    __device__ __forceinline__ void issue(int j, uint32_t lds) const {
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_ubyte %1, %2, 0 offen lds"
                     :: "s"(lds + j * NW * 256), "v"(off[j]), "s"(d[j]) : "m0");
    }
    __device__ __forceinline__ void issue_all(uint32_t lds) const {
#pragma unroll
        for (int j = 0; j < N; ++j) issue(j, lds);
    }
};

// Which step the streams stand at, as StepStream, with the scales' beside them.
template <bool PAIR, int STRIDE> struct Q8StepStream {
    StepStream<PAIR, STRIDE> st;
    template <typename OA, typename OB, typename SC>
    __device__ __forceinline__ void find(const Q8GemmArgs& a, const GemmWork& w, long row0, int col0, OA& oa, OB& ob, SC& sc, int tid) {
        const bool on = st.at < st.k_end, second = st.at >= st.ksteps;
        const int block = on ? (second ? st.at - st.ksteps : st.at) : 0;
        const void* pa = second || w.b ? a.g.A[1] : a.g.A[0];
        const void* pb = second && !PAIR ? a.g.B[1] : a.g.B[0];
        oa.set(pa, pa, a.g.lda, row0, a.g.M, a.g.K, block * 64, on, tid);
        ob.set(pb, PAIR ? a.g.B[1] : pb, a.g.ldb, col0, a.g.N, a.g.K, block * 64, on, tid);
        sc.set(a, w, row0, col0, block, second, on, tid);
        const int seg_end = second ? 2 * st.ksteps : st.ksteps, whole = seg_end - (a.g.K % 64 != 0);
        st.change = !on ? 0x7fffffff : min(st.k_end, st.at < whole ? whole : seg_end);
    }
    template <typename OA, typename OB, typename SC>
    __device__ __forceinline__ void next(const Q8GemmArgs& a, const GemmWork& w, long row0, int col0, OA& oa, OB& ob, SC& sc, int tid) {
        st.at += STRIDE;
        oa.template advance<STRIDE>();
        ob.template advance<STRIDE>();
        sc.template advance<STRIDE>();
        if (st.at >= st.change) find(a, w, row0, col0, oa, ob, sc, tid);
    }
};

// Tile BM x BN, WM x WN wavefronts, S LDS stages, KG groups of wavefronts: as gemm_bf16.  2000 x 4096 x 4096 by 512 tiles of 128 x 128, two a CU: 37 us
// (1.8 PFLOP/s; matrix unit 49 % busy, behind LDS and the two rounds' ends).
template <int BM, int BN, int WM, int WN, int S, int KG, bool PAIR> constexpr int gemm_q8_lds = KG * S * ((BM + BN) * 128 + ScaleStream<BM, BN, WM * WN, PAIR>::BYTES);
template <int BM, int BN, int WM, int WN, int S, int KG, bool PAIR, int EPI>
__device__ __forceinline__ void gemm_q8(const Q8GemmArgs& a, int tms, int tns, unsigned id, unsigned total, char* lds) {
    constexpr int NT = WM * WN * 64, TM = BM / WM, TN = BN / WN, MB = TM / 32, NB = TN / 32, BNO = PAIR ? BN / 2 : BN;
    typedef ScaleStream<BM, BN, WM * WN, PAIR> Scales;
    constexpr int ABYTES = BM * 128, BBYTES = BN * 128, TILES = ABYTES + BBYTES, STAGE = TILES + Scales::BYTES;
    constexpr int JOIN = (KG - 1) * WM * WN * MB * NB * 4096;
    static_assert(JOIN <= KG * S * STAGE, "the groups' results fit the stages");
    static_assert(KG * S * STAGE == gemm_q8_lds<BM, BN, WM, WN, S, KG, PAIR>, "the stages");
    const int tid = threadIdx.x % NT, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int group = KG == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / NT);
    const int wm = wave / WN, wn = wave % WN, l32 = lane & 31;
    const GemmWork w = gemm_work(xcd_range(id, total), tms, tns, a.g.split);
    const long row0 = (long)w.tm * BM;
    const int col0 = w.tn * BNO;

    OperandStream<BM, false, BM, NT, 1, false> oa;
    OperandStream<BNO, false, BNO, NT, PAIR ? 2 : 1, PAIR> ob;
    Scales sc;
    constexpr int LOADS = oa.N + (PAIR ? 2 : 1) * ob.N + Scales::N;     // requests of a wavefront per step
    Q8StepStream<PAIR, KG> qs;
    auto& st = qs.st;
    oa.init(a.g.lda, tid);
    ob.init(a.g.ldb, tid);
    st.ksteps = (a.g.K + 63) / 64;
    const int all = st.ksteps * a.g.segs, per = (all + a.g.split - 1) / a.g.split;
    const int k_begin = w.part * per;
    st.at = k_begin + group;
    st.k_end = min(all, k_begin + per);
    qs.find(a, w, row0, col0, oa, ob, sc, tid);
    char* ring = lds + group * S * STAGE;
    const uint32_t la = lds_addr(ring) + wave * 1024, lb = la + ABYTES, ls = lds_addr(ring) + TILES + wave * 256;
    auto request = [&](uint32_t off) {
        oa.template issue_all<0>(la + off);
        ob.template issue_all<0>(lb + off);
        if constexpr (PAIR) ob.template issue_all<1>(lb + BBYTES / 2 + off);
        sc.issue_all(ls + off);
        qs.next(a, w, row0, col0, oa, ob, sc, tid);
    };
    f32x16 acc[MB][NB];
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.0f;
    KFragReader<64> kf;
    kf.init(l32, lane >> 5);
    // row of B's tile where block j of this wavefront begins
    auto brow = [&](int j) { return PAIR ? (j & 1) * (BN / 2) + wn * (TN / 2) + (j >> 1) * 32 : wn * TN + j * 32; };

#pragma unroll
    for (int q = 0; q < S - 1; ++q) request(q * STAGE);
    uint32_t off = 0, next = (S - 1) * STAGE;
    for (int k = k_begin; k < st.k_end; k += KG) {
        wait_vmcnt<(S - 2) * LOADS>();
        // (the reads of the stage that is requested next have to be over, not only begun, when the wavefronts meet)
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        const char* A = ring + off;
        const char* B = A + ABYTES;
        const int* sw = reinterpret_cast<const int*>(A + TILES);
        i32x8 af[2][MB], bf[2][NB];
        int sa[MB], sb[NB];
#pragma unroll
        for (int i = 0; i < MB; ++i) sa[i] = sw[wm * TM + i * 32 + l32];
#pragma unroll
        for (int j = 0; j < NB; ++j) sb[j] = sw[BM + brow(j) + l32];
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
#pragma unroll
            for (int i = 0; i < MB; ++i) {
                const char* p = A + (wm * TM + i * 32) * 128;
                af[ks][i] = q8_frag(kf.load(p, 2 * ks, 0), kf.load(p, 2 * ks + 1, 0));
            }
#pragma unroll
            for (int j = 0; j < NB; ++j) {
                const char* p = B + brow(j) * 128;
                bf[ks][j] = q8_frag(kf.load(p, 2 * ks, 0), kf.load(p, 2 * ks + 1, 0));
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        request(next);
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int j = 0; j < NB; ++j) acc[i][j] = mma_q8<EPI>(af[ks][i], bf[ks][j], acc[i][j], sa[i], sb[j]);
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
    wave_epilogue<bf16_t, EPI, PAIR, MB, NB>(a.g, w, row0 + wm * TM, col0 + wn * (PAIR ? TN / 2 : TN), acc, lane);
}

template <int BM, int BN, int WM, int WN, int S, int KG, bool PAIR, int EPI>
__global__ void __launch_bounds__(KG* WM* WN * 64, 2) gemm_q8_kernel(Q8GemmArgs a, int tms, int tns) {
    __shared__ __align__(1024) char lds[gemm_q8_lds<BM, BN, WM, WN, S, KG, PAIR>];
    gemm_q8<BM, BN, WM, WN, S, KG, PAIR, EPI>(a, tms, tns, blockIdx.x, gridDim.x, lds);
}

// Both products of a small backward pass in one launch, those with the longer contraction first, and behind them the column sums of the
// bias gradients.  n: workgroups of the first product, of both, and all.
template <int KG, int S>
__global__ void __launch_bounds__(KG * 256, 2) gemm_q8_both_kernel(Q8GemmArgs x, Q8GemmArgs w, Q8Both n, Q8Sums sums) {
    __shared__ __align__(1024) char lds[gemm_q8_lds<64, 64, 2, 2, S, KG, false>];
    const unsigned i = blockIdx.x;
    if (i < n.first) gemm_q8<64, 64, 2, 2, S, KG, false, EPI_STORE>(x, n.tms[0], n.tns[0], i, n.first, lds);
    else if (i < n.both) gemm_q8<64, 64, 2, 2, S, KG, false, EPI_STORE>(w, n.tms[1], n.tns[1], i - n.first, n.both - n.first, lds);
    else {
        const int c = (i - n.both) * (KG * 256) + threadIdx.x, p = c / sums.n, col = c % sums.n;
        float* out = p == 0 ? sums.out[0] : sums.out[1];
        if (p >= sums.planes || !out) return;
        const float* from = sums.part + c;
        float s = 0.0f;
#pragma unroll 8
        for (int r = 0; r < sums.rows; ++r) s += from[(long)r * sums.planes * sums.n];
        out[col] = s;
    }
}

}  // namespace tfla
