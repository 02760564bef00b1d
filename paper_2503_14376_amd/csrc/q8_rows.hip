// Products of few rows of codes with a whole matrix of weights in 8 bits (tokens being generated), as gemm_rows.hip does them for
// bf16: one read of the weights bounds them, straight into the operand registers of v_mfma_scale_f32_16x16x128_f8f6f4, whose step is
// the 128 codes that share a scale.  Rows may start at any address.
// Measured: 1 token through 4096 x 4096 with bias and residual 8.2 us with the host's time (kernel 7.5; 16.8 MB, of which a first load takes 2 us
// to arrive), 4 through a pair of 10944 x 4096 18.9 (4.7 TB/s), its gate 4.0.  Scratch: pairs at odd addresses with sixteen wavefronts and two
// pieces in flight (17 to 32 rows 37 registers, 5 to 8 rows 4).
#include "gemm_epilogue.h"
#include "q8.h"
#include "q8_internal.h"

namespace tfla {

namespace {

// 32 codes of a row: 16 at k, 16 at k + 64 (so that an access reads 64 consecutive bytes of each row); left: codes from k on that exist
template <bool ODD> struct Codes32 {
    i32x8 w;
    __device__ __forceinline__ void load(const uint8_t* p) {
        __builtin_memcpy(&w, p, 16);
        __builtin_memcpy(reinterpret_cast<char*>(&w) + 16, p + 64, 16);
    }
    // (k: the row's length, a multiple of four.  Without branches, which would have one load wait for another, a row's end is read from inside
    // the row and moved, what does not exist at its beginning: 8 tokens through 10944 x 4104 15.2 us, so 12.7.  Of four slices only one ends with
    // the row, and its lanes' reads cost more than the branch: pair, 4 x 10944 x 10944 50 us, without branches 55)
    template <bool BRANCHES> __device__ __forceinline__ void load_tail(const uint8_t* p, int left, const uint8_t* row, int k) {
        if (!BRANCHES && k >= 16) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int n = left - h * 64, behind = n >= 16 || n <= 0 ? 0 : 16 - n;
                u32x4 v;
                __builtin_memcpy(&v, n > 0 ? p + h * 64 - behind : row, 16);
                const bool eight = (behind & 8) != 0, four = (behind & 4) != 0;
                v = u32x4{eight ? v[2] : v[0], eight ? v[3] : v[1], eight ? 0 : v[2], eight ? 0 : v[3]};
                v = u32x4{four ? v[1] : v[0], four ? v[2] : v[1], four ? v[3] : v[2], four ? 0 : v[3]};
#pragma unroll
                for (int e = 0; e < 4; ++e) w[h * 4 + e] = n > 0 ? (int)v[e] : 0;
            }
            return;
        }
        uint32_t t[8];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if (left - h * 64 >= 16) __builtin_memcpy(t + h * 4, p + h * 64, 16);
            else {
#pragma unroll
                for (int e = 0; e < 4; ++e) t[h * 4 + e] = 0;
#pragma unroll
                for (int e = 0; e < 15; ++e)
                    if (h * 64 + e < left) t[h * 4 + (e >> 2)] |= (uint32_t)p[h * 64 + e] << (8 * (e & 3));
            }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = (int)t[e];
    }
    __device__ __forceinline__ i32x8 codes(int) const { return w; }
};
// ... of a row at any address (ODD).  What is read are whole words of four bytes, one more than there are codes for, and moved by the row's place in its
// first word when the codes are wanted (16 bytes at an odd address are many accesses: 16 x 4095 through 4096 rows 18.7 us, so 10.6).  Such a
// word may hold up to three bytes before or behind the row, which count for nothing; one without a byte of the row is not read.
template <> struct Codes32<true> {
    uint32_t d[2][5];
    __device__ __forceinline__ void load(const uint8_t* p) {
        const uintptr_t at = reinterpret_cast<uintptr_t>(p);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            __builtin_memcpy(d[h], __builtin_assume_aligned(reinterpret_cast<const void*>((at & ~(uintptr_t)3) + h * 64), 4), 16);
            d[h][4] = *reinterpret_cast<const uint32_t*>(((at + 15) & ~(uintptr_t)3) + h * 64);
        }
    }
    // (words behind the end are read at `row`, so that no branch holds the others up, and cleared)
    template <bool BRANCHES> __device__ __forceinline__ void load_tail(const uint8_t* p, int left, const uint8_t* row, int) {
        const int shift = (int)(reinterpret_cast<uintptr_t>(p) & 3);
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < 5; ++j) {
                const int n = left > h * 64 ? min(left - h * 64, 16) + shift - 4 * j : 0;       // bytes of the word that are the row's or before it
                const uintptr_t from = reinterpret_cast<uintptr_t>(n > 0 ? p - shift + h * 64 + 4 * j : row) & ~(uintptr_t)3;
                const uint32_t v = *reinterpret_cast<const uint32_t*>(from);
                d[h][j] = n <= 0 ? 0u : (n >= 4 ? v : v & ((1u << 8 * n) - 1));
            }
    }
    __device__ __forceinline__ i32x8 codes(int shift) const {
        i32x8 w;
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = (int)__builtin_amdgcn_alignbyte(d[e / 4][e % 4 + 1], d[e / 4][e % 4], (uint32_t)shift);
        return w;
    }
};

// MB blocks of 16 rows of x, NW wavefronts, U pieces of 128 codes in flight per wavefront, SL slices, HOLD: as gemm_rows_kernel.
// A pair's products go to the partial planes, for its gate and the codes of 128 columns at a time are formed in a second launch.
template <int MB, int SL, bool PAIR, int NW, int U, bool HOLD, bool ODD>
__global__ void __launch_bounds__(NW * 64) q8_rows_kernel(Q8GemmArgs q, int blocks) {
    constexpr int P = PAIR ? 2 : 1, RB = 16 / SL, LD = RB + 4;
    static_assert(SL == 1 || MB == 1, "slices take one block of rows");
    const GemmArgs& a = q.g;
    __shared__ __align__(16) float red[NW * SL][P][MB * RB][LD];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, g = lane >> 4, slice = r / RB;
    const int full = q.k >> 7, pieces = (q.k + 127) >> 7, ps = (pieces + SL - 1) / SL;      // ps: pieces of a slice
    const uint8_t* xp = reinterpret_cast<const uint8_t*>(a.A[0]) + g * 16;
    long xrow[MB];
    int xm[MB];
#pragma unroll
    for (int i = 0; i < MB; ++i) {
        xm[i] = min(i * 16 + r % RB, a.M - 1);
        xrow[i] = (long)xm[i] * q.k;
    }
    Codes32<ODD> w[U][P], x[U][MB];
    int ws[U][P], xs[U][MB];
    // a row's place in its first word
    int wshift[P] = {}, xshift[MB] = {};
    if constexpr (ODD) {
#pragma unroll
        for (int i = 0; i < MB; ++i) xshift[i] = (int)(reinterpret_cast<uintptr_t>(xp + xrow[i]) & 3);
    }
    // piece c0 + u NW of this lane's slice
    auto fetch = [&](int c0, int n0, bool with_w, bool with_x) {
        // rows behind the last one read it again: their results are not stored
        const long wrow = (long)min(n0 + r % RB, a.N - 1) * q.k;
        if constexpr (ODD) {
#pragma unroll
            for (int p = 0; p < P; ++p) wshift[p] = (int)((reinterpret_cast<uintptr_t>(a.B[p]) + wrow) & 3);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c = c0 + u * NW, kb = slice * ps + c;
            if ((SL - 1) * ps + c < full && c < ps) {
#pragma unroll
                for (int p = 0; p < P; ++p)
                    if (with_w) w[u][p].load(reinterpret_cast<const uint8_t*>(a.B[p]) + wrow + g * 16 + (long)kb * 128);
#pragma unroll
                for (int i = 0; i < MB; ++i)
                    if (with_x) x[u][i].load(xp + xrow[i] + (long)kb * 128);
            } else {
                const int left = c < ps ? q.k - kb * 128 - g * 16 : 0;
#pragma unroll
                for (int p = 0; p < P; ++p)
                    if (with_w)
                        w[u][p].template load_tail<HOLD || SL == 4>(reinterpret_cast<const uint8_t*>(a.B[p]) + wrow + g * 16 + (long)kb * 128, left,
                                                         reinterpret_cast<const uint8_t*>(a.B[p]) + wrow, q.k);
#pragma unroll
                for (int i = 0; i < MB; ++i)
                    if (with_x) x[u][i].template load_tail<HOLD || SL == 4>(xp + xrow[i] + (long)kb * 128, left, xp - g * 16 + xrow[i], q.k);
            }
            const int ks = min(kb, pieces - 1);
#pragma unroll
            for (int p = 0; p < P; ++p)
                if (with_w) ws[u][p] = q.sb[p][(long)ks * q.lsb + (n0 >> 7)];
#pragma unroll
            for (int i = 0; i < MB; ++i)
                if (with_x) xs[u][i] = q.sa[0][(long)ks * q.lsa + xm[i]];
        }
    };
    int block = blockIdx.x;
    if (HOLD) {
        fetch(wave, block * RB, true, false);
        fetch(wave, block * RB, false, true);
    }
    for (; block < blocks; block += gridDim.x) {
        const int n0 = block * RB;
        f32x4 acc[P][MB];
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int i = 0; i < MB; ++i) acc[p][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        for (int c0 = wave; c0 < ps || HOLD; c0 += NW * U) {
            if (!HOLD) fetch(c0, n0, true, true);
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int p = 0; p < P; ++p)
#pragma unroll
                    for (int i = 0; i < MB; ++i)
                        acc[p][i] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w[u][p].codes(wshift[p]), x[u][i].codes(xshift[i]), acc[p][i], 0, 0, 0,
                                                                                                  ws[u][p], 0, xs[u][i]);
            if (HOLD) break;
        }
        if (HOLD && block + (int)gridDim.x < blocks) fetch(wave, n0 + gridDim.x * RB, true, false);
        // lane (r, g) holds column r (a slice and a row of x) of the rows 4 g ... 4 g + 3 (a slice, four rows of w)
        if (4 * g / RB == slice) {
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int i = 0; i < MB; ++i) *reinterpret_cast<f32x4*>(&red[wave * SL + slice][p][i * RB + r % RB][4 * g % RB]) = acc[p][i];
        }
        // (barriers without the fence of __syncthreads, which would wait for the next block's weights)
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        for (int i = threadIdx.x; i < P * MB * RB * RB; i += NW * 64) {
            const int n = i % RB, m = i / RB % (MB * RB), p = i / (MB * RB * RB);
            float s = red[0][p][m][n];
#pragma unroll
            for (int k = 1; k < NW * SL; ++k) s += red[k][p][m][n];
            if constexpr (PAIR) {
                if (m < a.M && n0 + n < a.N) partial_plane(a, 2, 0, p)[(long)m * a.ld_part + n0 + n] = s;
            } else {
                red[0][p][m][n] = s;
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if constexpr (!PAIR) {
            constexpr int W = RB < 8 ? RB : 8, GR = RB / W;
            const int m = threadIdx.x / GR, c = threadIdx.x % GR * W;
            if (m < MB * RB) {
                float v[8], u[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    v[e] = e < W ? red[0][0][m][c + e] : 0.0f;
                    u[e] = 0.0f;
                }
                epilogue8<bf16_t, EPI_LINEAR>(a, 0, m, n0 + c, v, u, W);
            }
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        }
    }
}

// (rows at odd addresses are not held over blocks: their words are more, and so are the registers)
template <int MB, int SL, bool PAIR, int NW> void launch(const Q8GemmArgs& a, const Q8RowsPlan& p, bool odd, hipStream_t s) {
    const dim3 threads(NW * 64);
    if constexpr (NW <= 8) {
        if constexpr (SL == 4 && !PAIR) {
            if (p.ahead == 3 && !odd) {
                hipLaunchKernelGGL((q8_rows_kernel<MB, SL, PAIR, NW, 3, true, false>), dim3(p.grid), threads, 0, s, a, p.blocks);
                return;
            }
        }
    }
    if (odd) {
        if (p.ahead == 2) hipLaunchKernelGGL((q8_rows_kernel<MB, SL, PAIR, NW, 2, false, true>), dim3(p.blocks), threads, 0, s, a, p.blocks);
        else hipLaunchKernelGGL((q8_rows_kernel<MB, SL, PAIR, NW, 1, false, true>), dim3(p.blocks), threads, 0, s, a, p.blocks);
        return;
    }
    if constexpr (NW <= 8) {
        if (p.hold) {
            hipLaunchKernelGGL((q8_rows_kernel<MB, SL, PAIR, NW, 2, true, false>), dim3(p.grid), threads, 0, s, a, p.blocks);
            return;
        }
    }
    if (p.ahead == 2) hipLaunchKernelGGL((q8_rows_kernel<MB, SL, PAIR, NW, 2, false, false>), dim3(p.grid), threads, 0, s, a, p.blocks);
    else hipLaunchKernelGGL((q8_rows_kernel<MB, SL, PAIR, NW, 1, false, false>), dim3(p.grid), threads, 0, s, a, p.blocks);
}
template <int MB, int SL, bool PAIR> void go(const Q8GemmArgs& a, const Q8RowsPlan& p, bool odd, hipStream_t s) {
    if (p.waves == 4) launch<MB, SL, PAIR, 4>(a, p, odd, s);
    else if (p.waves == 8) launch<MB, SL, PAIR, 8>(a, p, odd, s);
    else launch<MB, SL, PAIR, 16>(a, p, odd, s);
}
template <bool PAIR> void by_rows(const Q8GemmArgs& a, hipStream_t s) {
    const Q8RowsPlan p = q8_rows_plan(a.g.M, a.g.N, a.k, PAIR);
    const uintptr_t all = reinterpret_cast<uintptr_t>(a.g.A[0]) | reinterpret_cast<uintptr_t>(a.g.B[0]) | (PAIR ? reinterpret_cast<uintptr_t>(a.g.B[1]) : 0);
    const bool odd = ((all | (uintptr_t)a.k) & 3) != 0;
    if (p.slices == 4) go<1, 4, PAIR>(a, p, odd, s);
    else if (p.slices == 2) go<1, 2, PAIR>(a, p, odd, s);
    else if (p.row_blocks == 1) go<1, 1, PAIR>(a, p, odd, s);
    else go<2, 1, PAIR>(a, p, odd, s);
}

}  // namespace

hipError_t launch_q8_rows(const Q8GemmArgs& a, hipStream_t s) {
    if (a.g.pair) by_rows<true>(a, s);
    else by_rows<false>(a, s);
    return hipGetLastError();
}

}  // namespace tfla
