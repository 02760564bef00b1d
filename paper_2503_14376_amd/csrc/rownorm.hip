// The norm over a model's columns (RMS norm or LayerNorm of rows of D values), forward and backward, with the sums of the
// weights' gradients.  Memory-bound row work: a row is read once into the registers of one wavefront (D up to 1024) or one
// workgroup, its statistics are formed there in fp32, and it is written once.  Rows of 4096 in bf16, 16384 of them: forward 51.5 us,
// backward with residual and both sums 103.5, 5.2 TB/s each, the rate of a copy.  Rows that do not begin at multiples of 16 bytes
// take twice the accesses: 2999 rows of 1365 in fp32, backward, 14.6 us for 49 MB (3.4 TB/s).
#include "block_internal.h"
#include "row8.h"

namespace tfla {

namespace {

constexpr int WIDEST = 16;      // wavefronts of the largest workgroup

// A row of D values over T threads: thread t holds the groups of eight t, t + T, ... (J at most).
template <typename DT, int T, int J> struct RowPart {
    Vec8<DT> v[J];
    __device__ __forceinline__ void load(const void* base, long row, int D, int t) {
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int c = (t + T * j) * 8;
            v[j] = load8<DT>(base, row * D + c, D - c);
        }
    }
};
template <int T, int J> __device__ __forceinline__ void load_vector(const float* p, float (&x)[J][8], int D, int t, float fill) {
#pragma unroll
    for (int j = 0; j < J; ++j) {
        const int c = (t + T * j) * 8;
        if (p) load8<float>(p, c, D - c).get(x[j]);
        else {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[j][e] = fill;
        }
    }
}

// Two sums over the T threads of a row, in every thread.  Rows of one wavefront stay in registers; otherwise the
// wavefronts meet in LDS, in `slot`, which alternates from row to row so that one barrier a row is enough.
template <int T> __device__ __forceinline__ void row_sum2(float& a, float& b, float (*slot)[2]) {
    a = lanes_sum<64>(a);
    b = lanes_sum<64>(b);
    if constexpr (T > 64) {
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0) { slot[wave][0] = a; slot[wave][1] = b; }
        __syncthreads();
        a = 0.0f; b = 0.0f;
#pragma unroll
        for (int w = 0; w < T / 64; ++w) { a += slot[w][0]; b += slot[w][1]; }
    }
}

// Mean and 1/sqrt(variance + eps) of a row.  LayerNorm: every wavefront takes the squares about its own mean, and the
// wavefronts' means and sums of squares are joined with the between-means term, so that nothing cancels and the
// wavefronts meet once.
template <int T, int J>
__device__ __forceinline__ void row_stats(const float (&x)[J][8], int D, int t, bool layer, float eps, float& mean, float& rstd,
                                          float (*slot)[2]) {
    const int wave = threadIdx.x >> 6;
    float s = 0.0f, q = 0.0f;
    if (!layer) {
#pragma unroll
        for (int j = 0; j < J; ++j)
#pragma unroll
            for (int e = 0; e < 8; ++e) s += x[j][e] * x[j][e];
        row_sum2<T>(s, q, slot);
        mean = 0.0f;
        rstd = 1.0f / sqrtf(s / (float)D + eps);
        return;
    }
    // values that this wavefront holds: its lanes' groups of eight are 64 * 8 columns wide for every j
    int cnt = 0;
#pragma unroll
    for (int j = 0; j < J; ++j) {
        const int left = D - ((t & ~63) + T * j) * 8;
        cnt += left <= 0 ? 0 : (left < 512 ? left : 512);
#pragma unroll
        for (int e = 0; e < 8; ++e) s += x[j][e];
    }
    s = lanes_sum<64>(s);
    const float mw = cnt > 0 ? s / (float)cnt : 0.0f;
#pragma unroll
    for (int j = 0; j < J; ++j) {
        const int left = D - (t + T * j) * 8;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float d = x[j][e] - mw;
            q += e < left ? d * d : 0.0f;
        }
    }
    q = lanes_sum<64>(q);
    if constexpr (T == 64) {
        mean = mw;
    } else {
        if ((threadIdx.x & 63) == 0) { slot[wave][0] = s; slot[wave][1] = q; }
        __syncthreads();
        float tot = 0.0f;
#pragma unroll
        for (int w = 0; w < T / 64; ++w) tot += slot[w][0];
        mean = tot / (float)D;
        q = 0.0f;
#pragma unroll
        for (int w = 0; w < T / 64; ++w) {
            int n = 0;
#pragma unroll
            for (int j = 0; j < J; ++j) {
                const int left = D - (w * 64 + T * j) * 8;
                n += left <= 0 ? 0 : (left < 512 ? left : 512);
            }
            const float d = n > 0 ? slot[w][0] / (float)n - mean : 0.0f;
            q += slot[w][1] + d * d * (float)n;
        }
    }
    rstd = 1.0f / sqrtf(q / (float)D + eps);
}

// NT threads per workgroup, T of them per row; the rows go round the grid.
template <typename DT, int T, int J>
__global__ void __launch_bounds__(T < 256 ? 256 : T) rownorm_fwd_kernel(RowNormArgs a) {
    constexpr int G = T < 256 ? 256 / T : 1;            // rows at a time
    __shared__ float slots[2][WIDEST][2];
    const int t = threadIdx.x % T, grp = threadIdx.x / T;
    const bool layer = a.kind == 1;
    float g[J][8], be[J][8];
    load_vector<T, J>(a.gamma, g, a.D, t, 1.0f);
    load_vector<T, J>(layer ? a.beta : nullptr, be, a.D, t, 0.0f);
    const long step = (long)gridDim.x * G;
    long row = (long)blockIdx.x * G + grp;
    if (T <= 64 && row >= a.M) return;
    // (the next row is loaded ahead where the registers allow it: sixteen wavefronts of two groups have 128 and hide it by number)
    constexpr bool AHEAD = T * J < 2048;
    RowPart<DT, T, J> next;
    if (AHEAD) next.load(a.x, row, a.D, t);
    for (int par = 0; row < a.M; row += step, par ^= 1) {
        float x[J][8];
        if (!AHEAD) next.load(a.x, row, a.D, t);
#pragma unroll
        for (int j = 0; j < J; ++j) next.v[j].get(x[j]);
        if (AHEAD && row + step < a.M) next.load(a.x, row + step, a.D, t);
        float mean, rstd;
        row_stats<T, J>(x, a.D, t, layer, a.eps, mean, rstd, slots[par]);
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int c = (t + T * j) * 8;
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = (x[j][e] - mean) * rstd * g[j][e] + be[j][e];
            store8<DT>(a.y, row * a.D + c, a.D - c, y);
        }
        if (t == 0) {
            if (a.rstd) a.rstd[row] = rstd;
            if (a.mean) a.mean[row] = mean;
        }
    }
}

// dx = rstd (g - xh mean(g xh) - [LayerNorm] mean(g)) + d_residual with xh = (x - mean) rstd, g = dy gamma.  Every row
// group keeps the sums of dy xh and dy over its rows in registers; the groups of a workgroup meet in LDS, and its sums go to
// part[workgroup], which sum_rows_kernel adds in that order, so that the result does not depend on the order of execution.
template <typename DT, int T, int J>
__global__ void __launch_bounds__(T < 256 ? 256 : T) rownorm_bwd_kernel(RowNormBwdArgs a) {
    constexpr int G = T < 256 ? 256 / T : 1;
    __shared__ float slots[2][WIDEST][2];
    const int t = threadIdx.x % T, grp = threadIdx.x / T;
    const bool layer = a.kind == 1;
    const long step = (long)a.blocks * G;
    long row = (long)blockIdx.x * G + grp;
    float g[J][8], ag[J][8], ab[J][8];
    load_vector<T, J>(a.gamma, g, a.D, t, 1.0f);
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) { ag[j][e] = 0.0f; ab[j][e] = 0.0f; }
    constexpr bool AHEAD = T * J < 2048;
    RowPart<DT, T, J> nx, ndy;
    float nr = 0.0f, nm = 0.0f;
    auto fetch = [&](long r) {
        nx.load(a.x, r, a.D, t);
        ndy.load(a.dy, r, a.D, t);
        nr = a.rstd[r];
        nm = layer ? a.mean[r] : 0.0f;
    };
    if (AHEAD && row < a.M) fetch(row);
    const float inv = 1.0f / (float)a.D;
    for (int par = 0; row < a.M; row += step, par ^= 1) {
        float xh[J][8], dy[J][8];
        if (!AHEAD) fetch(row);
        const float rstd = nr, mean = nm;
        RowPart<DT, T, J> res;
        if (a.d_residual) res.load(a.d_residual, row, a.D, t);
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int j = 0; j < J; ++j) {
            nx.v[j].get(xh[j]);
            ndy.v[j].get(dy[j]);
        }
        if (AHEAD && row + step < a.M) fetch(row + step);
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int left = a.D - (t + T * j) * 8;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                // (columns behind the row count as zero gradients; their x^ must not count either)
                xh[j][e] = e < left ? (xh[j][e] - mean) * rstd : 0.0f;
                ag[j][e] += dy[j][e] * xh[j][e];
                ab[j][e] += dy[j][e];
                dy[j][e] *= g[j][e];
                s1 += dy[j][e] * xh[j][e];
                s2 += dy[j][e];
            }
        }
        row_sum2<T>(s1, s2, slots[par]);
        s1 *= inv;
        s2 = layer ? s2 * inv : 0.0f;
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int c = (t + T * j) * 8;
            float d[8];
            float r[8];
            if (a.d_residual) res.v[j].get(r);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                d[e] = (dy[j][e] - xh[j][e] * s1 - s2) * rstd;
                if (a.d_residual) d[e] += r[e];
            }
            store8<DT>(a.dx, row * a.D + c, a.D - c, d);
        }
    }
    if (!a.part && !a.dgamma && !a.dbeta) return;
    if constexpr (G > 1) {
        __shared__ __align__(16) float join[G - 1][2][J * T * 8];
        if (grp > 0) {
#pragma unroll
            for (int j = 0; j < J; ++j) {
                store8<float>(join[grp - 1][0], (t + T * j) * 8, 8, ag[j]);
                store8<float>(join[grp - 1][1], (t + T * j) * 8, 8, ab[j]);
            }
        }
        __syncthreads();
        if (grp > 0) return;
#pragma unroll
        for (int k = 0; k < G - 1; ++k)
#pragma unroll
            for (int j = 0; j < J; ++j) {
                float u[8], w[8];
                load8<float>(join[k][0], (t + T * j) * 8, 8).get(u);
                load8<float>(join[k][1], (t + T * j) * 8, 8).get(w);
#pragma unroll
                for (int e = 0; e < 8; ++e) { ag[j][e] += u[e]; ab[j][e] += w[e]; }
            }
    }
    const long first = blockIdx.x;
    float* pg = a.part ? a.part + first * 2 * a.D : a.dgamma;
    float* pb = a.part ? a.part + first * 2 * a.D + a.D : a.dbeta;
#pragma unroll
    for (int j = 0; j < J; ++j) {
        const int c = (t + T * j) * 8;
        if (pg) store8<float>(pg, c, a.D - c, ag[j]);
        if (pb) store8<float>(pb, c, a.D - c, ab[j]);
    }
}

// Column sums of partial rows: 32 columns per workgroup, 32 slices of the rows side by side, joined in LDS in order.  A slice
// has eight loads under way, also at its end (in place of those behind it, its last row), where a plain loop would wait for one
// after another: 1132 rows of 125 columns 3.8 us, against 6.7 by 16 slices of 64 columns in a plain loop.
__global__ void __launch_bounds__(1024) sum_rows_kernel(const float* part, int rows, long rstride, long ostride, int n, float* out0,
                                                        float* out1) {
    __shared__ float red[32][32];
    const int lane = threadIdx.x & 31, sl = threadIdx.x >> 5;
    const int c = blockIdx.x * 32 + lane;
    float* out = blockIdx.y ? out1 : out0;
    const int per = (rows + 31) / 32, r0 = sl * per, left = min(rows - r0, per);
    const float* p = part + (blockIdx.y ? ostride : 0) + c + r0 * rstride;
    float s = 0.0f;
    if (c < n) {
        int r = 0;
        for (; r + 8 <= left; r += 8, p += 8 * rstride) {
#pragma unroll
            for (int k = 0; k < 8; ++k) s += p[k * rstride];
        }
        if (r < left) {
            float v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = p[min(k, left - 1 - r) * rstride];
#pragma unroll
            for (int k = 0; k < 8; ++k) s += r + k < left ? v[k] : 0.0f;
        }
    }
    red[sl][lane] = s;
    __syncthreads();
    if (sl == 0 && c < n) {
        s = red[0][lane];
#pragma unroll
        for (int k = 1; k < 32; ++k) s += red[k][lane];
        out[c] = s;
    }
}

template <typename DT, int T, int J> void fwd(const RowNormArgs& a, hipStream_t s) {
    constexpr int NT = T < 256 ? 256 : T, G = NT / T;
    // as many workgroups as the chip holds (2048 threads per CU): rows go round so that gamma and beta stay in registers
    const long need = (a.M + G - 1) / G, most = 256L * (2048 / NT);
    hipLaunchKernelGGL((rownorm_fwd_kernel<DT, T, J>), dim3((unsigned)(need < most ? need : most)), dim3(NT), 0, s, a);
}
template <typename DT, int T, int J> void bwd(const RowNormBwdArgs& a, hipStream_t s) {
    hipLaunchKernelGGL((rownorm_bwd_kernel<DT, T, J>), dim3((unsigned)a.blocks), dim3(T < 256 ? 256 : T), 0, s, a);
}

}  // namespace

// (4097 to 8192 columns: forward two workgroups of 512 threads share a CU; backward 1024 threads, of which one fits either way)
#define TFLA_BY_WIDTH(F, DT, T8K, J8K)             \
    do {                                           \
        if (a.D <= 512) F<DT, 64, 1>(a, s);        \
        else if (a.D <= 1024) F<DT, 64, 2>(a, s);  \
        else if (a.D <= 2048) F<DT, 256, 1>(a, s); \
        else if (a.D <= 4096) F<DT, 256, 2>(a, s); \
        else if (a.D <= 8192) F<DT, T8K, J8K>(a, s); \
        else F<DT, 1024, 2>(a, s);                 \
    } while (0)

int rownorm_bwd_blocks(long M, int D) {
    // workgroups = partial sums per column: enough of them to fill the chip, few enough that the partial sums stay a small
    // part of the traffic.  Where one takes no more than 8 rows a group (wide rows: 4), its sums are the results: 3.4 us of the
    // host's time and a launch saved for some 0.5 us a row (wide: 1.2).
    const int groups = D <= 1024 ? 4 : 1;
    if (M <= (D <= 4096 ? 8 * groups : 4)) return 1;
    const long most = D <= 4096 ? 512 : 256, need = (M + groups - 1) / groups;
    return (int)(need < most ? need : most);
}

hipError_t launch_rownorm_fwd(const RowNormArgs& a, hipStream_t s) {
    if (a.dtype == 1) TFLA_BY_WIDTH(fwd, bf16_t, 512, 2);
    else TFLA_BY_WIDTH(fwd, float, 512, 2);
    return hipGetLastError();
}
hipError_t launch_rownorm_bwd(const RowNormBwdArgs& a, hipStream_t s) {
    if (a.dtype == 1) TFLA_BY_WIDTH(bwd, bf16_t, 1024, 1);
    else TFLA_BY_WIDTH(bwd, float, 1024, 1);
    return hipGetLastError();
}
hipError_t launch_sum_rows(const float* part, int rows, long rstride, long ostride, int n, float* out0, float* out1, hipStream_t s) {
    // (a column sum over no rows is zero: rows = 0 fills the outputs)
    const bool both = out0 && out1;
    if (!out0 && !out1) return hipSuccess;
    const float* p = out0 ? part : part + ostride;
    hipLaunchKernelGGL(sum_rows_kernel, dim3((n + 31) / 32, both ? 2 : 1), dim3(1024), 0, s, p, rows, rstride, ostride, n,
                       out0 ? out0 : out1, out1);
    return hipGetLastError();
}

}  // namespace tfla
