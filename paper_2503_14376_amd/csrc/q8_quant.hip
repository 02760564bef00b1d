// Quantisation to 8 bits in tiles of 128 x 128: a matrix, its transpose, or both in one pass; the backward pass of an activation
// with the column sums of the bias gradients on the way.  Memory-bound: every value is read once, its codes are written once per
// direction.
#include "gemm_epilogue.h"
#include "q8.h"
#include "q8_internal.h"

namespace tfla {

namespace {

constexpr int TILE = 128, NT = 512, R = 4, WAVES = NT / 64;

// Thread (g = t % 16, r = t / 16) holds the columns 8 g ... of the rows 4 r ... 4 r + 3 of the tile.
template <typename DT, int MODE> __global__ void __launch_bounds__(NT, 2) q8_tile_kernel(Q8TileArgs a) {
    constexpr int P = MODE == Q8_PAIR ? 2 : 1, PITCH = TILE + 4;
    __shared__ uint32_t colmax[WAVES][TILE];
    __shared__ float colsum[WAVES][TILE];
    __shared__ uint32_t turn[TILE * PITCH / 4];
    const int t = threadIdx.x, g = t & 15, rg = t >> 4, wave = t >> 6;
    const long r0 = (long)blockIdx.x * TILE;
    const int c0 = blockIdx.y * TILE, c = c0 + g * 8, left = a.N - c;
    float v[P][R][8];
    {
        Vec8<DT> x[R], z[R], u[R];
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const long row = r0 + rg * R + i;
            const int n = row < a.M ? left : 0;
            x[i] = load8<DT>(a.x, row * a.N + c, n);
            if constexpr (MODE != Q8_VALUES) z[i] = load8<DT>(a.z, row * a.N + c, n);
            if constexpr (MODE == Q8_PAIR) u[i] = load8<DT>(a.u, row * a.N + c, n);
        }
#pragma unroll
        for (int i = 0; i < R; ++i) {
            x[i].get(v[0][i]);
            if constexpr (MODE != Q8_VALUES) {
                float zf[8], uf[8];
                z[i].get(zf);
                if constexpr (MODE == Q8_PAIR) u[i].get(uf);
                // (the activation as for fp32: a value next to a border between two codes is worth a sixteenth of itself)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    float slope;
                    const float value = act_both<float>(zf[e], a.act, slope), d = v[0][i][e];
                    if constexpr (MODE == Q8_PAIR) {
                        v[0][i][e] = d * uf[e] * slope;
                        v[1][i][e] = d * value;
                    } else {
                        v[0][i][e] = d * slope;
                    }
                }
            }
        }
    }
#pragma unroll
    for (int p = 0; p < P; ++p) {
        const Q8Out& o = a.out[p];
        float* db = a.part ? a.part + ((long)blockIdx.x * P + p) * a.ldp : a.db[p];
        if (p > 0) __syncthreads();
        uint32_t cm[8];
        if (db || o.qt || a.rows > 1) {
            float cs[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                cm[e] = 0;
                cs[e] = 0.0f;
#pragma unroll
                for (int i = 0; i < R; ++i) {
                    cm[e] = max(cm[e], q8_magnitude(v[p][i][e]));
                    cs[e] += v[p][i][e];
                }
            }
            if (db) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    cs[e] += __shfl_xor(cs[e], 16, 64);
                    cs[e] += __shfl_xor(cs[e], 32, 64);
                    if ((t & 48) == 0) colsum[wave][g * 8 + e] = cs[e];
                }
            }
            if (o.qt || a.rows > 1) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    cm[e] = max(cm[e], (uint32_t)__shfl_xor((int)cm[e], 16, 64));
                    cm[e] = max(cm[e], (uint32_t)__shfl_xor((int)cm[e], 32, 64));
                    if ((t & 48) == 0) colmax[wave][g * 8 + e] = cm[e];
                }
            }
            __syncthreads();
            if (o.qt || a.rows > 1) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    cm[e] = colmax[0][g * 8 + e];
#pragma unroll
                    for (int w = 1; w < WAVES; ++w) cm[e] = max(cm[e], colmax[w][g * 8 + e]);
                }
            }
            if (db && t < TILE && c0 + t < a.N) {
                float s = colsum[0][t];
#pragma unroll
                for (int w = 1; w < WAVES; ++w) s += colsum[w][t];
                db[c0 + t] = s;
            }
        }
        uint32_t whole = 0;         // rows = 128: the tile's largest magnitude
        if (a.rows > 1) {
#pragma unroll
            for (int e = 0; e < 8; ++e) whole = max(whole, cm[e]);
            whole = lanes_max<16>(whole);
        }
        if (o.q) {
#pragma unroll
            for (int i = 0; i < R; ++i) {
                const long row = r0 + rg * R + i;
                const uint32_t s = q8_scale(a.rows > 1 ? whole : lanes_max<16>(q8_magnitude8(v[p][i])));
                const u32x2 w = q8_codes8(v[p][i], q8_inverse(s));
                if (row < a.M) {
                    q8_store8(o.q + row * o.ldq + c, w, o.wq - c);
                    if (g == 0 && a.rows == 1) o.s[(long)blockIdx.y * o.lds + row] = (uint8_t)s;
                }
            }
            if (a.rows > 1 && t == 0) o.s[(long)blockIdx.y * o.lds + blockIdx.x] = (uint8_t)q8_scale(whole);
        }
        if (o.qt) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t s = q8_scale(a.rows > 1 ? whole : cm[e]);
                static_assert(R == 4, "a word of four rows");
                turn[((g * 8 + e) * PITCH + rg * R) / 4] = q8_codes(v[p][0][e], v[p][1][e], v[p][2][e], v[p][3][e], q8_inverse(s));
                if (rg == 0 && a.rows == 1 && c + e < a.N) o.st[(long)blockIdx.x * o.ldst + c + e] = (uint8_t)s;
            }
            if (a.rows > 1 && t == 0) o.st[(long)blockIdx.x * o.ldst + blockIdx.y] = (uint8_t)q8_scale(whole);
            __syncthreads();
            // rows of the transpose: eight pieces of 16 codes each
#pragma unroll
            for (int k = 0; k < TILE * 8 / NT; ++k) {
                const int i = t + k * NT, col = i >> 3, at = (i & 7) * 16;
                if (c0 + col >= a.N || r0 + at >= o.wt) continue;
                uint32_t w[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = turn[(col * PITCH + at) / 4 + e];
                uint8_t* d = o.qt + (long)(c0 + col) * o.ldt + r0 + at;
                const long n = o.wt - r0 - at;
                if (n >= 16) __builtin_memcpy(d, w, 16);
                else {
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        if (e < n) d[e] = (uint8_t)(w[e >> 2] >> (8 * (e & 3)));
                }
            }
        }
    }
}

__global__ void __launch_bounds__(256) q8_repack_kernel(Q8RepackArgs a) {
    const int c = (blockIdx.y * 64 + (threadIdx.x & 63)) * 16, q = blockIdx.z;
    if (c >= a.ldd) return;
    const long step = (long)gridDim.x * 4;
    for (long r = (long)blockIdx.x * 4 + (threadIdx.x >> 6); r < a.rows[q]; r += step) {
        const uint8_t* p = a.src[q] + r * a.cols + c;
        u32x4 w = {0u, 0u, 0u, 0u};
        if (c + 16 <= a.cols) __builtin_memcpy(&w, p, 16);
        else {
#pragma unroll
            for (int e = 0; e < 16; ++e)
                if (c + e < a.cols) w[e >> 2] |= (uint32_t)p[e] << (8 * (e & 3));
        }
        *reinterpret_cast<u32x4*>(a.dst[q] + r * a.ldd + c) = w;
    }
}

// Sixteen lanes hold 128 columns of a row, eight each.
__global__ void __launch_bounds__(256) q8_gated_join_kernel(Q8GemmArgs a) {
    const GemmArgs& x = a.g;
    const int n = (blockIdx.y * 64 + (threadIdx.x & 63)) * 8, left = x.N - n;
    const long m = (long)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (m >= x.M) return;           // (whole wavefronts)
    float v[2][8];
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
        for (int e = 0; e < 8; ++e) v[p][e] = 0.0f;
    if (left > 0) {
#pragma unroll 4
        for (int q = 0; q < x.split; ++q)
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                float t[8];
                load8<float>(x.part, (((long)q * 2 + p) * x.M + m) * x.ld_part + n, 8).get(t);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[p][e] += t[e];
            }
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            if (x.bias[p]) {
                float b[8];
                load8<float>(x.bias[p], n, left).get(b);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[p][e] += b[e];
            }
            if (x.z[p]) store8<bf16_t>(x.z[p], m * x.N + n, left, v[p]);
        }
    }
    float h[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) h[e] = e < left ? act_value<bf16_t>(v[0][e], x.act) * v[1][e] : 0.0f;
    const uint32_t s = q8_scale(lanes_max<16>(q8_magnitude8(h)));
    if (left <= 0) return;
    q8_store8(a.h.q + m * x.N + n, q8_codes8(h, q8_inverse(s)), left);
    if ((threadIdx.x & 15) == 0) a.h.s[(long)(n / Q8_GROUP) * x.M + m] = (uint8_t)s;
    if (a.hc) store8<bf16_t>(a.hc, m * x.N + n, left, h);
}

template <typename DT> hipError_t tiles(const Q8TileArgs& a, hipStream_t s) {
    const dim3 grid((unsigned)((a.M + TILE - 1) / TILE), (unsigned)((a.N + TILE - 1) / TILE));
    if (a.mode == Q8_VALUES) hipLaunchKernelGGL((q8_tile_kernel<DT, Q8_VALUES>), grid, dim3(NT), 0, s, a);
    else if constexpr (sizeof(DT) == 2) {
        if (a.mode == Q8_ACT) hipLaunchKernelGGL((q8_tile_kernel<DT, Q8_ACT>), grid, dim3(NT), 0, s, a);
        else hipLaunchKernelGGL((q8_tile_kernel<DT, Q8_PAIR>), grid, dim3(NT), 0, s, a);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_q8_tiles(const Q8TileArgs& a, hipStream_t s) { return a.dtype == 1 ? tiles<bf16_t>(a, s) : tiles<float>(a, s); }

hipError_t launch_q8_repack(const Q8RepackArgs& a, hipStream_t s) {
    if (a.count == 0) return hipSuccess;
    long most = 1;
    for (int q = 0; q < a.count; ++q) most = a.rows[q] > most ? a.rows[q] : most;
    const long n = (most + 3) / 4;
    const dim3 grid((unsigned)(n < 1024 ? n : 1024), (unsigned)((a.ldd + 1023) / 1024), a.count);
    hipLaunchKernelGGL(q8_repack_kernel, grid, dim3(256), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_q8_gated_join(const Q8GemmArgs& a, hipStream_t s) {
    const dim3 grid((unsigned)((a.g.M + 3) / 4), (unsigned)((a.g.N + 511) / 512));
    hipLaunchKernelGGL(q8_gated_join_kernel, grid, dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace tfla
