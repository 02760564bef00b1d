// Quantisation to 8 bits in tiles of 128 x 128: a matrix, its transpose, or both in one pass; the backward pass of an activation
// with the column sums of the bias gradients on the way.  Memory-bound: every value is read once, its codes are written once per
// direction.
#include "gemm.h"
#include "q8.h"
#include "q8_internal.h"

namespace tfla {

namespace {

constexpr int TILE = Q8_TILE, NT = Q8_TILE_THREADS, WAVES = NT / 64, RPI = NT / 16;

// act(z) and act'(z) of a bf16 value, to 2^-20 (1 + |z|) of it: of a gradient that is rounded to 8 bits a value next to the border between
// two codes is worth a sixteenth of itself, so that an error of 2^-13, as the bf16 products' gelu has, would show in dx, dw and the sums.  (The
// library's functions for fp32 bound the pass instead: gated pair backward, 8192 x 10944, 406 us.)
// silu: sigma by the hardware's exponential and reciprocal.  gelu: Phi(-|z|) = exp(-z^2 / 2) h(|z|), h = t P(t), t = 1 / (1 + c |z|), P of
// degree 8 fitted to the smallest relative error over |z| <= 14.5 (with these constants in fp32 2^-24.3, evaluated in fp32 2^-21.3, with a
// reciprocal one unit off 2^-20.3; beyond, exp(-z^2 / 2) leaves fp32).  z^2 is exact.
template <int ACT> __device__ __forceinline__ float act_fine(float z, float& slope) {
    if constexpr (ACT == ACT_SILU) {
        const float g = __builtin_amdgcn_rcpf(1.0f + fast_exp2(-1.44269504f * z));
        slope = g * (1.0f + z * (1.0f - g));
        return z * g;
    } else if constexpr (ACT == ACT_GELU) {
        const float e = fast_exp2(-0.72134752f * (z * z));
        const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.26f, fabsf(z), 1.0f));
        constexpr float P[9] = {0.10375702f, 0.10305099f, 0.10278856f, 0.05196531f, 0.1587576f, -0.14778766f, 0.24873173f, -0.15149373f, 0.030230155f};
        float p = P[8];
#pragma unroll
        for (int k = 7; k >= 0; --k) p = __builtin_fmaf(t, p, P[k]);
        const float h = t * p * e, c = z < 0.0f ? h : 1.0f - h;
        slope = __builtin_fmaf(z * 0.39894228f, e, c);
        return z * c;
    } else return act_both<float>(z, ACT, slope);
}

// A tile's values, for what has to wait for its scale: bf16 where they are bf16, else fp32.  A row's columns are turned by 32 bytes from one
// block of 16 rows to the next, so that the transposed reads, 8 columns of 8 such blocks at a time, meet no bank twice.
template <typename VT> struct TileValues {
    static constexpr int PITCH = TILE + 16 / (int)sizeof(VT), STEP = 32 / (int)sizeof(VT);
    VT v[TILE * PITCH];
    static __device__ __forceinline__ int place(int row, int c) { return row * PITCH + ((c + STEP * (row >> 4)) & (TILE - 1)); }
};
template <typename VT> struct TileMemory {
    TileValues<VT> values;
    uint32_t most[WAVES];
};
template <typename DT, int MODE> struct Kept { typedef float type; };
template <> struct Kept<bf16_t, Q8_VALUES> { typedef bf16_t type; };

// Eight values that were read `shift` places before their own, from inside the row: moved into place, zeros behind the row's end.  (A read that
// ends with the row needs no branch, and nothing waits for it; element by element, in a branch, the twelve reads of a pair's tile waited one after
// another: 1000 x 1365 20.5 us, x 1360 14.2.)
__device__ __forceinline__ void into_place(Vec8<bf16_t>& x, int shift) {
    uint64_t lo = (uint64_t)x.w[1] << 32 | x.w[0], hi = (uint64_t)x.w[3] << 32 | x.w[2];
    if (shift & 4) { lo = hi; hi = 0; }
    const int bits = (shift & 3) * 16;
    lo = lo >> bits | (hi << 1) << (63 - bits);
    hi >>= bits;
    if (shift >= 8) { lo = 0; hi = 0; }
    x.w = u32x4{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
}
__device__ __forceinline__ void into_place(Vec8<float>& x, int shift) {
#pragma unroll
    for (int b = 4; b > 0; b >>= 1)
        if (shift & b) {
#pragma unroll
            for (int e = 0; e < 8; ++e) x.v[e] = e + b < 8 ? x.v[e + b] : 0.0f;
        }
    if (shift >= 8) x.zero();
}

// Tile (bx, by).  By rows, thread (g = t % 16, r = t / 16) takes the columns 8 g ... of the rows r and r + 64: what a row needs is
// done there, from registers, and the values are left in LDS for what a block or a column needs.  By columns, a thread takes 16 rows of a
// column, eight neighbouring lanes all of it, so that neither scales nor sums need LDS.  A pair's second gradient waits in registers: a pair's
// backward 8192 x 10944 takes 193 us (4.6 TB/s of its 898 MB; 265 with a workgroup for each gradient, which computes the activation twice
// and by rows from LDS), a weight of 10944 x 4096 with its transpose 39.5 (4.6 TB/s).  512 threads with twice the rows each have as much in flight
// in a full card, but where there are few tiles, their instructions, which each workgroup fetches once, are twice as many (1000 x 1365: pair
// 18.0 us against 15.4, fp32 with its transpose 9.4 against 8.6).
template <typename DT, int MODE, int ACT, typename MEM> __device__ __forceinline__ void q8_tile(const Q8TileArgs& a, int bx, int by, MEM& m) {
    typedef typename Kept<DT, MODE>::type VT;
    typedef TileValues<VT> Values;
    constexpr int ROWS = TILE / RPI, P = MODE == Q8_PAIR ? 2 : 1;
    const int t = threadIdx.x, g = t & 15;
    const long r0 = (long)bx * TILE;
    const int c0 = by * TILE, c = c0 + g * 8, left = a.N - c;
    const bool blocks = a.rows > 1;
    VT* const kept = reinterpret_cast<VT*>(&m);
    Vec8<DT> x[ROWS], z[ROWS], u[ROWS];
    const int behind = left >= 8 ? 0 : min(8 - left, 8);      // by how much a read ends behind the row
    if (a.N >= 8) {
#pragma unroll
        for (int k = 0; k < ROWS; ++k) {
            const long row = min(r0 + (t >> 4) + k * RPI, a.M - 1), at = row * a.N + min(c, a.N - 8);
            x[k].load(a.x, at);
            if constexpr (MODE != Q8_VALUES) z[k].load(a.z, at);
            if constexpr (MODE == Q8_PAIR) u[k].load(a.u, at);
        }
    } else {
#pragma unroll
        for (int k = 0; k < ROWS; ++k) {
            const long row = min(r0 + (t >> 4) + k * RPI, a.M - 1);
            x[k] = load8<DT>(a.x, row * a.N + c, left);
            if constexpr (MODE != Q8_VALUES) z[k] = load8<DT>(a.z, row * a.N + c, left);
            if constexpr (MODE == Q8_PAIR) u[k] = load8<DT>(a.u, row * a.N + c, left);
        }
    }
    float second[MODE == Q8_PAIR ? ROWS : 1][8];
    uint32_t all = 0;
    auto keep = [&](int i, const float (&v)[8]) {
        VT* d = kept + Values::place(i, g * 8);
        if constexpr (sizeof(VT) == 4) {
            *reinterpret_cast<f32x4*>(d) = f32x4{v[0], v[1], v[2], v[3]};
            *reinterpret_cast<f32x4*>(d + 4) = f32x4{v[4], v[5], v[6], v[7]};
        }
    };
    auto codes = [&](const Q8Out& o, int i, const float (&v)[8]) {
        const uint32_t most = q8_largest(v);
        all = max(all, most);
        if (!o.q || blocks) return;
        const long row = r0 + i;
        const uint32_t s = q8_scale(lanes_max<16>(most));
        if (row < a.M) {
            q8_store8(o.q + row * o.ldq + c, q8_codes8(v, q8_power(s)), o.wq - c);
            if (g == 0) o.s[(long)by * o.lds + row] = (uint8_t)s;
        }
    };
#pragma unroll
    for (int k = 0; k < ROWS; ++k) {
        const int i = (t >> 4) + k * RPI;
        // (rows behind the last one have read it again)
        const int shift = r0 + i < a.M ? (a.N >= 8 ? behind : 0) : 8;
        if (__any(shift > 0)) {
            into_place(x[k], shift);
            if constexpr (MODE != Q8_VALUES) into_place(z[k], shift);
            if constexpr (MODE == Q8_PAIR) into_place(u[k], shift);
        }
        float v[8];
        x[k].get(v);
        if constexpr (sizeof(VT) == 2) *reinterpret_cast<u32x4*>(kept + Values::place(i, g * 8)) = x[k].w;
        if constexpr (MODE != Q8_VALUES) {
            float zf[8], uf[8];
            z[k].get(zf);
            if constexpr (MODE == Q8_PAIR) u[k].get(uf);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float slope;
                const float value = act_fine<ACT>(zf[e], slope);
                if constexpr (MODE == Q8_PAIR) {
                    second[k][e] = v[e] * value;
                    v[e] *= uf[e];
                }
                v[e] *= slope;
            }
        }
        codes(a.out[0], i, v);
        keep(i, v);
        if constexpr (MODE == Q8_PAIR) {
            codes(a.out[1], i, second[k]);
            // (row after row, so that the registers do for two workgroups on a CU)
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    uint32_t whole = 0;         // the scale of a block
    if (blocks) {
        all = lanes_max<64>(all);
        if ((t & 63) == 0) m.most[t >> 6] = all;
    }
    __syncthreads();
    if (blocks) {
        const Q8Out& o = a.out[0];
#pragma unroll
        for (int w = 0; w < WAVES; ++w) whole = max(whole, m.most[w]);
        whole = q8_scale(whole);
        if (t == 0 && o.q) o.s[(long)by * o.lds + bx] = (uint8_t)whole;
        if (t == 0 && o.qt) o.st[(long)bx * o.ldst + by] = (uint8_t)whole;
        if (o.q) {
#pragma unroll 1
            for (int i = t >> 4; i < TILE && r0 + i < a.M; i += RPI) {
                float v[8];
                load8<VT>(kept, Values::place(i, g * 8), 8).get(v);
                q8_store8(o.q + (r0 + i) * o.ldq + c, q8_codes8(v, q8_power(whole)), o.wq - c);
            }
        }
    }
#pragma unroll
    for (int p = 0; p < P; ++p) {
        const Q8Out& o = a.out[p];
        float* db = a.part ? a.part + ((long)bx * P + p) * a.ldp : a.db[p];
        if constexpr (MODE == Q8_PAIR) {
            if (p > 0) {
                __syncthreads();
#pragma unroll
                for (int k = 0; k < ROWS; ++k) keep((t >> 4) + k * RPI, second[k]);
                __syncthreads();
            }
        }
        if (!o.qt && !db) continue;
        // rows of the transpose: eight pieces of 16 codes each
#pragma unroll 1
        for (int i = t; i < TILE * 8; i += NT) {
            const int col = i >> 3, at = (i & 7) * 16;
            const VT* d = kept + Values::place(at, col);        // (whole blocks of 16 rows are turned alike)
            float v[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) v[e] = (float)d[e * Values::PITCH];
            if (db) {
                float s = v[0];
#pragma unroll
                for (int e = 1; e < 16; ++e) s += v[e];
                s = lanes_sum<8>(s);
                if (at == 0 && c0 + col < a.N) db[c0 + col] = s;
            }
            if (!o.qt) continue;
            uint32_t s = whole;
            if (!blocks) {
                uint32_t most = q8_largest(v);
                most = max(most, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)most, 0xb1, 0xf, 0xf, true));
                most = max(most, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)most, 0x4e, 0xf, 0xf, true));
                s = q8_scale(max(most, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)most, 0x141, 0xf, 0xf, true)));
                if (at == 0 && c0 + col < a.N) o.st[(long)bx * o.ldst + c0 + col] = (uint8_t)s;
            }
            const long n = o.wt - r0 - at;
            if (c0 + col >= a.N || n <= 0) continue;
            const float power = q8_power(s);
            uint32_t w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = q8_codes(v[4 * e], v[4 * e + 1], v[4 * e + 2], v[4 * e + 3], power);
            uint8_t* to = o.qt + (long)(c0 + col) * o.ldt + r0 + at;
            if (n >= 16) __builtin_memcpy(to, w, 16);
            else {
                for (int e = 0; e < n; ++e) {
                    uint32_t q = w[0];
                    q = e >= 4 ? w[1] : q;
                    q = e >= 8 ? w[2] : q;
                    q = e >= 12 ? w[3] : q;
                    to[e] = (uint8_t)(q >> (8 * (e & 3)));
                }
            }
        }
    }
}

// Rows of bytes at any address to rows of ldd bytes: block x of `blocks` of THREADS, 16 bytes a lane.  A row's end is read from inside the row, as
// a tile's (byte by byte, in a branch, a product of 33 x 1365 x 1000 with
// its copies took 15.6 us, so 10.5).
template <int THREADS> __device__ __forceinline__ void q8_repack(const Q8RepackArgs& a, unsigned block, unsigned blocks) {
    const unsigned per = (unsigned)(a.ldd >> 4);
    for (int q = 0; q < a.count; ++q) {
        const long all = a.rows[q] * per;
        const bool narrow = all < 1l << 32;
        for (long i = (long)block * THREADS + threadIdx.x; i < all; i += (long)blocks * THREADS) {
            const long r = narrow ? (long)((unsigned)i / per) : i / per;
            const int c = (int)(i - r * per) * 16, behind = max(c + 16 - a.cols, 0);      // how far a read goes past the row
            const uint8_t* p = a.src[q] + r * a.cols + c;
            u32x4 w = {0u, 0u, 0u, 0u};
            if (a.cols >= 16) {
                uint64_t d[2];
                __builtin_memcpy(d, p - behind, 16);
                uint64_t lo = behind & 8 ? d[1] : d[0], hi = behind & 8 ? 0 : d[1];
                const int bits = (behind & 7) * 8;
                lo = lo >> bits | (hi << 1) << (63 - bits);
                hi >>= bits;
                w = u32x4{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
            } else {
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (c + e < a.cols) w[e >> 2] |= (uint32_t)p[e] << (8 * (e & 3));
            }
            *reinterpret_cast<u32x4*>(a.dst[q] + r * a.ldd + c) = w;
        }
    }
}
constexpr int COPY = 256;
__global__ void __launch_bounds__(COPY) q8_repack_kernel(Q8RepackArgs a) { q8_repack<COPY>(a, blockIdx.x, gridDim.x); }

// Which tile workgroup i takes.  Rows of codes that are no multiple of 64 bytes: neighbours share cache lines, and an XCD takes a range of them, so that it
// writes whole ones (16384 x 4097, four matrices in turn, 46.0 us, one after another 56.6; with the transpose 61.3, 79.4).  Otherwise one after
// another (16384 x 4096 38.5, in ranges 46.4; 10944 x 4096 with its transpose 40.3, 44.3).
__device__ __forceinline__ unsigned tile_of(const Q8TileArgs& a, unsigned i, unsigned n) { return a.N % 64 ? xcd_range(i, n) : i; }

// The tiles of a, those of a row of tiles next to each other, then the tiles of b (plain values; none where b.M is 0), then copies: of all of
// these workgroups the ones from `first` on.
template <typename DT, int MODE, int ACT> __global__ void __launch_bounds__(NT, 8) q8_tiles_kernel(Q8TileArgs a, Q8TileArgs b, Q8RepackArgs rp,
                                                                                                   unsigned na, unsigned nb, unsigned copies, unsigned first) {
    __shared__ __align__(16) TileMemory<typename Kept<DT, MODE>::type> m;
    const unsigned i = first + blockIdx.x;
    if (i < na) {
        const unsigned across = (a.N + TILE - 1) / TILE, t = tile_of(a, i, na);
        q8_tile<DT, MODE, ACT>(a, t / across, t % across, m);
    } else if (i < na + nb) {
        const unsigned across = (b.N + TILE - 1) / TILE, t = tile_of(b, i - na, nb);
        q8_tile<DT, Q8_VALUES, ACT_NONE>(b, t / across, t % across, m);
    } else {
        q8_repack<NT>(rp, i - na - nb, copies);
    }
}

// A pair's gate behind partial results, which it adds in order.  Sixteen lanes hold 128 columns of a row, eight each.  4 x 10944: 4 us, most of
// it the launch.
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
    const uint32_t s = q8_scale(lanes_max<16>(q8_largest(h)));
    if (left <= 0) return;
    q8_store8(a.h.q + m * x.N + n, q8_codes8(h, q8_power(s)), left);
    if ((threadIdx.x & 15) == 0) a.h.s[(long)(n / Q8_GROUP) * x.M + m] = (uint8_t)s;
    if (a.hc) store8<bf16_t>(a.hc, m * x.N + n, left, h);
}

// workgroups of a launch's copies: a piece a thread, up to as many as the chip holds (beside a quantisation half of them)
unsigned copies_of(const Q8RepackArgs& a, int threads, unsigned most) {
    long all = 0;
    for (int q = 0; q < a.count; ++q) all = max(all, a.rows[q] * (a.ldd >> 4));
    const long n = (all + threads - 1) / threads;
    return n < most ? (unsigned)n : most;
}
template <typename DT, int MODE, int ACT> void tiles(const Q8TileArgs& a, const Q8TileArgs& b, const Q8RepackArgs& rp, hipStream_t s) {
    const unsigned na = q8_tiles(a.M, a.N), nb = q8_tiles(b.M, b.N), copies = copies_of(rp, NT, 256), all = na + nb + copies;
    for (unsigned first = 0; first < all; first += q8_launch(first, all))
        hipLaunchKernelGGL((q8_tiles_kernel<DT, MODE, ACT>), dim3(q8_launch(first, all)), dim3(NT), 0, s, a, b, rp, na, nb, copies, first);
}
template <int MODE> void by_act(const Q8TileArgs& a, const Q8TileArgs& b, const Q8RepackArgs& rp, hipStream_t s) {
    if (a.act == ACT_SILU) tiles<bf16_t, MODE, ACT_SILU>(a, b, rp, s);
    else if (a.act == ACT_GELU) tiles<bf16_t, MODE, ACT_GELU>(a, b, rp, s);
    else if (MODE == Q8_ACT || a.act == ACT_RELU) tiles<bf16_t, MODE, ACT_RELU>(a, b, rp, s);
    else if constexpr (MODE == Q8_PAIR) tiles<bf16_t, MODE, ACT_NONE>(a, b, rp, s);     // (a single product without an activation: Q8_VALUES)
}

}  // namespace

hipError_t launch_q8_tiles(const Q8TileArgs& a, const Q8TileArgs& b, const Q8RepackArgs& rp, hipStream_t s) {
    if (a.dtype != 1) tiles<float, Q8_VALUES, ACT_NONE>(a, b, rp, s);
    else if (a.mode == Q8_PAIR) by_act<Q8_PAIR>(a, b, rp, s);
    else if (a.mode == Q8_ACT) by_act<Q8_ACT>(a, b, rp, s);
    else tiles<bf16_t, Q8_VALUES, ACT_NONE>(a, b, rp, s);
    return hipGetLastError();
}

hipError_t launch_q8_repack(const Q8RepackArgs& a, hipStream_t s) {
    if (a.count == 0) return hipSuccess;
    hipLaunchKernelGGL(q8_repack_kernel, dim3(copies_of(a, COPY, 2048)), dim3(COPY), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_q8_gated_join(const Q8GemmArgs& a, hipStream_t s) {
    const dim3 grid((unsigned)((a.g.M + 3) / 4), (unsigned)((a.g.N + 511) / 512));
    hipLaunchKernelGGL(q8_gated_join_kernel, grid, dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace tfla
