// Compiled once per TFLA_Q8 (0: linear, 1: plain results, 2: parts, 3: parts of a pair, 4: a pair's gate, 5: both products of
// a small backward pass): the product kernels in 8 bits
// with that epilogue and their launcher.
#ifndef TFLA_Q8
#error "compile with -DTFLA_Q8=<0..5>"
#endif
#include "q8_wide.h"

namespace tfla {

#if TFLA_Q8 == 5

hipError_t launch_q8_both(const Q8GemmArgs& x, const Q8GemmArgs& w, const Q8Sums& sums, hipStream_t s) {
    const bool turn = (long)w.k * w.g.segs > (long)x.k * x.g.segs;
    const Q8GemmArgs& a = turn ? w : x;
    const Q8GemmArgs& b = turn ? x : w;
    Q8Both n;
    unsigned of[2];
    for (int i = 0; i < 2; ++i) {
        const GemmArgs& g = i == 0 ? a.g : b.g;
        n.tms[i] = (g.M + 63) / 64;
        n.tns[i] = (g.N + 63) / 64;
        of[i] = (unsigned)(n.tms[i] * n.tns[i] * g.batch);
    }
    n.first = of[0];
    n.both = of[0] + of[1];
    const bool many = gemm_many(n.both);
    const int threads = many ? 256 : 512;
    const unsigned all = n.both + (unsigned)((sums.planes * sums.n + threads - 1) / threads);
    // (up to a workgroup per CU two groups of wavefronts share a tile's steps)
    if (many) hipLaunchKernelGGL((gemm_q8_both_kernel<1, 3>), dim3(all), dim3(256), 0, s, a, b, n, sums);
    else hipLaunchKernelGGL((gemm_q8_both_kernel<2, 4>), dim3(all), dim3(512), 0, s, a, b, n, sums);
    return hipGetLastError();
}

#else

template <int V> hipError_t launch_q8_gemm_as(const Q8GemmArgs& a, const GemmPlan& p, hipStream_t s);
template <> hipError_t launch_q8_gemm_as<TFLA_Q8>(const Q8GemmArgs& a, const GemmPlan& p, hipStream_t s) {
    constexpr bool PAIR = TFLA_Q8 >= 3;
    constexpr int EPI = TFLA_Q8 == 0 ? EPI_LINEAR : (TFLA_Q8 == 1 ? EPI_STORE : (TFLA_Q8 == 4 ? EPI_GATED : EPI_PART));
    const int bno = PAIR ? p.bn / 2 : p.bn;
    const int tms = (a.g.M + p.bm - 1) / p.bm, tns = (a.g.N + bno - 1) / bno;
    const unsigned n = (unsigned)gemm_workgroups(p, a.g.M, a.g.N, a.g.batch, PAIR);
    // (one workgroup of the wide kernels fits a CU; the 256 of them take the tiles in turn)
    const unsigned wide = n < 256 ? n : 256;
#if TFLA_Q8 == 4
    hipLaunchKernelGGL((gemm_q8_wide_kernel<256, PAIR, EPI>), dim3(wide), dim3(256), 0, s, a, tms, tns);
#else
    const bool many = gemm_many(n);
    if (p.bn == 256) hipLaunchKernelGGL((gemm_q8_wide_kernel<256, PAIR, EPI>), dim3(wide), dim3(256), 0, s, a, tms, tns);
    else if (p.bm == 256) hipLaunchKernelGGL((gemm_q8_wide_kernel<128, PAIR, EPI>), dim3(wide), dim3(256), 0, s, a, tms, tns);
    else if (p.bm == 128) {
        if (many) hipLaunchKernelGGL((gemm_q8_kernel<128, 128, 2, 2, 2, 1, PAIR, EPI>), dim3(n), dim3(256), 0, s, a, tms, tns);
        else hipLaunchKernelGGL((gemm_q8_kernel<128, 128, 4, 2, 4, 1, PAIR, EPI>), dim3(n), dim3(512), 0, s, a, tms, tns);
    } else if constexpr (PAIR) {
        if (many) hipLaunchKernelGGL((gemm_q8_kernel<64, 128, 2, 2, 3, 1, true, EPI>), dim3(n), dim3(256), 0, s, a, tms, tns);
        else hipLaunchKernelGGL((gemm_q8_kernel<64, 128, 2, 2, 3, 2, true, EPI>), dim3(n), dim3(512), 0, s, a, tms, tns);
    } else {
        if (many) hipLaunchKernelGGL((gemm_q8_kernel<64, 64, 2, 2, 3, 1, false, EPI>), dim3(n), dim3(256), 0, s, a, tms, tns);
        else hipLaunchKernelGGL((gemm_q8_kernel<64, 64, 2, 2, 4, 2, false, EPI>), dim3(n), dim3(512), 0, s, a, tms, tns);
    }
#endif
    return hipGetLastError();
}

#endif

}  // namespace tfla
