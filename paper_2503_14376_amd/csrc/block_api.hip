// C ABI of the residual block's operators: argument checks, workspace layout and kernel sequence of the norm over a model's
// columns, the linear projection and the gated projection pair.  See include/tfla_mlstm.h for the contract.
#include "../../include/tfla_mlstm.h"
#include "block_internal.h"
#include "host_util.h"
#include "profiler.h"

using namespace tfla;

namespace {

constexpr int MAX_ROWS = 1 << 24, MAX_COLS = 1 << 20, MAX_NORM_COLS = 16384;
constexpr long MAX_ELEMS = 1L << 36;

inline size_t esize(int dtype) { return dtype == TFLA_BF16 ? 2 : 4; }
// pitch of a row in the workspace: the passes that write there store eight elements at a time
inline long padded(int n) { return (n + 7L) & ~7L; }
// whether a product's operand is copied into the workspace: the bf16 kernels bring rows into LDS by 16-byte requests, which
// want addresses in multiples of that; the fp32 kernels read any rows in place (bwd 14251 x 5170 x 84: 359 us, 495 with a copy)
inline bool moved(int cols, bool off, int dtype) { return dtype == TFLA_BF16 && (cols % 8 != 0 || off); }

int check_norm(int M, int D, int dtype, int kind) {
    if (dtype != TFLA_F32 && dtype != TFLA_BF16) return TFLA_ERR_ENUM;
    if (kind != TFLA_NORM_RMS && kind != TFLA_NORM_LAYER) return TFLA_ERR_ENUM;
    if (M < 0 || M > MAX_ROWS || D <= 0 || D > MAX_NORM_COLS) return TFLA_ERR_SHAPE;
    return TFLA_OK;
}
int check_product(int M, int K, int N, int act, int dtype) {
    if (dtype != TFLA_F32 && dtype != TFLA_BF16) return TFLA_ERR_ENUM;
    if (act < TFLA_ACT_NONE || act > TFLA_ACT_RELU) return TFLA_ERR_ENUM;
    if (M < 0 || M > MAX_ROWS || K <= 0 || K > MAX_COLS || N <= 0 || N > MAX_COLS) return TFLA_ERR_SHAPE;
    if ((long)M * K > MAX_ELEMS || (long)M * N > MAX_ELEMS || (long)N * K > MAX_ELEMS) return TFLA_ERR_SHAPE;
    return TFLA_OK;
}

// Where the pieces of a product's workspace lie.  `pair`: the gated pair.  The same walk serves the query (unaligned as the
// caller says) and the call (as the pointers are).
struct FwdLayout {
    size_t x, w0, w1, part, bytes;
    GemmPlan plan; bool rows, move_x, move_w;
};
FwdLayout fwd_layout(int M, int K, int N, int dtype, bool pair, bool x_off, bool w_off) {
    FwdLayout l{};
    l.move_x = moved(K, x_off, dtype);
    l.move_w = moved(K, w_off, dtype);
    l.rows = gemm_rows_applies(M, N, K, pair, dtype, l.move_x || l.move_w);
    if (l.rows) return l;      // that kernel reads the tensors where they are
    const size_t e = esize(dtype), Kp = padded(K);
    l.plan = gemm_plan(M, N, K, 1, 1, pair, dtype);
    Carver c(nullptr);
    if (l.move_x) { l.x = c.off; c.take(M * Kp * e); }
    if (l.move_w) {
        l.w0 = c.off; c.take(N * Kp * e);
        if (pair) { l.w1 = c.off; c.take(N * Kp * e); }
    }
    l.part = c.off;
    if (l.plan.split > 1) c.take((size_t)l.plan.split * (pair ? 2 : 1) * M * (((size_t)N + 7) & ~(size_t)7) * sizeof(float));
    l.bytes = c.off;
    return l;
}
// what a query answers: with tensors off 16 bytes, which of them is not known (few rows of x or w then need no workspace, of the
// others may)
size_t fwd_bytes(int M, int K, int N, int dtype, bool pair, bool off) {
    if (M == 0) return 0;
    const size_t in = fwd_layout(M, K, N, dtype, pair, false, false).bytes, out = off ? fwd_layout(M, K, N, dtype, pair, true, true).bytes : 0;
    return in > out ? in : out;
}
struct BwdLayout {
    size_t dz0, dz1, x, w0, w1, dbpart, part, bytes;
    GemmPlan plan_dx, plan_dw; bool move_dz, move_x, move_w;
};
BwdLayout bwd_layout(int M, int K, int N, int act, int dtype, bool pair, bool dy_off, bool x_off, bool w_off) {
    BwdLayout l{};
    const size_t e = esize(dtype), Kp = padded(K), Np = padded(N);
    l.plan_dx = gemm_plan(M, K, N, pair ? 2 : 1, 1, 0, dtype);
    l.plan_dw = gemm_plan(N, K, M, 1, pair ? 2 : 1, 0, dtype);
    l.move_dz = pair || act != TFLA_ACT_NONE || moved(N, dy_off, dtype);
    l.move_x = moved(K, x_off, dtype);
    l.move_w = moved(K, w_off, dtype);
    Carver c(nullptr);
    if (l.move_dz) {
        l.dz0 = c.off; c.take(M * Np * e);
        if (pair) { l.dz1 = c.off; c.take(M * Np * e); }
    }
    if (l.move_x) { l.x = c.off; c.take(M * Kp * e); }
    if (l.move_w) {
        l.w0 = c.off; c.take(N * Kp * e);
        if (pair) { l.w1 = c.off; c.take(N * Kp * e); }
    }
    l.dbpart = c.off; c.take((size_t)act_bwd_row_blocks(M, N) * (pair ? 2 : 1) * Np * sizeof(float));
    // (the two products run one after the other and share the memory of their partial results)
    const size_t K8 = ((size_t)K + 7) & ~(size_t)7;
    const size_t pdx = l.plan_dx.split > 1 ? (size_t)l.plan_dx.split * M * K8 * sizeof(float) : 0;
    const size_t pdw = l.plan_dw.split > 1 ? (size_t)l.plan_dw.split * (pair ? 2 : 1) * N * K8 * sizeof(float) : 0;
    l.part = c.off; c.take(pdx > pdw ? pdx : pdw);
    l.bytes = c.off;
    return l;
}

int product_fwd(const void* x, const void* const (&w)[2], const float* const (&bias)[2], const void* residual, int M, int K, int N, int act,
                int dtype, void* out, void* const (&z)[2], bool pair, void* workspace, size_t workspace_bytes, hipStream_t s) {
    const FwdLayout l = fwd_layout(M, K, N, dtype, pair, off16(x), off16(w[0]) || (pair && off16(w[1])));
    const int rc = check_workspace(workspace, workspace_bytes, l.bytes);
    if (rc != TFLA_OK) return rc;
    char* ws = reinterpret_cast<char*>(workspace);
    const long Kp = padded(K);
    GemmArgs g{};
    g.A[0] = x; g.B[0] = w[0]; g.B[1] = w[1]; g.lda = K; g.ldb = K;
    g.M = M; g.N = N; g.K = K; g.segs = 1; g.batch = 1; g.pair = pair;
    g.bias[0] = bias[0]; g.bias[1] = bias[1]; g.residual = residual; g.out[0] = out; g.z[0] = z[0]; g.z[1] = z[1];
    g.act = act; g.dtype = dtype;
    if (l.rows) {
        TFLA_LAUNCH(K_GEMM, launch_gemm_rows(g, s));
        return TFLA_OK;
    }
    RepackArgs rp{};
    rp.cols = K; rp.ldd = Kp;
    if (l.move_x) {
        rp.add(x, ws + l.x, M);
        g.A[0] = ws + l.x; g.lda = Kp;
    }
    if (l.move_w) {
        rp.add(w[0], ws + l.w0, N);
        if (pair) rp.add(w[1], ws + l.w1, N);
        g.B[0] = ws + l.w0; g.B[1] = pair ? ws + l.w1 : nullptr; g.ldb = Kp;
    }
    if (rp.count > 0) TFLA_LAUNCH(K_ACT_BWD, launch_repack(rp, s));
    g.split = l.plan.split; g.part = reinterpret_cast<float*>(ws + l.part); g.ld_part = (N + 7) & ~7;
    TFLA_LAUNCH(K_GEMM, launch_gemm(g, l.plan, false, false, pair ? EPI_GATED : EPI_LINEAR, s));
    return TFLA_OK;
}

int product_bwd(const void* x, const void* const (&w)[2], const void* dy, const void* z, const void* u, int M, int K, int N, int act,
                int dtype, void* dx, void* const (&dw)[2], float* const (&db)[2], bool pair, void* workspace, size_t workspace_bytes,
                hipStream_t s) {
    const BwdLayout l = bwd_layout(M, K, N, act, dtype, pair, off16(dy), off16(x), off16(w[0]) || (pair && off16(w[1])));
    const int rc = check_workspace(workspace, workspace_bytes, l.bytes);
    if (rc != TFLA_OK) return rc;
    char* ws = reinterpret_cast<char*>(workspace);
    const long Kp = padded(K), Np = padded(N);
    const bool want_dw = dw[0] || dw[1], want_db = db[0] || db[1];
    const void* dz[2] = {dy, nullptr};
    long ldz = N;
    if (l.move_dz) { dz[0] = ws + l.dz0; dz[1] = pair ? ws + l.dz1 : nullptr; ldz = Np; }
    const bool store_dz = l.move_dz && (dx || want_dw);      // (bias gradients alone need the sums only)
    if (M > 0 && (store_dz || want_db)) {
        ActBwdArgs a{};
        a.dy = dy; a.z = act == TFLA_ACT_NONE && !pair ? nullptr : z; a.u = u;
        a.dz0 = store_dz ? ws + l.dz0 : nullptr; a.dz1 = store_dz && pair ? ws + l.dz1 : nullptr;
        const bool direct = act_bwd_row_blocks(M, N) == 1;       // the sums need not be joined
        a.part = want_db && !direct ? reinterpret_cast<float*>(ws + l.dbpart) : nullptr;
        a.db0 = direct ? db[0] : nullptr; a.db1 = direct ? db[1] : nullptr;
        a.M = M; a.N = N; a.ldd = Np; a.ldp = Np; a.act = act; a.dtype = dtype; a.pair = pair;
        TFLA_LAUNCH(K_ACT_BWD, launch_act_bwd(a, s));
    }
    if (want_db && (M == 0 || act_bwd_row_blocks(M, N) > 1))
        TFLA_LAUNCH(K_ACT_BWD, launch_sum_rows(reinterpret_cast<float*>(ws + l.dbpart), M > 0 ? act_bwd_row_blocks(M, N) : 0,
                                               (pair ? 2 : 1) * Np, Np, N, db[0], db[1], s));
    GemmArgs gx{}, gw{};
    RepackArgs rp{};
    rp.cols = K; rp.ldd = Kp;
    if (dx && M > 0) {
        gx.A[0] = dz[0]; gx.A[1] = dz[1]; gx.lda = ldz;
        gx.B[0] = w[0]; gx.B[1] = w[1]; gx.ldb = K;
        if (l.move_w) {
            rp.add(w[0], ws + l.w0, N);
            if (pair) rp.add(w[1], ws + l.w1, N);
            gx.B[0] = ws + l.w0; gx.B[1] = pair ? ws + l.w1 : nullptr; gx.ldb = Kp;
        }
        gx.M = M; gx.N = K; gx.K = N; gx.segs = pair ? 2 : 1; gx.batch = 1; gx.out[0] = dx; gx.dtype = dtype;
        gx.split = l.plan_dx.split; gx.part = reinterpret_cast<float*>(ws + l.part); gx.ld_part = (K + 7) & ~7;
    }
    if (want_dw) {
        gw.A[0] = dz[0]; gw.A[1] = dz[1]; gw.lda = ldz; gw.B[0] = x; gw.ldb = K;
        if (l.move_x && M > 0) {
            rp.add(x, ws + l.x, M);
            gw.B[0] = ws + l.x; gw.ldb = Kp;
        }
        gw.M = N; gw.N = K; gw.K = M; gw.segs = 1; gw.batch = pair ? 2 : 1; gw.out[0] = dw[0]; gw.out[1] = dw[1]; gw.dtype = dtype;
        gw.split = l.plan_dw.split; gw.part = reinterpret_cast<float*>(ws + l.part); gw.ld_part = (K + 7) & ~7;
    }
    if (rp.count > 0) TFLA_LAUNCH(K_ACT_BWD, launch_repack(rp, s));
    if (gx.M > 0 && gw.M > 0 && gemm_both_applies(l.plan_dx, l.plan_dw, M, K, N, pair, dtype)) {
        gx.split = gw.split = 1;
        TFLA_LAUNCH(K_GEMM, launch_gemm_both(gx, gw, l.plan_dx, s));
    } else {
        if (gx.M > 0) TFLA_LAUNCH(K_GEMM, launch_gemm(gx, l.plan_dx, false, true, EPI_STORE, s));
        if (gw.M > 0) TFLA_LAUNCH(K_GEMM, launch_gemm(gw, l.plan_dw, true, true, EPI_STORE, s));
    }
    return TFLA_OK;
}

}  // namespace

extern "C" {

size_t tfla_norm_workspace_bytes(int direction, int M, int D, int dtype, int norm_kind) {
    if ((direction != TFLA_FWD && direction != TFLA_BWD) || check_norm(M, D, dtype, norm_kind) != TFLA_OK) return 0;
    if (direction == TFLA_FWD || M == 0 || rownorm_bwd_blocks(M, D) == 1) return 0;
    return align_up((size_t)rownorm_bwd_blocks(M, D) * 2 * D * sizeof(float));
}

int tfla_norm_fwd(const void* x, const float* gamma, const float* beta, int M, int D, int dtype, int norm_kind, float norm_eps, void* y,
                  float* rstd, float* mean, void* stream) {
    const int rc = check_norm(M, D, dtype, norm_kind);
    if (rc != TFLA_OK) return rc;
    if (!(norm_eps >= 0.0f)) return TFLA_ERR_SHAPE;
    if (M == 0) return TFLA_OK;
    if (!x || !y) return TFLA_ERR_NULL;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    RowNormArgs a{x, gamma, beta, y, rstd, mean, M, D, norm_kind, dtype, norm_eps};
    TFLA_LAUNCH(K_ROWNORM_FWD, launch_rownorm_fwd(a, s));
    return TFLA_OK;
}

int tfla_norm_bwd(const void* x, const void* dy, const float* rstd, const float* mean, const float* gamma, const void* d_residual, int M,
                  int D, int dtype, int norm_kind, void* dx, float* dgamma, float* dbeta, void* workspace, size_t workspace_bytes,
                  void* stream) {
    int rc = check_norm(M, D, dtype, norm_kind);
    if (rc != TFLA_OK) return rc;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    const bool params = dgamma || dbeta;
    if (M == 0) {
        if (params) TFLA_LAUNCH(K_ROWNORM_BWD, launch_sum_rows(nullptr, 0, 0, 0, D, dgamma, dbeta, s));
        return TFLA_OK;
    }
    if (!x || !dy || !rstd || !dx || (norm_kind == TFLA_NORM_LAYER && !mean)) return TFLA_ERR_NULL;
    if (params) {
        rc = check_workspace(workspace, workspace_bytes, tfla_norm_workspace_bytes(TFLA_BWD, M, D, dtype, norm_kind));
        if (rc != TFLA_OK) return rc;
    }
    const int blocks = rownorm_bwd_blocks(M, D);
    float* part = reinterpret_cast<float*>(workspace);
    const bool join = params && blocks > 1;
    RowNormBwdArgs a{x, dy, rstd, mean, gamma, d_residual, dx, join ? part : nullptr, blocks > 1 ? nullptr : dgamma, blocks > 1 ? nullptr : dbeta,
                     M, D, norm_kind, dtype, blocks};
    TFLA_LAUNCH(K_ROWNORM_BWD, launch_rownorm_bwd(a, s));
    if (join) TFLA_LAUNCH(K_ROWNORM_BWD, launch_sum_rows(part, blocks, 2L * D, D, D, dgamma, dbeta, s));
    return TFLA_OK;
}

size_t tfla_linear_workspace_bytes(int direction, int M, int K, int N, int act, int dtype, int unaligned) {
    if (check_product(M, K, N, act, dtype) != TFLA_OK) return 0;
    const bool off = unaligned != 0;
    if (direction == TFLA_FWD) return fwd_bytes(M, K, N, dtype, false, off);
    if (direction == TFLA_BWD) return bwd_layout(M, K, N, act, dtype, false, off, off, off).bytes;
    return 0;
}

int tfla_linear_fwd(const void* x, const void* w, const float* bias, const void* residual, int M, int K, int N, int act, int dtype, void* y,
                    void* z, void* workspace, size_t workspace_bytes, void* stream) {
    const int rc = check_product(M, K, N, act, dtype);
    if (rc != TFLA_OK) return rc;
    if (M == 0) return TFLA_OK;
    if (!x || !w || !y) return TFLA_ERR_NULL;
    return product_fwd(x, {w, nullptr}, {bias, nullptr}, residual, M, K, N, act, dtype, y, {z, nullptr}, false, workspace, workspace_bytes,
                       reinterpret_cast<hipStream_t>(stream));
}

int tfla_linear_bwd(const void* x, const void* w, const void* dy, const void* z, int M, int K, int N, int act, int dtype, void* dx, void* dw,
                    float* db, void* workspace, size_t workspace_bytes, void* stream) {
    const int rc = check_product(M, K, N, act, dtype);
    if (rc != TFLA_OK) return rc;
    if (M > 0 && (!dy || (dw && !x) || (dx && !w) || (act != TFLA_ACT_NONE && !z))) return TFLA_ERR_NULL;
    return product_bwd(x, {w, nullptr}, dy, z, nullptr, M, K, N, act, dtype, dx, {dw, nullptr}, {db, nullptr}, false, workspace,
                       workspace_bytes, reinterpret_cast<hipStream_t>(stream));
}

size_t tfla_gated_workspace_bytes(int direction, int M, int K, int N, int act, int dtype, int unaligned) {
    if (check_product(M, K, N, act, dtype) != TFLA_OK) return 0;
    const bool off = unaligned != 0;
    if (direction == TFLA_FWD) return fwd_bytes(M, K, N, dtype, true, off);
    if (direction == TFLA_BWD) return bwd_layout(M, K, N, act, dtype, true, off, off, off).bytes;
    return 0;
}

int tfla_gated_fwd(const void* x, const void* w_gate, const void* w_up, const float* b_gate, const float* b_up, int M, int K, int N, int act,
                   int dtype, void* h, void* a, void* u, void* workspace, size_t workspace_bytes, void* stream) {
    const int rc = check_product(M, K, N, act, dtype);
    if (rc != TFLA_OK) return rc;
    if (M == 0) return TFLA_OK;
    if (!x || !w_gate || !w_up || !h) return TFLA_ERR_NULL;
    return product_fwd(x, {w_gate, w_up}, {b_gate, b_up}, nullptr, M, K, N, act, dtype, h, {a, u}, true, workspace, workspace_bytes,
                       reinterpret_cast<hipStream_t>(stream));
}

int tfla_gated_bwd(const void* x, const void* w_gate, const void* w_up, const void* a, const void* u, const void* dh, int M, int K, int N,
                   int act, int dtype, void* dx, void* dw_gate, void* dw_up, float* db_gate, float* db_up, void* workspace,
                   size_t workspace_bytes, void* stream) {
    const int rc = check_product(M, K, N, act, dtype);
    if (rc != TFLA_OK) return rc;
    if ((dw_gate != nullptr) != (dw_up != nullptr)) return TFLA_ERR_NULL;
    if (M > 0 && (!dh || !a || !u || (dw_gate && !x) || (dx && (!w_gate || !w_up)))) return TFLA_ERR_NULL;
    return product_bwd(x, {w_gate, w_up}, dh, a, u, M, K, N, act, dtype, dx, {dw_gate, dw_up}, {db_gate, db_up}, true, workspace,
                       workspace_bytes, reinterpret_cast<hipStream_t>(stream));
}

}  // extern "C"
