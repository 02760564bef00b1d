// C ABI of the residual block in 8 bits: argument checks, workspace layout and kernel sequence.  See include/tfla_mlstm.h for the contract.
#include "host_util.h"
#include "profiler.h"
#include "q8_internal.h"

using namespace tfla;

namespace {

constexpr int MAX_ROWS = 1 << 24, MAX_ROWS_BWD = 1 << 21, MAX_COLS = 1 << 20, MAX_NORM_COLS = 16384;
constexpr long MAX_ELEMS = 1L << 36;

inline long up16(long n) { return (n + 15) & ~15L; }
inline long blocks(long n) { return (n + 127) / 128; }
// the kernels bring rows of codes into LDS by 16-byte requests
inline bool moved(int cols, bool off) { return cols % 16 != 0 || off; }
inline const uint8_t* u8(const void* p) { return reinterpret_cast<const uint8_t*>(p); }
inline uint8_t* u8(void* p) { return reinterpret_cast<uint8_t*>(p); }

// M tokens: the transposed operands of a backward call have rows of M codes, whose offsets within a tile are 32-bit
int check_product(int direction, int M, int K, int N, int act) {
    if (direction != TFLA_FWD && direction != TFLA_BWD) return TFLA_ERR_ENUM;
    if (act < TFLA_ACT_NONE || act > TFLA_ACT_RELU) return TFLA_ERR_ENUM;
    if (M < 0 || M > (direction == TFLA_BWD ? MAX_ROWS_BWD : MAX_ROWS) || K <= 0 || K > MAX_COLS || N <= 0 || N > MAX_COLS) return TFLA_ERR_SHAPE;
    if ((long)M * K > MAX_ELEMS || (long)M * N > MAX_ELEMS || (long)N * K > MAX_ELEMS) return TFLA_ERR_SHAPE;
    return TFLA_OK;
}

struct FwdLayout {
    size_t x, w0, w1, part, bytes;
    GemmPlan plan; bool rows, join, move_x, move_w;     // join: a pair's gate is a launch of its own
};
FwdLayout fwd_layout(int M, int K, int N, bool pair, bool x_off, bool w_off) {
    FwdLayout l{};
    l.move_x = moved(K, x_off);
    l.move_w = moved(K, w_off);
    l.rows = q8_rows_applies(M, N, K, pair, l.move_x || l.move_w);
    Carver c(nullptr);
    if (l.rows) {       // that kernel reads the codes where they are
        l.move_x = l.move_w = false;
        l.plan.split = 1;
    } else {
        l.plan = q8_plan(M, N, K, 1, 1, pair);
        if (l.move_x) { l.x = c.off; c.take(M * up16(K)); }
        if (l.move_w) {
            l.w0 = c.off; c.take(N * up16(K));
            if (pair) { l.w1 = c.off; c.take(N * up16(K)); }
        }
    }
    l.join = pair && (l.rows || !q8_gate_inside(l.plan.bn, l.plan.split));
    l.part = c.off;
    if (l.plan.split > 1 || l.join) c.take((size_t)l.plan.split * (pair ? 2 : 1) * M * (((size_t)N + 7) & ~(size_t)7) * sizeof(float));
    l.bytes = c.off;
    return l;
}
// what a query answers: with tensors off 16 bytes, which of them is not known
size_t fwd_bytes(int M, int K, int N, bool pair, bool off) {
    if (M == 0) return 0;
    const size_t in = fwd_layout(M, K, N, pair, false, false).bytes, out = off ? fwd_layout(M, K, N, pair, true, true).bytes : 0;
    return in > out ? in : out;
}

// A gradient of pre-activations in 8 bits (dz, s), its transpose (dzt, st); x transposed (xt, sx); moved weights; sums; parts
struct BwdLayout {
    size_t dz[2], s[2], dzt[2], st[2], xt, sx, w[2], dbpart, part, bytes;
    GemmPlan plan_dx, plan_dw; bool move_w;
};
BwdLayout bwd_layout(int M, int K, int N, bool pair, bool w_off) {
    BwdLayout l{};
    l.plan_dx = q8_plan(M, K, N, pair ? 2 : 1, 1, 0);
    l.plan_dw = q8_plan(N, K, M, 1, pair ? 2 : 1, 0);
    l.move_w = moved(N, w_off);
    Carver c(nullptr);
    for (int p = 0; p < (pair ? 2 : 1); ++p) {
        l.dz[p] = c.off; c.take(M * up16(N));
        l.s[p] = c.off; c.take(blocks(N) * M);
        l.dzt[p] = c.off; c.take(N * up16(M));
        l.st[p] = c.off; c.take(blocks(M) * N);
        if (l.move_w) { l.w[p] = c.off; c.take(K * up16(N)); }
    }
    l.xt = c.off; c.take(K * up16(M));
    l.sx = c.off; c.take(blocks(M) * K);
    l.dbpart = c.off; c.take((size_t)blocks(M) * (pair ? 2 : 1) * N * sizeof(float));
    // (the two products run one after the other and share the memory of their partial results)
    const size_t K8 = ((size_t)K + 7) & ~(size_t)7;
    const size_t pdx = l.plan_dx.split > 1 ? (size_t)l.plan_dx.split * M * K8 * sizeof(float) : 0;
    const size_t pdw = l.plan_dw.split > 1 ? (size_t)l.plan_dw.split * (pair ? 2 : 1) * N * K8 * sizeof(float) : 0;
    l.part = c.off; c.take(pdx > pdw ? pdx : pdw);
    l.bytes = c.off;
    return l;
}

// operands in pairs of codes, as the kernels address them
void operands(Q8GemmArgs& q, long pitch_a, long pitch_b, int M, int N, int K) {
    q.g.lda = pitch_a / 2; q.g.ldb = pitch_b / 2;
    q.g.M = M; q.g.N = N; q.g.K = (K + 1) / 2; q.k = K;
    q.g.segs = 1; q.g.batch = 1; q.g.dtype = TFLA_BF16; q.g.ld_part = (N + 7) & ~7;
}

int product_fwd(const void* xq, const void* x_scale, const void* const (&wq)[2], const void* const (&w_scale)[2], const float* const (&bias)[2],
                const void* residual, int M, int K, int N, int act, void* y, void* y_scale, void* h, void* const (&z)[2], bool pair, void* workspace,
                size_t workspace_bytes, hipStream_t s) {
    const FwdLayout l = fwd_layout(M, K, N, pair, off16(xq), off16(wq[0]) || (pair && off16(wq[1])));
    const int rc = check_workspace(workspace, workspace_bytes, l.bytes);
    if (rc != TFLA_OK) return rc;
    uint8_t* ws = u8(workspace);
    const long pitch = up16(K);
    Q8GemmArgs q{};
    GemmArgs& g = q.g;
    operands(q, K, K, M, N, K);
    g.A[0] = xq; g.B[0] = wq[0]; g.B[1] = wq[1]; g.pair = pair;
    q.sa[0] = q.sa[1] = u8(x_scale); q.sb[0] = u8(w_scale[0]); q.sb[1] = u8(w_scale[1]);
    q.lsa = M; q.lsb = blocks(N); q.shb = 7;
    for (int p = 0; p < 2; ++p) { g.bias[p] = bias[p]; g.z[p] = z[p]; }
    g.residual = residual; g.act = act; g.split = l.plan.split;
    g.part = reinterpret_cast<float*>(ws + l.part);
    if (pair) { q.h.q = u8(y); q.h.s = u8(y_scale); q.hc = h; }
    else g.out[0] = y;
    if (l.rows) {
        TFLA_LAUNCH(K_GEMM, launch_q8_rows(q, s));
    } else {
        Q8RepackArgs rp{};
        rp.cols = K; rp.ldd = pitch;
        if (l.move_x) {
            rp.add(u8(xq), ws + l.x, M);
            g.A[0] = ws + l.x; g.lda = pitch / 2;
        }
        if (l.move_w) {
            rp.add(u8(wq[0]), ws + l.w0, N);
            if (pair) rp.add(u8(wq[1]), ws + l.w1, N);
            g.B[0] = ws + l.w0; g.B[1] = pair ? ws + l.w1 : nullptr; g.ldb = pitch / 2;
        }
        if (rp.count > 0) TFLA_LAUNCH(K_ACT_BWD, launch_q8_repack(rp, s));
        TFLA_LAUNCH(K_GEMM, launch_q8_gemm(q, l.plan, l.join ? EPI_PART : (pair ? EPI_GATED : EPI_LINEAR), s));
    }
    if (l.join) TFLA_LAUNCH(K_ACT_BWD, launch_q8_gated_join(q, s));
    return TFLA_OK;
}

int product_bwd(const void* x, const void* const (&wqt)[2], const void* const (&wt_scale)[2], const void* dy, const void* z, const void* u, int M,
                int K, int N, int act, void* dx, void* const (&dw)[2], float* const (&db)[2], bool pair, void* workspace, size_t workspace_bytes,
                hipStream_t s) {
    const int P = pair ? 2 : 1;
    const BwdLayout l = bwd_layout(M, K, N, pair, off16(wqt[0]) || (pair && off16(wqt[1])));
    const int rc = check_workspace(workspace, workspace_bytes, l.bytes);
    if (rc != TFLA_OK) return rc;
    uint8_t* ws = u8(workspace);
    const bool want_dw = dw[0] || dw[1], want_db = db[0] || db[1];
    const long Np = up16(N), Mp = up16(M);
    const bool one = blocks(M) == 1;         // (block of rows: its sums are the results)
    Q8Sums sums{reinterpret_cast<float*>(ws + l.dbpart), (int)blocks(M), want_db && !one ? P : 0, N, {db[0], db[1]}};
    if (M > 0 && (dx || want_dw || want_db)) {
        Q8TileArgs a{}, b{};
        a.x = dy; a.z = z; a.u = u; a.M = M; a.N = N; a.act = act; a.dtype = TFLA_BF16; a.rows = 1;
        a.mode = pair ? Q8_PAIR : (act != TFLA_ACT_NONE ? Q8_ACT : Q8_VALUES);
        for (int p = 0; p < P; ++p) {
            Q8Out& o = a.out[p];
            if (dx) { o.q = ws + l.dz[p]; o.s = ws + l.s[p]; o.ldq = Np; o.lds = M; o.wq = (int)Np; }
            if (want_dw) { o.qt = ws + l.dzt[p]; o.st = ws + l.st[p]; o.ldt = Mp; o.ldst = N; o.wt = (int)Mp; }
        }
        if (sums.planes) { a.part = reinterpret_cast<float*>(ws + l.dbpart); a.ldp = N; }
        if (one) { a.db[0] = db[0]; a.db[1] = db[1]; }
        if (want_dw) {      // x along the tokens
            b.x = x; b.M = M; b.N = K; b.dtype = TFLA_BF16; b.rows = 1; b.mode = Q8_VALUES;
            Q8Out& o = b.out[0];
            o.qt = ws + l.xt; o.st = ws + l.sx; o.ldt = Mp; o.ldst = K; o.wt = (int)Mp;
        }
        Q8RepackArgs rp{};
        rp.cols = N; rp.ldd = Np;
        for (int p = 0; p < P && dx && l.move_w; ++p) rp.add(u8(wqt[p]), ws + l.w[p], K);
        TFLA_LAUNCH(K_ACT_BWD, launch_q8_tiles(a, b, rp, s));
    }
    Q8GemmArgs qx{}, qw{};
    if (dx && M > 0) {
        operands(qx, Np, N, M, K, N);
        qx.lsa = M; qx.lsb = blocks(K); qx.shb = 7;
        for (int p = 0; p < P; ++p) {
            qx.g.A[p] = ws + l.dz[p]; qx.sa[p] = ws + l.s[p];
            qx.g.B[p] = l.move_w ? ws + l.w[p] : u8(wqt[p]); qx.sb[p] = u8(wt_scale[p]);
        }
        if (l.move_w) qx.g.ldb = Np / 2;
        qx.g.segs = P; qx.g.out[0] = dx; qx.g.split = l.plan_dx.split; qx.g.part = reinterpret_cast<float*>(ws + l.part);
    }
    if (want_dw) {
        operands(qw, Mp, Mp, N, K, M);
        qw.lsa = N; qw.lsb = K; qw.shb = 0;
        for (int p = 0; p < P; ++p) { qw.g.A[p] = ws + l.dzt[p]; qw.sa[p] = ws + l.st[p]; qw.g.out[p] = dw[p]; }
        qw.g.B[0] = ws + l.xt; qw.sb[0] = qw.sb[1] = ws + l.sx;
        qw.g.batch = P; qw.g.split = l.plan_dw.split; qw.g.part = reinterpret_cast<float*>(ws + l.part);
    }
    if (qx.g.M > 0 && qw.g.M > 0 && q8_both_applies(l.plan_dx, l.plan_dw, M, K, N, pair)) {
        qx.g.split = qw.g.split = 1;
        TFLA_LAUNCH(K_GEMM, launch_q8_both(qx, qw, sums, s));
        return TFLA_OK;
    }
    if (want_db && !one) TFLA_LAUNCH(K_ACT_BWD, launch_sum_rows(sums.part, sums.rows, (long)P * N, N, N, db[0], db[1], s));
    if (qx.g.M > 0) TFLA_LAUNCH(K_GEMM, launch_q8_gemm(qx, l.plan_dx, EPI_STORE, s));
    if (qw.g.M > 0) TFLA_LAUNCH(K_GEMM, launch_q8_gemm(qw, l.plan_dw, EPI_STORE, s));
    return TFLA_OK;
}

}  // namespace

namespace tfla {

template <int V> hipError_t launch_q8_gemm_as(const Q8GemmArgs& a, const GemmPlan& p, hipStream_t s);

hipError_t launch_q8_gemm(const Q8GemmArgs& a, const GemmPlan& p, int epi, hipStream_t s) {
    if (a.g.pair) return epi == EPI_GATED ? launch_q8_gemm_as<4>(a, p, s) : launch_q8_gemm_as<3>(a, p, s);
    if (a.g.split == 1) return epi == EPI_LINEAR ? launch_q8_gemm_as<0>(a, p, s) : launch_q8_gemm_as<1>(a, p, s);
    const hipError_t rc = launch_q8_gemm_as<2>(a, p, s);
    return rc != hipSuccess ? rc : launch_gemm_reduce(a.g, epi, s);
}

}  // namespace tfla

extern "C" {

int tfla_q8_quant(const void* x, int M, int K, int dtype, int rows, void* q, void* scale, void* qt, void* scale_t, void* stream) {
    if (dtype != TFLA_F32 && dtype != TFLA_BF16) return TFLA_ERR_ENUM;
    if (rows != 1 && rows != 128) return TFLA_ERR_ENUM;
    if (M < 0 || M > MAX_ROWS || K <= 0 || K > MAX_COLS || (long)M * K > MAX_ELEMS) return TFLA_ERR_SHAPE;
    if ((q != nullptr) != (scale != nullptr) || (qt != nullptr) != (scale_t != nullptr)) return TFLA_ERR_NULL;
    if (M == 0 || (!q && !qt)) return TFLA_OK;
    if (!x) return TFLA_ERR_NULL;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    Q8TileArgs a{};
    a.x = x; a.M = M; a.N = K; a.dtype = dtype; a.rows = rows; a.mode = Q8_VALUES;
    a.out[0] = {u8(q), u8(scale), u8(qt), u8(scale_t), K, rows == 1 ? M : blocks(M), M, rows == 1 ? K : blocks(K), K, M};
    TFLA_LAUNCH(K_ACT_BWD, launch_q8_tiles(a, {}, {}, s));
    return TFLA_OK;
}

int tfla_norm_q8_fwd(const void* x, const float* gamma, const float* beta, const void* residual, int M, int D, int dtype, int norm_kind,
                     float norm_eps, void* q, void* scale, void* sum, void* y, float* rstd, float* mean, void* stream) {
    if (dtype != TFLA_F32 && dtype != TFLA_BF16) return TFLA_ERR_ENUM;
    if (norm_kind != TFLA_NORM_RMS && norm_kind != TFLA_NORM_LAYER) return TFLA_ERR_ENUM;
    if (M < 0 || M > MAX_ROWS || D <= 0 || D > MAX_NORM_COLS || !(norm_eps >= 0.0f)) return TFLA_ERR_SHAPE;
    if (M == 0) return TFLA_OK;
    if (!x || !q || !scale) return TFLA_ERR_NULL;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    Q8NormArgs a{};
    static_cast<RowNormArgs&>(a) = {x, gamma, beta, y, rstd, mean, M, D, norm_kind, dtype, norm_eps};
    a.residual = residual; a.sum = sum; a.q = u8(q); a.s = u8(scale);
    TFLA_LAUNCH(K_ROWNORM_FWD, launch_rownorm_q8(a, s));
    return TFLA_OK;
}

size_t tfla_linear_q8_workspace_bytes(int direction, int M, int K, int N, int act, int unaligned) {
    if (check_product(direction, M, K, N, act) != TFLA_OK) return 0;
    return direction == TFLA_FWD ? fwd_bytes(M, K, N, false, unaligned != 0) : bwd_layout(M, K, N, false, unaligned != 0).bytes;
}

int tfla_linear_q8_fwd(const void* xq, const void* x_scale, const void* wq, const void* w_scale, const float* bias, const void* residual, int M,
                       int K, int N, int act, void* y, void* z, void* workspace, size_t workspace_bytes, void* stream) {
    const int rc = check_product(TFLA_FWD, M, K, N, act);
    if (rc != TFLA_OK) return rc;
    if (M == 0) return TFLA_OK;
    if (!xq || !x_scale || !wq || !w_scale || !y) return TFLA_ERR_NULL;
    return product_fwd(xq, x_scale, {wq, nullptr}, {w_scale, nullptr}, {bias, nullptr}, residual, M, K, N, act, y, nullptr, nullptr, {z, nullptr},
                       false, workspace, workspace_bytes, reinterpret_cast<hipStream_t>(stream));
}

int tfla_linear_q8_bwd(const void* x, const void* wqt, const void* wt_scale, const void* dy, const void* z, int M, int K, int N, int act, void* dx,
                       void* dw, float* db, void* workspace, size_t workspace_bytes, void* stream) {
    const int rc = check_product(TFLA_BWD, M, K, N, act);
    if (rc != TFLA_OK) return rc;
    if (M > 0 && (!dy || (dw && !x) || (dx && (!wqt || !wt_scale)) || (act != TFLA_ACT_NONE && !z))) return TFLA_ERR_NULL;
    return product_bwd(x, {wqt, nullptr}, {wt_scale, nullptr}, dy, z, nullptr, M, K, N, act, dx, {dw, nullptr}, {db, nullptr}, false, workspace,
                       workspace_bytes, reinterpret_cast<hipStream_t>(stream));
}

size_t tfla_gated_q8_workspace_bytes(int direction, int M, int K, int N, int act, int unaligned) {
    if (check_product(direction, M, K, N, act) != TFLA_OK) return 0;
    return direction == TFLA_FWD ? fwd_bytes(M, K, N, true, unaligned != 0) : bwd_layout(M, K, N, true, unaligned != 0).bytes;
}

int tfla_gated_q8_fwd(const void* xq, const void* x_scale, const void* wq_gate, const void* w_scale_gate, const void* wq_up, const void* w_scale_up,
                      const float* b_gate, const float* b_up, int M, int K, int N, int act, void* hq, void* h_scale, void* h, void* a, void* u,
                      void* workspace, size_t workspace_bytes, void* stream) {
    const int rc = check_product(TFLA_FWD, M, K, N, act);
    if (rc != TFLA_OK) return rc;
    if (M == 0) return TFLA_OK;
    if (!xq || !x_scale || !wq_gate || !w_scale_gate || !wq_up || !w_scale_up || !hq || !h_scale) return TFLA_ERR_NULL;
    return product_fwd(xq, x_scale, {wq_gate, wq_up}, {w_scale_gate, w_scale_up}, {b_gate, b_up}, nullptr, M, K, N, act, hq, h_scale, h, {a, u},
                       true, workspace, workspace_bytes, reinterpret_cast<hipStream_t>(stream));
}

int tfla_gated_q8_bwd(const void* x, const void* wqt_gate, const void* wt_scale_gate, const void* wqt_up, const void* wt_scale_up, const void* a,
                      const void* u, const void* dh, int M, int K, int N, int act, void* dx, void* dw_gate, void* dw_up, float* db_gate,
                      float* db_up, void* workspace, size_t workspace_bytes, void* stream) {
    const int rc = check_product(TFLA_BWD, M, K, N, act);
    if (rc != TFLA_OK) return rc;
    if ((dw_gate != nullptr) != (dw_up != nullptr)) return TFLA_ERR_NULL;
    if (M > 0 && (!dh || !a || !u || (dw_gate && !x) || (dx && (!wqt_gate || !wt_scale_gate || !wqt_up || !wt_scale_up)))) return TFLA_ERR_NULL;
    return product_bwd(x, {wqt_gate, wqt_up}, {wt_scale_gate, wt_scale_up}, dh, a, u, M, K, N, act, dx, {dw_gate, dw_up}, {db_gate, db_up}, true,
                       workspace, workspace_bytes, reinterpret_cast<hipStream_t>(stream));
}

}  // extern "C"
