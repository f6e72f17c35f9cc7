// C ABI of the feed-forward sublayer (include/ffn.h): argument checks,
// workspaces, and the order of the launches.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstddef>
#include <new>

#include "cgtp_internal.h"
#include "ffn_internal.h"

struct ffn_plan_s {
    int64_t d_in, d_ff, d_out;
    int32_t act, dtype, device;
};

namespace {

constexpr int64_t kMaxStride = 1LL << 22;

struct Range { const void* p; int64_t bytes; };

bool overlaps(const Range& a, const Range& b) {
    if (!a.p || !b.p || a.bytes <= 0 || b.bytes <= 0) return false;
    const char *pa = (const char*)a.p, *pb = (const char*)b.p;
    return pa < pb + b.bytes && pb < pa + a.bytes;
}

// Whether any of the outputs meets an input or a later output.
template <size_t A, size_t B> bool any_overlap(const Range (&outs)[A], const Range (&ins)[B]) {
    for (size_t i = 0; i < A; ++i) {
        for (size_t j = 0; j < B; ++j)
            if (overlaps(outs[i], ins[j])) return true;
        for (size_t j = i + 1; j < A; ++j)
            if (overlaps(outs[i], outs[j])) return true;
    }
    return false;
}

int64_t size_of(int32_t dtype) { return dtype == FFN_FP32 ? 4 : 2; }
bool known(int32_t dtype) { return dtype == FFN_FP32 || dtype == FFN_BF16 || dtype == FFN_FP16; }
int64_t aligned(int64_t bytes) { return (bytes + 255) & ~255LL; }
// bytes from the first to the last value of N rows
int64_t span(int64_t N, int64_t ld, int64_t width, int64_t e) { return N > 0 ? ((N - 1) * ld + width) * e : 0; }

bool misaligned(std::initializer_list<const void*> ps, int64_t e) {
    uintptr_t all = 0;
    for (const void* p : ps) all |= (uintptr_t)p;
    return (all & (uintptr_t)(e - 1)) != 0;
}

int workspace_ok(const void* ws, int64_t bytes, int64_t need) {
    if (bytes < need || (need > 0 && !ws) || ((uintptr_t)ws & 255)) return CGTP_EINVAL;
    return CGTP_OK;
}

int status(int err) {
    if (err == 0) return CGTP_OK;
    cgtp::set_last_hip_error(err);
    return CGTP_EHIP;
}

int current_device_is(int device) {
    int dev = -1;
    const hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return status((int)e);
    return dev == device ? CGTP_OK : CGTP_EINVAL;
}

// p in [0, 1]: threshold of the 16-bit draws and the scale that keeps the expected value
bool drop_args(double p, uint64_t seed, uint64_t offset, ffn::DropArgs* d) {
    if (!(p >= 0.0 && p <= 1.0)) return false;
    d->threshold = (uint32_t)std::floor(p * 65536.0 + 0.5);
    d->scale = d->threshold < 65536u ? (float)(65536.0 / (65536.0 - d->threshold)) : 0.0f;
    d->seed = seed;
    d->offset = offset;
    return true;
}

int check_norm(const ffn_norm* n, int64_t N, ffn::NormArgs* a) {
    if (!n || N < 0 || n->width < 1 || n->rows_per_gate < 1) return CGTP_EINVAL;
    if (!(n->eps > 0.0f) || std::isinf(n->eps)) return CGTP_EINVAL;
    if (!known(n->dtype)) return CGTP_EDTYPE;
    *a = ffn::NormArgs();
    if (!drop_args(n->dropout, n->seed, n->offset, &a->drop)) return CGTP_EINVAL;
    if (n->width > FFN_MAX_WIDTH || N > FFN_MAX_ROWS) return CGTP_EUNSUP;
    a->width = n->width;
    a->N = N;
    a->rows_per_gate = n->rows_per_gate;
    a->eps = n->eps;
    return CGTP_OK;
}

// Byte offsets of the block's intermediates in its workspace.
struct Layout { int64_t h, dgu, total; };
Layout layout(const ffn_plan_s* p, int64_t N, bool backward) {
    const int64_t e = size_of(p->dtype);
    Layout l = {};
    l.dgu = aligned(N * p->d_ff * e);
    l.total = l.dgu + (backward ? aligned(N * 2 * p->d_ff * e) : 0);
    return l;
}

}  // namespace

extern "C" {

int ffn_plan(int64_t d_in, int64_t d_ff, int64_t d_out, int32_t activation, int32_t dtype, ffn_plan_t* plan_out) {
    if (!plan_out || d_in < 1 || d_ff < 1 || d_out < 1) return CGTP_EINVAL;
    if (activation < FFN_SILU || activation > FFN_RELU) return CGTP_EINVAL;
    if (!known(dtype)) return CGTP_EDTYPE;
    if (d_in > FFN_MAX_WIDTH || d_ff > FFN_MAX_WIDTH || d_out > FFN_MAX_WIDTH) return CGTP_EUNSUP;
    int dev = -1;
    const hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return status((int)e);
    ffn_plan_s* p = new (std::nothrow) ffn_plan_s{d_in, d_ff, d_out, activation, dtype, dev};
    if (!p) return CGTP_ENOMEM;
    *plan_out = p;
    return CGTP_OK;
}

int ffn_destroy(ffn_plan_t plan) {
    delete plan;
    return CGTP_OK;
}

int64_t ffn_workspace_bytes(ffn_plan_t plan, int64_t N) {
    if (!plan || N < 0 || N > FFN_MAX_ROWS) return -1;
    return layout(plan, N, false).total;
}

int64_t ffn_backward_workspace_bytes(ffn_plan_t plan, int64_t N) {
    if (!plan || N < 0 || N > FFN_MAX_ROWS) return -1;
    return layout(plan, N, true).total;
}

int ffn_forward(ffn_plan_t plan, const void* x, int64_t ldx, const void* w_in, const void* w_out, void* y, void* saved,
                int64_t N, void* workspace, int64_t workspace_bytes, void* hip_stream) {
    if (!plan || N < 0) return CGTP_EINVAL;
    if (N == 0) return CGTP_OK;
    if (!x || !w_in || !w_out || !y || ldx < plan->d_in) return CGTP_EINVAL;
    if (N > FFN_MAX_ROWS || ldx > kMaxStride) return CGTP_EUNSUP;
    const int64_t e = size_of(plan->dtype), di = plan->d_in, df = plan->d_ff, d_o = plan->d_out;
    if (misaligned({x, w_in, w_out, y}, e) || misaligned({saved}, 4)) return CGTP_EINVAL;
    const Layout l = layout(plan, N, false);
    int rc = workspace_ok(workspace, workspace_bytes, l.total);
    if (rc != CGTP_OK) return rc;
    const Range ins[] = {{x, span(N, ldx, di, e)}, {w_in, 2 * df * di * e}, {w_out, d_o * df * e}};
    const Range outs[] = {{y, N * d_o * e}, {saved, N * 2 * df * 4}, {workspace, l.total}};
    if (any_overlap(outs, ins)) return CGTP_EINVAL;
    rc = current_device_is(plan->device);
    if (rc != CGTP_OK) return rc;
    char* ws = (char*)workspace;
    ffn::GemmArgs g = {};
    g.a = x; g.lda = ldx; g.b = w_in; g.ldb = di;
    g.M = N; g.N = df; g.K = di;
    g.c = ws + l.h; g.ldc = df;
    g.epilogue = ffn::kGate; g.act = plan->act; g.saved = saved;
    rc = status(ffn::launch_gemm(g, plan->dtype, hip_stream));
    if (rc != CGTP_OK) return rc;
    ffn::GemmArgs o = {};
    o.a = ws + l.h; o.lda = df; o.b = w_out; o.ldb = df;
    o.M = N; o.N = d_o; o.K = df;
    o.c = y; o.ldc = d_o;
    return status(ffn::launch_gemm(o, plan->dtype, hip_stream));
}

int ffn_backward(ffn_plan_t plan, const void* x, int64_t ldx, const void* w_in, const void* w_out, const void* saved,
                 const void* grad_y, int64_t ldg, void* grad_x, void* grad_w_in, void* grad_w_out, int64_t N,
                 void* workspace, int64_t workspace_bytes, void* hip_stream) {
    if (!plan || N < 0 || (!grad_x && !grad_w_in && !grad_w_out)) return CGTP_EINVAL;
    const int64_t e = size_of(plan->dtype), di = plan->d_in, df = plan->d_ff, d_o = plan->d_out;
    if (N > 0 && (!x || !w_in || !w_out || !saved || !grad_y || ldx < di || ldg < d_o)) return CGTP_EINVAL;
    if (N > FFN_MAX_ROWS || ldx > kMaxStride || ldg > kMaxStride) return CGTP_EUNSUP;
    if (misaligned({x, w_in, w_out, grad_y, grad_x, grad_w_in, grad_w_out}, e) || misaligned({saved}, 4)) return CGTP_EINVAL;
    const Layout l = layout(plan, N, true);
    int rc = workspace_ok(workspace, workspace_bytes, l.total);
    if (rc != CGTP_OK) return rc;
    const Range ins[] = {{x, span(N, ldx, di, e)}, {w_in, 2 * df * di * e}, {w_out, d_o * df * e},
                         {saved, N * 2 * df * 4}, {grad_y, span(N, ldg, d_o, e)}};
    const Range outs[] = {{grad_x, N * di * e}, {grad_w_in, 2 * df * di * e}, {grad_w_out, d_o * df * e},
                          {workspace, l.total}};
    if (any_overlap(outs, ins)) return CGTP_EINVAL;
    rc = current_device_is(plan->device);
    if (rc != CGTP_OK) return rc;
    char* ws = (char*)workspace;
    if (N > 0) {
        ffn::GemmArgs g = {};
        g.a = grad_y; g.lda = ldg; g.b = w_out; g.ldb = df; g.b_cols = 1;
        g.M = N; g.N = df; g.K = d_o;
        g.c = ws + l.dgu; g.ldc = 2 * df;
        g.epilogue = ffn::kGateGrad; g.act = plan->act; g.saved = const_cast<void*>(saved); g.h = ws + l.h;
        rc = status(ffn::launch_gemm(g, plan->dtype, hip_stream));
        if (rc != CGTP_OK) return rc;
    }
    if (grad_x && N > 0) {
        ffn::GemmArgs g = {};
        g.a = ws + l.dgu; g.lda = 2 * df; g.b = w_in; g.ldb = di; g.b_cols = 1;
        g.M = N; g.N = di; g.K = 2 * df;
        g.c = grad_x; g.ldc = di;
        rc = status(ffn::launch_gemm(g, plan->dtype, hip_stream));
        if (rc != CGTP_OK) return rc;
    }
    if (grad_w_in) {
        ffn::GemmArgs g = {};
        g.a = ws + l.dgu; g.lda = 2 * df; g.a_cols = 1; g.b = x; g.ldb = ldx; g.b_cols = 1;
        g.M = 2 * df; g.N = di; g.K = N;
        g.c = grad_w_in; g.ldc = di;
        rc = status(ffn::launch_gemm(g, plan->dtype, hip_stream));
        if (rc != CGTP_OK) return rc;
    }
    if (grad_w_out) {
        ffn::GemmArgs g = {};
        g.a = grad_y; g.lda = ldg; g.a_cols = 1; g.b = ws + l.h; g.ldb = df; g.b_cols = 1;
        g.M = d_o; g.N = df; g.K = N;
        g.c = grad_w_out; g.ldc = df;
        rc = status(ffn::launch_gemm(g, plan->dtype, hip_stream));
    }
    return rc;
}

int ffn_norm_forward(const ffn_norm* norm, const void* x, int64_t ldx, const void* w, void* u, int64_t ldu, float* rstd,
                     int64_t N, void* hip_stream) {
    ffn::NormArgs a;
    const int rc = check_norm(norm, N, &a);
    if (rc != CGTP_OK) return rc;
    if (N == 0) return CGTP_OK;
    if (!x || !u || ldx < a.width || ldu < a.width) return CGTP_EINVAL;
    if (ldx > kMaxStride || ldu > kMaxStride) return CGTP_EUNSUP;
    const int64_t e = size_of(norm->dtype);
    if (misaligned({x, w, u}, e) || misaligned({rstd}, 4)) return CGTP_EINVAL;
    const Range in_x[] = {{u == x && ldu == ldx ? nullptr : x, span(N, ldx, a.width, e)}, {w, a.width * e}};
    const Range outs[] = {{u, span(N, ldu, a.width, e)}, {rstd, N * 4}};
    const Range also[] = {{x, span(N, ldx, a.width, e)}};
    const Range stat[] = {{rstd, N * 4}};
    if (any_overlap(outs, in_x) || any_overlap(stat, also)) return CGTP_EINVAL;
    a.x = x; a.ldx = ldx;
    a.u = u; a.ldu = ldu; a.wn = w; a.rstd_y = rstd;
    return status(ffn::launch_norm_forward(a, norm->dtype, hip_stream));
}

int64_t ffn_norm_workspace_bytes(const ffn_norm* norm, int64_t N, int32_t residual) {
    ffn::NormArgs a;
    if ((residual & ~1) || check_norm(norm, N, &a) != CGTP_OK) return -1;
    return aligned(ffn::norm_workspace_floats(a.width, N, a.rows_per_gate, residual != 0) * 4);
}

int ffn_norm_backward(const ffn_norm* norm, const void* x, int64_t ldx, const void* w, const float* rstd,
                      const void* grad_u, int64_t ldg, void* grad_x, void* grad_w, int64_t N, void* workspace,
                      int64_t workspace_bytes, void* hip_stream) {
    ffn::NormArgs a;
    int rc = check_norm(norm, N, &a);
    if (rc != CGTP_OK) return rc;
    if (!grad_x && !grad_w) return CGTP_EINVAL;
    if (N > 0 && (!x || !rstd || !grad_u || ldx < a.width || ldg < a.width)) return CGTP_EINVAL;
    if (ldx > kMaxStride || ldg > kMaxStride) return CGTP_EUNSUP;
    const int64_t e = size_of(norm->dtype);
    if (misaligned({x, w, grad_u, grad_x, grad_w}, e) || misaligned({rstd}, 4)) return CGTP_EINVAL;
    const int64_t need = ffn_norm_workspace_bytes(norm, N, 0);
    rc = workspace_ok(workspace, workspace_bytes, need);
    if (rc != CGTP_OK) return rc;
    const Range ins[] = {{x, span(N, ldx, a.width, e)}, {w, a.width * e}, {rstd, N * 4}, {grad_u, span(N, ldg, a.width, e)}};
    const Range outs[] = {{grad_x, N * a.width * e}, {grad_w, a.width * e}, {workspace, need}};
    if (any_overlap(outs, ins)) return CGTP_EINVAL;
    a.y = const_cast<void*>(x); a.ldx = ldx; a.wn = w; a.rstd_y = const_cast<float*>(rstd);
    a.gu = grad_u; a.ldg = ldg; a.gx = grad_x; a.gwn = grad_w;
    a.partial = (float*)workspace;
    return status(ffn::launch_norm_backward(a, norm->dtype, hip_stream));
}

int ffn_residual_forward(const ffn_norm* norm, const void* x, const void* h, const void* w, const void* gate,
                         const void* scale, const void* w_next, void* y, void* u, float* stats, int64_t N,
                         void* hip_stream) {
    ffn::NormArgs a;
    const int rc = check_norm(norm, N, &a);
    if (rc != CGTP_OK) return rc;
    if (N == 0) return CGTP_OK;
    if (!x || !h || !y) return CGTP_EINVAL;
    if (!u) w_next = nullptr;
    const int64_t e = size_of(norm->dtype), D = a.width, all = N * D * e;
    if (misaligned({x, h, w, gate, scale, w_next, y, u}, e) || misaligned({stats}, 4)) return CGTP_EINVAL;
    const int64_t gates = (N + a.rows_per_gate - 1) / a.rows_per_gate;
    const Range ins[] = {{y == x ? nullptr : x, all}, {h, all}, {w, D * e}, {gate, gates * D * e}, {scale, D * e}, {w_next, D * e}};
    const Range outs[] = {{y, all}, {u, all}, {stats, 2 * N * 4}};
    if (any_overlap(outs, ins)) return CGTP_EINVAL;
    a.x = x; a.ldx = D; a.h = h; a.w = w; a.gate = gate; a.scale = scale; a.wn = w_next;
    a.y = y; a.u = u; a.ldu = D;
    a.rstd_h = stats;
    a.rstd_y = stats ? stats + N : nullptr;
    return status(ffn::launch_norm_forward(a, norm->dtype, hip_stream));
}

int ffn_residual_backward(const ffn_norm* norm, const void* h, const void* y, const void* w, const void* gate,
                          const void* scale, const void* w_next, const float* stats, const void* grad_y,
                          const void* grad_u, void* grad_x, void* grad_h, void* grad_w, void* grad_gate,
                          void* grad_scale, void* grad_w_next, int64_t N, void* workspace, int64_t workspace_bytes,
                          void* hip_stream) {
    ffn::NormArgs a;
    int rc = check_norm(norm, N, &a);
    if (rc != CGTP_OK) return rc;
    if (N > 0 && (!h || !stats || (!grad_y && !grad_u) || (grad_u && !y) || !grad_x || !grad_h || (grad_gate && !gate)))
        return CGTP_EINVAL;
    if (!grad_u) { w_next = nullptr; y = nullptr; }
    const int64_t e = size_of(norm->dtype), D = a.width, all = N * D * e;
    if (misaligned({h, y, w, gate, scale, w_next, grad_y, grad_u, grad_x, grad_h, grad_w, grad_gate, grad_scale, grad_w_next}, e) ||
        misaligned({stats}, 4))
        return CGTP_EINVAL;
    const int64_t need = ffn_norm_workspace_bytes(norm, N, 1);
    rc = workspace_ok(workspace, workspace_bytes, need);
    if (rc != CGTP_OK) return rc;
    const int64_t gates = (N + a.rows_per_gate - 1) / a.rows_per_gate;
    const Range ins[] = {{h, all}, {y, all}, {w, D * e}, {gate, gates * D * e}, {scale, D * e}, {w_next, D * e},
                         {stats, 2 * N * 4}, {grad_x == grad_y ? nullptr : grad_y, all}, {grad_u, all}};
    const Range outs[] = {{grad_x, all}, {grad_h, all}, {grad_w, D * e}, {grad_gate, gates * D * e}, {grad_scale, D * e},
                          {grad_w_next, D * e}, {workspace, need}};
    if (any_overlap(outs, ins)) return CGTP_EINVAL;
    a.h = h; a.y = const_cast<void*>(y); a.ldx = D; a.w = w; a.gate = gate; a.scale = scale; a.wn = w_next;
    a.rstd_h = const_cast<float*>(stats);
    a.rstd_y = const_cast<float*>(stats) + N;
    a.gy = grad_y; a.gu = grad_u; a.ldg = D;
    a.gx = grad_x; a.gh = grad_h; a.gw = grad_w; a.ggate = N > 0 ? grad_gate : nullptr; a.gscale = grad_scale; a.gwn = grad_w_next;
    a.partial = (float*)workspace;
    return status(ffn::launch_norm_backward(a, norm->dtype, hip_stream));
}

int ffn_dropout(const void* x, int64_t ldx, void* y, int64_t ldy, int64_t N, int64_t width, int32_t dtype, double p,
                uint64_t seed, uint64_t offset, void* hip_stream) {
    ffn::DropArgs d;
    if (N < 0 || width < 1) return CGTP_EINVAL;
    if (!known(dtype)) return CGTP_EDTYPE;
    if (!drop_args(p, seed, offset, &d)) return CGTP_EINVAL;
    if (N == 0) return CGTP_OK;
    if (!x || !y || ldx < width || ldy < width) return CGTP_EINVAL;
    const int64_t e = size_of(dtype);
    if (misaligned({x, y}, e)) return CGTP_EINVAL;
    // one row may be a whole array; the column's block index is 32 bits wide
    if (N > FFN_MAX_ROWS || width > (1LL << 34) || ldx > (1LL << 34) || ldy > (1LL << 34) ||
        N > (1LL << 60) / ((ldx > ldy ? ldx : ldy) * e))
        return CGTP_EUNSUP;
    const Range ins[] = {{y == x && ldy == ldx ? nullptr : x, span(N, ldx, width, e)}};
    const Range outs[] = {{y, span(N, ldy, width, e)}};
    if (any_overlap(outs, ins)) return CGTP_EINVAL;
    return status(ffn::launch_dropout(x, ldx, y, ldy, N, width, dtype, d, hip_stream));
}

}  // extern "C"
