// C ABI of the layer norm (include/ffn.h): argument checks and launches.
#include <hip/hip_runtime.h>

#include "experts_internal.h"
#include "ffn_checks.h"

namespace {

int check(const ffn_norm* norm, int64_t N, ffn::LayerArgs* a) {
    ffn::NormArgs n;
    const int rc = check_norm(norm, N, &n);
    if (rc != CGTP_OK) return rc;
    *a = ffn::LayerArgs();
    a->width = n.width;
    a->N = N;
    a->eps = n.eps;
    return CGTP_OK;
}

}  // namespace

extern "C" {

int ffn_layer_forward(const ffn_norm* norm, const void* x, int64_t ldx, const void* w, const void* b, void* u, int64_t ldu,
                      float* stats, int64_t N, void* hip_stream) {
    ffn::LayerArgs a;
    const int rc = check(norm, N, &a);
    if (rc != CGTP_OK) return rc;
    if (N == 0) return CGTP_OK;
    if (!x || !u || ldx < a.width || ldu < a.width) return CGTP_EINVAL;
    if (ldx > kMaxStride || ldu > kMaxStride) return CGTP_EUNSUP;
    const int64_t e = size_of(norm->dtype), D = a.width;
    if (misaligned({x, w, b, u}, e) || misaligned({stats}, 4)) return CGTP_EINVAL;
    const Range ins[] = {rows(u == x && ldu == ldx ? nullptr : x, N, ldx, D, e), {w, D * e}, {b, D * e}};
    const Range outs[] = {rows(u, N, ldu, D, e), {stats, 2 * N * 4}};
    const Range all[] = {rows(x, N, ldx, D, e)}, stat[] = {{stats, 2 * N * 4}};
    if (any_overlap(outs, ins) || any_overlap(stat, all)) return CGTP_EINVAL;
    a.x = x; a.ldx = ldx; a.w = w; a.b = b;
    a.u = u; a.ldu = ldu; a.stats = stats;
    switch (norm->dtype) {
        case FFN_FP32: return status(ffn::launch_layer_forward_fp32(a, hip_stream));
        case FFN_BF16: return status(ffn::launch_layer_forward_bf16(a, hip_stream));
        default: return status(ffn::launch_layer_forward_fp16(a, hip_stream));
    }
}

int64_t ffn_layer_workspace_bytes(const ffn_norm* norm, int64_t N) {
    ffn::LayerArgs a;
    if (check(norm, N, &a) != CGTP_OK) return -1;
    return aligned(ffn::layer_workspace_floats(a.width, N, (int)size_of(norm->dtype)) * 4);
}

int ffn_layer_backward(const ffn_norm* norm, const void* x, int64_t ldx, const void* w, const float* stats,
                       const void* grad_u, int64_t ldg, void* grad_x, void* grad_w, void* grad_b, int64_t N,
                       void* workspace, int64_t workspace_bytes, void* hip_stream) {
    ffn::LayerArgs a;
    int rc = check(norm, N, &a);
    if (rc != CGTP_OK) return rc;
    if (N == 0 && !grad_w && !grad_b) return CGTP_OK;   // (an empty grad_x may be NULL)
    if (!grad_x && !grad_w && !grad_b) return CGTP_EINVAL;
    if (N > 0 && (!x || !stats || !grad_u || ldx < a.width || ldg < a.width)) return CGTP_EINVAL;
    if (ldx > kMaxStride || ldg > kMaxStride) return CGTP_EUNSUP;
    const int64_t e = size_of(norm->dtype), D = a.width;
    if (misaligned({x, w, grad_u, grad_x, grad_w, grad_b}, e) || misaligned({stats}, 4)) return CGTP_EINVAL;
    const int64_t need = ffn_layer_workspace_bytes(norm, N);
    rc = workspace_ok(workspace, workspace_bytes, need);
    if (rc != CGTP_OK) return rc;
    const Range ins[] = {rows(x, N, ldx, D, e), {w, D * e}, {stats, 2 * N * 4}, rows(grad_u, N, ldg, D, e)};
    const Range outs[] = {{grad_x, N * D * e}, {grad_w, D * e}, {grad_b, D * e}, {workspace, need}};
    if (any_overlap(outs, ins)) return CGTP_EINVAL;
    a.x = x; a.ldx = ldx; a.w = w; a.stats = const_cast<float*>(stats);
    a.gu = grad_u; a.ldg = ldg; a.gx = grad_x; a.gw = grad_w; a.gb = grad_b;
    a.partial = (float*)workspace;
    switch (norm->dtype) {
        case FFN_FP32: return status(ffn::launch_layer_backward_fp32(a, hip_stream));
        case FFN_BF16: return status(ffn::launch_layer_backward_bf16(a, hip_stream));
        default: return status(ffn::launch_layer_backward_fp16(a, hip_stream));
    }
}

}  // extern "C"
