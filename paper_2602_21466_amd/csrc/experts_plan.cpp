// C ABI of mixtures of feed-forward blocks (include/experts.h): argument checks, workspaces, and the order of the launches.
#include <hip/hip_runtime.h>

#include <new>

#include "experts_internal.h"
#include "ffn_checks.h"

namespace {

// Slots a work-group of the sorting kernels, and work-groups.  One alone up to 8192 slots; at most 128, each of which reads
// all of the others' counts.
struct Sort { int64_t chunk; int32_t groups; };
Sort sort_of(int64_t slots) {
    if (slots <= 8192) return {8192, 1};
    int64_t chunk = (slots + 127) / 128;
    if (chunk < 2048) chunk = 2048;
    return {chunk, (int32_t)((slots + chunk - 1) / chunk)};
}

int check_slots(int64_t N, int64_t per_row, int64_t experts) {
    if (N < 0 || per_row < 1 || experts < 1) return CGTP_EINVAL;
    if (experts > FFN_MAX_EXPERTS || per_row > FFN_MAX_EXPERTS || N > FFN_MAX_ROWS || N * per_row > FFN_MAX_ROWS) return CGTP_EUNSUP;
    return CGTP_OK;
}

int check_rows(int64_t N, int64_t per_row, int64_t experts, int64_t width, int32_t dtype) {
    if (width < 1) return CGTP_EINVAL;
    const int rc = check_slots(N, per_row, experts);
    if (rc == CGTP_EINVAL) return rc;
    if (!known(dtype)) return CGTP_EDTYPE;
    return width > FFN_MAX_WIDTH ? CGTP_EUNSUP : rc;
}

}  // namespace

extern "C" {

int64_t ffn_route_workspace_bytes(int64_t N, int32_t per_row, int32_t experts) {
    if (check_slots(N, per_row, experts) != CGTP_OK) return -1;
    const Sort s = sort_of(N * per_row);
    return s.groups > 1 ? aligned((int64_t)s.groups * experts * 4) : 0;
}

int ffn_route(const void* index, int32_t index_bytes, int64_t N, int32_t per_row, int32_t experts, int32_t* place,
              int32_t* source, int32_t* offsets, void* workspace, int64_t workspace_bytes, void* hip_stream) {
    int rc = check_slots(N, per_row, experts);
    if (rc != CGTP_OK) return rc;
    if ((index_bytes != 4 && index_bytes != 8) || !offsets || (N > 0 && (!index || !place || !source))) return CGTP_EINVAL;
    if (misaligned({index}, index_bytes) || misaligned({place, source, offsets}, 4)) return CGTP_EINVAL;
    const int64_t slots = N * per_row, need = ffn_route_workspace_bytes(N, per_row, experts);
    rc = workspace_ok(workspace, workspace_bytes, need);
    if (rc != CGTP_OK) return rc;
    const Range ins[] = {{index, slots * index_bytes}};
    const Range outs[] = {{place, slots * 4}, {source, slots * 4}, {offsets, (experts + 1) * 4LL}, {workspace, need}};
    if (any_overlap(outs, ins)) return CGTP_EINVAL;
    const Sort s = sort_of(slots);
    ffn::SortArgs a = {};
    a.index = index; a.index_bytes = index_bytes; a.experts = experts;
    a.slots = slots; a.chunk = s.chunk; a.groups = s.groups;
    a.place = place; a.source = source; a.offsets = offsets;
    a.counts = (int32_t*)workspace;
    return status(ffn::launch_sort(a, hip_stream));
}

int ffn_route_gather(const void* x, int64_t ldx, const int32_t* place, const int32_t* offsets, void* xs, int64_t N,
                     int32_t per_row, int32_t experts, int64_t width, int32_t dtype, void* hip_stream) {
    const int rc = check_rows(N, per_row, experts, width, dtype);
    if (rc != CGTP_OK) return rc;
    if (N == 0) return CGTP_OK;
    if (!x || !place || !offsets || !xs || ldx < width) return CGTP_EINVAL;
    if (ldx > kMaxStride) return CGTP_EUNSUP;
    const int64_t e = size_of(dtype), slots = N * per_row;
    if (misaligned({x, xs}, e) || misaligned({place, offsets}, 4)) return CGTP_EINVAL;
    const Range ins[] = {rows(x, N, ldx, width, e), {place, slots * 4}, {offsets, (experts + 1) * 4LL}};
    const Range outs[] = {{xs, slots * width * e}};
    if (any_overlap(outs, ins)) return CGTP_EINVAL;
    ffn::RouteArgs a = {};
    a.N = N; a.width = width; a.per_row = per_row; a.slots = slots;
    a.place = place; a.offsets = offsets; a.experts = experts;
    a.rows = x; a.ld = ldx; a.out_sorted = xs; a.ld_sorted = width;
    return status(ffn::launch_gather(a, dtype, hip_stream));
}

int ffn_route_combine(const void* ys, const int32_t* place, const float* weights, void* y, int64_t ldy, int64_t N,
                      int32_t per_row, int64_t width, int32_t dtype, void* hip_stream) {
    const int rc = check_rows(N, per_row, 1, width, dtype);
    if (rc != CGTP_OK) return rc;
    if (N == 0) return CGTP_OK;
    if (!ys || !place || !y || ldy < width) return CGTP_EINVAL;
    if (ldy > kMaxStride) return CGTP_EUNSUP;
    const int64_t e = size_of(dtype), slots = N * per_row;
    if (misaligned({ys, y}, e) || misaligned({place, weights}, 4)) return CGTP_EINVAL;
    const Range ins[] = {{ys, slots * width * e}, {place, slots * 4}, {weights, slots * 4}};
    const Range outs[] = {rows(y, N, ldy, width, e)};
    if (any_overlap(outs, ins)) return CGTP_EINVAL;
    ffn::RouteArgs a = {};
    a.N = N; a.width = width; a.per_row = per_row; a.slots = slots;
    a.place = place; a.weights = weights;
    a.sorted = ys; a.out_rows = y; a.ld_out = ldy;
    return status(ffn::launch_combine(a, dtype, hip_stream));
}

int ffn_route_combine_backward(const void* ys, const int32_t* place, const int32_t* offsets, const float* weights,
                               const void* grad_y, int64_t ldg, void* grad_ys, float* grad_weights, int64_t N,
                               int32_t per_row, int32_t experts, int64_t width, int32_t dtype, void* hip_stream) {
    const int rc = check_rows(N, per_row, experts, width, dtype);
    if (rc != CGTP_OK) return rc;
    if (N == 0) return CGTP_OK;
    if (!grad_ys && !grad_weights) return CGTP_EINVAL;
    if (!place || !offsets || !grad_y || (grad_weights && !ys) || ldg < width) return CGTP_EINVAL;
    if (ldg > kMaxStride) return CGTP_EUNSUP;
    const int64_t e = size_of(dtype), slots = N * per_row;
    if (!grad_weights) ys = nullptr;
    if (!grad_ys) weights = nullptr;
    if (misaligned({ys, grad_y, grad_ys}, e) || misaligned({place, offsets, weights, grad_weights}, 4)) return CGTP_EINVAL;
    const Range ins[] = {{ys, slots * width * e}, {place, slots * 4}, {offsets, (experts + 1) * 4LL}, {weights, slots * 4},
                         rows(grad_y, N, ldg, width, e)};
    const Range outs[] = {{grad_ys, slots * width * e}, {grad_weights, slots * 4}};
    if (any_overlap(outs, ins)) return CGTP_EINVAL;
    ffn::RouteArgs a = {};
    a.N = N; a.width = width; a.per_row = per_row; a.slots = slots;
    a.place = place; a.offsets = offsets; a.experts = experts; a.weights = weights;
    a.rows = grad_y; a.ld = ldg; a.sorted = ys;
    a.out_sorted = grad_ys; a.ld_sorted = width; a.grad_weights = grad_weights;
    return status(ffn::launch_combine_backward(a, dtype, hip_stream));
}

}  // extern "C"
