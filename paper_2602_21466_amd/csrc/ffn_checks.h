// Argument checks and sizes that the C entries of the feed-forward sublayer and of its experts share: ranges that overlap,
// alignment, workspaces, norms' descriptions, operands that are packed before a product.  Internal; host code.
#pragma once

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstddef>
#include <cstdint>
#include <initializer_list>

#include "cgtp_internal.h"
#include "ffn_internal.h"

namespace {

constexpr int64_t kMaxStride = 1LL << 21;   // byte offsets within a tile of 256 rows stay below 2^31

// An array's bytes, from the first to the last; for rows with a stride, that and the row's own bytes (else 0).
struct Range { const void* p; int64_t bytes, ld, width; };

// Rows of one stride, or a block beside them, may lie in one another's gaps, as neighbouring columns of one array do.
inline bool overlaps(const Range& a, const Range& b) {
    if (!a.p || !b.p || a.bytes <= 0 || b.bytes <= 0) return false;
    const int64_t apart = (int64_t)((uintptr_t)b.p - (uintptr_t)a.p);
    if (apart >= a.bytes || -apart >= b.bytes) return false;
    const int64_t ld = a.ld ? a.ld : b.ld;
    if (ld == 0 || (b.ld && b.ld != ld)) return true;
    int64_t at = apart % ld;   // of b's rows in a's
    if (at < 0) at += ld;
    return at < (a.ld ? a.width : a.bytes) || at + (b.ld ? b.width : b.bytes) > ld;
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

inline int64_t size_of(int32_t dtype) { return dtype == FFN_FP32 ? 4 : 2; }
inline bool known(int32_t dtype) { return dtype == FFN_FP32 || dtype == FFN_BF16 || dtype == FFN_FP16; }
inline int64_t aligned(int64_t bytes) { return (bytes + 255) & ~255LL; }
// N rows of `width` values, `ld` apart
inline Range rows(const void* p, int64_t N, int64_t ld, int64_t width, int64_t e) {
    return {p, N > 0 ? ((N - 1) * ld + width) * e : 0, ld * e, width * e};
}

inline bool misaligned(std::initializer_list<const void*> ps, int64_t e) {
    uintptr_t all = 0;
    for (const void* p : ps) all |= (uintptr_t)p;
    return (all & (uintptr_t)(e - 1)) != 0;
}

inline int workspace_ok(const void* ws, int64_t bytes, int64_t need) {
    if (bytes < need || (need > 0 && !ws) || ((uintptr_t)ws & 255)) return CGTP_EINVAL;
    return CGTP_OK;
}

inline int status(int err) {
    if (err == 0) return CGTP_OK;
    cgtp::set_last_hip_error(err);
    return CGTP_EHIP;
}

inline int current_device_is(int device) {
    int dev = -1;
    const hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return status((int)e);
    return dev == device ? CGTP_OK : CGTP_EINVAL;
}

// p in [0, 1]: threshold of the 16-bit draws and the scale that keeps the expected value
inline bool drop_args(double p, uint64_t seed, uint64_t offset, ffn::DropArgs* d) {
    if (!(p >= 0.0 && p <= 1.0)) return false;
    d->threshold = (uint32_t)std::floor(p * 65536.0 + 0.5);
    d->scale = d->threshold < 65536u ? (float)(65536.0 / (65536.0 - d->threshold)) : 0.0f;
    d->seed = seed;
    d->offset = offset;
    return true;
}

inline int check_norm(const ffn_norm* n, int64_t N, ffn::NormArgs* a) {
    if (!n || N < 0 || n->width < 1 || n->rows_per_gate < 1) return CGTP_EINVAL;
    if (!(n->eps > 0.0f) || std::isinf(n->eps)) return CGTP_EINVAL;
    if (!known(n->dtype)) return CGTP_EDTYPE;
    *a = ffn::NormArgs();
    if (!drop_args(n->dropout, n->seed, n->offset, &a->drop)) return CGTP_EINVAL;
    if (n->width > FFN_MAX_WIDTH || N > FFN_MAX_ROWS) return CGTP_EUNSUP;
    a->width = n->width;
    a->N = N;
    a->rows_per_gate = n->rows_per_gate < FFN_MAX_ROWS ? n->rows_per_gate : FFN_MAX_ROWS;   // (32 bits)
    a->eps = n->eps;
    return CGTP_OK;
}

inline int64_t up8(int64_t n) { return (n + 7) & ~7LL; }
inline int64_t tiles(int64_t n, int64_t t) { return (n + t - 1) / t; }

// A matrix as the products read it.
struct Operand { const void* p; int64_t ld; };

inline int64_t packed_bytes(int64_t rows, int64_t width, int32_t dtype) { return aligned(rows * up8(width) * size_of(dtype)); }

// Values a 16-byte chunk holds.
inline int64_t chunk(int32_t dtype) { return 16 / size_of(dtype); }

// Matrices whose rows start on 16 bytes and hold whole chunks of 16 are read where they are, others packed.
inline bool as_is(const void* p, int64_t ld, int64_t rows, int64_t width, int32_t dtype) {
    const int64_t c = chunk(dtype);
    return ((uintptr_t)p & 15) == 0 && width % c == 0 && (ld % c == 0 || rows == 1);
}

inline Operand operand(const void* p, int64_t ld, int64_t rows, int64_t width, int32_t dtype, void* scratch, ffn::PackJobs* jobs) {
    if (as_is(p, ld, rows, width, dtype)) return {p, ld % chunk(dtype) == 0 ? ld : up8(width)};
    jobs->job[jobs->n++] = {p, scratch, ld, rows, width, up8(width), 0};
    return {scratch, up8(width)};
}

}  // namespace
