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

constexpr int64_t kMaxStride = 1LL << 21;   // byte offsets within a tile of 256 rows stay below 2^31

// An array's bytes, from the first to the last; for rows with a stride, that and the row's own bytes (else 0).
struct Range { const void* p; int64_t bytes, ld, width; };

// Rows of one stride, or a block beside them, may lie in one another's gaps, as neighbouring columns of one array do.
bool overlaps(const Range& a, const Range& b) {
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

int64_t size_of(int32_t dtype) { return dtype == FFN_FP32 ? 4 : 2; }
bool known(int32_t dtype) { return dtype == FFN_FP32 || dtype == FFN_BF16 || dtype == FFN_FP16; }
int64_t aligned(int64_t bytes) { return (bytes + 255) & ~255LL; }
// N rows of `width` values, `ld` apart
Range rows(const void* p, int64_t N, int64_t ld, int64_t width, int64_t e) {
    return {p, N > 0 ? ((N - 1) * ld + width) * e : 0, ld * e, width * e};
}

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
    a->rows_per_gate = n->rows_per_gate < FFN_MAX_ROWS ? n->rows_per_gate : FFN_MAX_ROWS;   // (32 bits)
    a->eps = n->eps;
    return CGTP_OK;
}

int64_t up8(int64_t n) { return (n + 7) & ~7LL; }
int64_t tiles(int64_t n, int64_t t) { return (n + t - 1) / t; }

// How a product is cut up: work-groups of `tile` x `tile` outputs, k in `splits` parts; joined: the parts' sums (also of
// one part) go to memory and a second kernel finishes them.
struct Cut { int32_t tile, splits; bool joined; };

// The shortest by this count, in microseconds.  A compute unit takes a 256-wide tile's step (64 k of 16 bits, 32 of 32
// bits) in 1.6 (4.5), or two 128-wide tiles' in 1.06 (2.6), one alone in about three quarters of that (measured on large products:
// bf16 1.33 and 1.0 PFLOP/s, fp32 238 and 209 TFLOP/s).  Four (two) steps stand for a tile's start and end.  Parts of k cost
// a launch (three microseconds, and a tenth of one a part) and their sums, written and read once at 4 TB/s; the gate's
// gradient in the tiles' own epilogue costs ten where they are few (4004 rows, 144 x 348: 26 us, against 17 with the
// joining kernel).
Cut choose(int64_t M, int64_t N, int64_t K, int32_t dtype, int32_t epilogue) {
    const bool wide = dtype == FFN_FP32;
    const int64_t steps = tiles(K, wide ? 32 : 64);
    const double ends = wide ? 2.0 : 4.0;
    Cut best = {256, 1, false};
    double least = 1e300;
    for (int32_t tile : {256, 128}) {
        const int64_t groups = tiles(M, tile) * tiles(N, tile), slots = tile == 256 ? 256 : 512;
        const double step = tile == 256 ? (wide ? 4.5 : 1.6) : (wide ? 2.6 : 1.06);
        for (int32_t s = 1; s <= 64 && (s == 1 || steps / s >= 4); ++s) {
            const int64_t whole = groups * s / slots, rest = groups * s - whole * slots;
            const double rounds = (double)whole + (rest == 0 ? 0.0 : tile == 128 && rest <= 256 ? 0.75 : 1.0);
            const double t = rounds * ((double)tiles(steps, s) + ends) * step;
            const double join = 3.0 + 0.1 * s + (double)(M * N * s) * 8.0 / 4e6, own = epilogue == ffn::kGateGrad ? 10.0 : 0.0;
            const bool joined = s > 1 || own > join;
            if (t + (joined ? join : own) < least) { least = t + (joined ? join : own); best = {tile, s, joined}; }
        }
    }
    return best;
}

// Bytes of the partial sums of an [M, N] product.
int64_t partial_bytes(int64_t M, int64_t N, int64_t K, int32_t dtype, int32_t epilogue = ffn::kStore) {
    const Cut c = choose(M, N, K, dtype, epilogue);
    return c.joined ? aligned(c.splits * M * ((N + 3) & ~3LL) * 4) : 0;
}

// Whether an [M, N] product's work-groups are within one launch.
bool fits(int64_t M, int64_t N, int64_t K, int32_t dtype, int32_t epilogue = ffn::kStore) {
    const Cut c = choose(M, N, K, dtype, epilogue);
    return tiles(M, c.tile) * tiles(N, c.tile) * c.splits <= 0x7FFFFFFF / 512;
}

int launch_tile(const ffn::TileArgs& t, int32_t epilogue, bool ac, bool bc, int32_t dtype, int32_t tile, void* stream) {
    switch (dtype) {
        case FFN_FP32: return ffn::launch_tile_fp32(t, epilogue, ac, bc, tile, stream);
        case FFN_BF16: return ffn::launch_tile_bf16(t, epilogue, ac, bc, tile, stream);
        default: return ffn::launch_tile_fp16(t, epilogue, ac, bc, tile, stream);
    }
}

// Runs the product whose operands, sizes and results `t` describes; `partial` is scratch of partial_bytes() (for kGate,
// of 2 N columns).
int product(ffn::TileArgs t, int32_t epilogue, bool ac, bool bc, int32_t dtype, void* partial, void* stream) {
    const int64_t columns = epilogue == ffn::kGate ? 2 * t.N : t.N;
    const Cut c = choose(t.M, columns, t.K, dtype, epilogue);
    const int64_t tm = tiles(t.M, c.tile), tn = tiles(columns, c.tile);
    t.tiles_m = (int32_t)tm;
    t.tiles_n = (int32_t)tn;
    t.splits = c.splits;
    if (!c.joined) return status(launch_tile(t, epilogue, ac, bc, dtype, c.tile, stream));
    ffn::TileArgs s = t;
    s.c = partial;
    s.N = columns;
    s.ldc = (columns + 3) & ~3LL;
    const int rc = status(launch_tile(s, ffn::kPartial, ac, bc, dtype, c.tile, stream));
    if (rc != CGTP_OK) return rc;
    if (epilogue == ffn::kStore)
        return status(ffn::launch_join((const float*)partial, s.ldc, c.splits, t.M, t.N, t.c, dtype, stream));
    return status(ffn::launch_join_gate(t, epilogue, (const float*)partial, s.ldc, dtype, stream));
}

// A product for few rows: weight rows a work-group, and waves (parts of k).  Measured, bf16: up to 16 rows of x, 8 a
// work-group (2048 x 8192, one row: 9.7 us against 12.6 with 16; 16384 x 4096 gated: 48.7 against 49.6), which the
// 32-bit instruction, at an eighth of the rate, does not follow; with more rows of x 16 (4096 x 16384, 24 rows: 45
// against 62), and 32 where two work-groups a compute unit are left (16384 x 4096 gated, 24 rows: 57 against 61).  8
// always where 16 would leave a quarter of the compute units idle (2048 x 2048 gated, 40 rows: 10.3 against 11.7).
int few_product(const ffn::FewArgs& p, int32_t epilogue, int32_t dtype, void* stream) {
    const bool gate = epilogue == ffn::kGate;
    const int32_t nr = (p.M <= 16 && dtype != FFN_FP32) || p.N < 16 * 192 ? 8 : gate && p.M > 16 && p.N >= 32 * 512 ? 32 : 16;
    const int32_t mt = p.M <= 16 ? 1 : p.M <= 32 ? 2 : 4, per = (nr > 16 ? 2 : 1) * (gate ? 2 : 1) * mt;
    int32_t waves = 8;
    // blocks of k: one a wave or more, and where there are waves enough, four (8192 x 2048 gated: 13.5 us, with two 14.4)
    const int64_t blocks = tiles(p.K, dtype == FFN_FP32 ? 64 : 128), groups = tiles(p.N, nr);
    while (waves > 1 && (waves * per > 64 || waves > 2 * blocks || (waves * 4 > blocks && groups * waves > 4096))) waves /= 2;
    switch (dtype) {
        case FFN_FP32: return status(ffn::launch_few_fp32(p, epilogue, nr, waves, stream));
        case FFN_BF16: return status(ffn::launch_few_bf16(p, epilogue, nr, waves, stream));
        default: return status(ffn::launch_few_fp16(p, epilogue, nr, waves, stream));
    }
}

// Gradients' products for few rows of 32-bit arrays: about two work-groups a compute unit by parts of k.
bool few_grad(int64_t M, int64_t N, int32_t dtype) { return dtype == FFN_FP32 && M <= ffn::kFewRows && N >= 4; }
struct FewCut { int32_t splits, waves; };
FewCut few_cut(int64_t M, int64_t N, int64_t K) {
    const int32_t waves = M <= 32 ? 8 : 4;
    const int64_t blocks = tiles(N, 64), most = tiles(K, 32 * waves), want = tiles(512, blocks);
    return {(int32_t)(want < most ? want : most), waves};
}
int64_t few_grad_bytes(int64_t M, int64_t N, int64_t K) { return aligned(few_cut(M, N, K).splits * M * ((N + 3) & ~3LL) * 4); }

// t describes the product and its results as for product(): t.a the rows, t.b [K, N].
int few_grad_product(ffn::TileArgs t, int32_t epilogue, void* partial, void* stream) {
    const FewCut c = few_cut(t.M, t.N, t.K);
    ffn::FewGradArgs f = {};
    f.x = t.a; f.ldx = t.lda; f.w = t.b; f.ldw = t.ldb;
    f.M = t.M; f.N = t.N; f.K = t.K;
    f.c = (float*)partial; f.ldc = (t.N + 3) & ~3LL;
    f.splits = c.splits; f.waves = c.waves;
    const int rc = status(ffn::launch_few_grad(f, stream));
    if (rc != CGTP_OK) return rc;
    t.splits = c.splits;
    if (epilogue == ffn::kGateGrad) return status(ffn::launch_join_gate(t, epilogue, f.c, f.ldc, FFN_FP32, stream));
    return status(ffn::launch_join(f.c, f.ldc, c.splits, t.M, t.N, t.c, FFN_FP32, stream));
}

// A matrix as the products read it.
struct Operand { const void* p; int64_t ld; };

int64_t packed_bytes(int64_t rows, int64_t width, int32_t dtype) { return aligned(rows * up8(width) * size_of(dtype)); }

// Values a 16-byte chunk holds.
int64_t chunk(int32_t dtype) { return 16 / size_of(dtype); }

// Matrices whose rows start on 16 bytes and hold whole chunks of 16 are read where they are, others packed.
bool as_is(const void* p, int64_t ld, int64_t rows, int64_t width, int32_t dtype) {
    const int64_t c = chunk(dtype);
    return ((uintptr_t)p & 15) == 0 && width % c == 0 && (ld % c == 0 || rows == 1);
}

Operand operand(const void* p, int64_t ld, int64_t rows, int64_t width, int32_t dtype, void* scratch, ffn::PackJobs* jobs) {
    if (as_is(p, ld, rows, width, dtype)) return {p, ld % chunk(dtype) == 0 ? ld : up8(width)};
    jobs->job[jobs->n++] = {p, scratch, ld, rows, width, up8(width), 0};
    return {scratch, up8(width)};
}

// Byte offsets in the block's workspace: intermediates, operands to be packed, partial sums.
struct Layout { int64_t h, dgu, x, w_in, w_out, gy, partial, total; };
Layout layout(const ffn_plan_s* p, int64_t N, bool backward) {
    const int64_t di = p->d_in, df = p->d_ff, d_o = p->d_out;
    const int32_t t = p->dtype;
    Layout l = {};
    int64_t at = 0;
    auto take = [&](int64_t bytes) { const int64_t o = at; at += bytes; return o; };
    // weights are contiguous and start on 16 bytes: they need packing by their width alone
    l.h = take(packed_bytes(N, df, t));
    l.x = take(packed_bytes(N, di, t));
    l.w_in = take(di % chunk(t) ? packed_bytes(2 * df, di, t) : 0);
    l.w_out = take(df % chunk(t) ? packed_bytes(d_o, df, t) : 0);
    int64_t partial = 0;
    auto also = [&](int64_t bytes) { partial = bytes > partial ? bytes : partial; };
    if (backward) {
        l.dgu = take(packed_bytes(N, 2 * df, t));
        l.gy = take(packed_bytes(N, d_o, t));
        also(few_grad(N, df, t) ? few_grad_bytes(N, df, d_o) : partial_bytes(N, df, d_o, t, ffn::kGateGrad));
        also(few_grad(N, di, t) ? few_grad_bytes(N, di, 2 * df) : partial_bytes(N, di, 2 * df, t));
        also(partial_bytes(2 * df, di, N, t));
        also(partial_bytes(d_o, df, N, t));
    } else {
        also(partial_bytes(N, 2 * df, di, t));
        also(partial_bytes(N, d_o, df, t));
    }
    l.partial = take(partial);
    l.total = at;
    return l;
}

int norm_forward(const ffn::NormArgs& a, int32_t dtype, void* stream) {
    return dtype == FFN_FP32   ? ffn::launch_norm_forward_fp32(a, stream)
           : dtype == FFN_BF16 ? ffn::launch_norm_forward_bf16(a, stream)
                               : ffn::launch_norm_forward_fp16(a, stream);
}
int norm_backward(const ffn::NormArgs& a, int32_t dtype, void* stream) {
    return dtype == FFN_FP32   ? ffn::launch_norm_backward_fp32(a, stream)
           : dtype == FFN_BF16 ? ffn::launch_norm_backward_bf16(a, stream)
                               : ffn::launch_norm_backward_fp16(a, stream);
}
int dropout(const void* x, int64_t ldx, void* y, int64_t ldy, int64_t N, int64_t width, int32_t dtype, const ffn::DropArgs& d,
            void* stream) {
    return dtype == FFN_FP32   ? ffn::launch_dropout_fp32(x, ldx, y, ldy, N, width, d, stream)
           : dtype == FFN_BF16 ? ffn::launch_dropout_bf16(x, ldx, y, ldy, N, width, d, stream)
                               : ffn::launch_dropout_fp16(x, ldx, y, ldy, N, width, d, stream);
}

// Y = H Wo^T by tiles.
int down(const ffn_plan_s* plan, const void* h, const Operand& w, void* y, int64_t N, void* partial, void* stream) {
    ffn::TileArgs o = {};
    o.a = h; o.lda = up8(plan->d_ff);
    o.b = w.p; o.ldb = w.ld;
    o.M = N; o.N = plan->d_out; o.K = plan->d_ff;
    o.c = y; o.ldc = plan->d_out;
    return product(o, ffn::kStore, false, false, plan->dtype, partial, stream);
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
    if (misaligned({x}, e) || misaligned({w_in, w_out, y, saved}, 16)) return CGTP_EINVAL;
    if (!fits(N, 2 * df, di, plan->dtype) || !fits(N, d_o, df, plan->dtype)) return CGTP_EUNSUP;
    const Layout l = layout(plan, N, false);
    int rc = workspace_ok(workspace, workspace_bytes, l.total);
    if (rc != CGTP_OK) return rc;
    const Range ins[] = {rows(x, N, ldx, di, e), {w_in, 2 * df * di * e}, {w_out, d_o * df * e}};
    const Range outs[] = {{y, N * d_o * e}, {saved, N * 2 * df * 4}, {workspace, l.total}};
    if (any_overlap(outs, ins)) return CGTP_EINVAL;
    rc = current_device_is(plan->device);
    if (rc != CGTP_OK) return rc;
    char* ws = (char*)workspace;
    if (N <= ffn::kFewRows) {
        ffn::FewArgs g = {};
        g.x = x; g.ldx = ldx; g.w = w_in; g.ldw = di;
        g.M = N; g.N = df; g.K = di;
        g.c = ws + l.h; g.ldc = up8(df);
        g.act = plan->act; g.saved = (float*)saved;
        rc = few_product(g, ffn::kGate, plan->dtype, hip_stream);
        if (rc != CGTP_OK) return rc;
        // from here on the weights alone are many: 16-bit ones that need no packing go through LDS in 128-wide tiles with
        // k in parts, which passes 16 rows of x (4096 x 16384, 24 rows: 38 us with the joining, against 44)
        if (N > 16 && plan->dtype != FFN_FP32 && as_is(w_out, df, d_o, df, plan->dtype)) return down(plan, ws + l.h, {w_out, df}, y, N, ws + l.partial, hip_stream);
        ffn::FewArgs o = {};
        o.x = ws + l.h; o.ldx = up8(df); o.w = w_out; o.ldw = df;
        o.M = N; o.N = d_o; o.K = df;
        o.c = y; o.ldc = d_o;
        return few_product(o, ffn::kStore, plan->dtype, hip_stream);
    }
    ffn::PackJobs jobs = {};
    const Operand X = operand(x, ldx, N, di, plan->dtype, ws + l.x, &jobs), Wi = operand(w_in, di, 2 * df, di, plan->dtype, ws + l.w_in, &jobs),
                  Wo = operand(w_out, df, d_o, df, plan->dtype, ws + l.w_out, &jobs);
    rc = status(ffn::launch_pack(jobs, plan->dtype, hip_stream));
    if (rc != CGTP_OK) return rc;
    ffn::TileArgs g = {};
    g.a = X.p; g.lda = X.ld;
    g.b = Wi.p; g.ldb = Wi.ld;
    g.M = N; g.N = df; g.K = di;
    g.c = ws + l.h; g.ldc = up8(df);
    g.act = plan->act; g.saved = (float*)saved;
    rc = product(g, ffn::kGate, false, false, plan->dtype, ws + l.partial, hip_stream);
    if (rc != CGTP_OK) return rc;
    return down(plan, ws + l.h, Wo, y, N, ws + l.partial, hip_stream);
}

int ffn_backward(ffn_plan_t plan, const void* x, int64_t ldx, const void* w_in, const void* w_out, const void* saved,
                 const void* grad_y, int64_t ldg, void* grad_x, void* grad_w_in, void* grad_w_out, int64_t N,
                 void* workspace, int64_t workspace_bytes, void* hip_stream) {
    if (!plan || N < 0 || (!grad_x && !grad_w_in && !grad_w_out)) return CGTP_EINVAL;
    const int64_t e = size_of(plan->dtype), di = plan->d_in, df = plan->d_ff, d_o = plan->d_out;
    if (N > 0 && (!x || !w_in || !w_out || !saved || !grad_y || ldx < di || ldg < d_o)) return CGTP_EINVAL;
    if (N > FFN_MAX_ROWS || ldx > kMaxStride || ldg > kMaxStride) return CGTP_EUNSUP;
    if (misaligned({x, grad_y}, e) || misaligned({w_in, w_out, saved, grad_x, grad_w_in, grad_w_out}, 16)) return CGTP_EINVAL;
    if (!fits(N, df, d_o, plan->dtype, ffn::kGateGrad) || !fits(N, di, 2 * df, plan->dtype) || !fits(2 * df, di, N, plan->dtype) || !fits(d_o, df, N, plan->dtype))
        return CGTP_EUNSUP;
    const Layout l = layout(plan, N, true);
    int rc = workspace_ok(workspace, workspace_bytes, l.total);
    if (rc != CGTP_OK) return rc;
    const Range ins[] = {rows(x, N, ldx, di, e), {w_in, 2 * df * di * e}, {w_out, d_o * df * e},
                         {saved, N * 2 * df * 4}, rows(grad_y, N, ldg, d_o, e)};
    const Range outs[] = {{grad_x, N * di * e}, {grad_w_in, 2 * df * di * e}, {grad_w_out, d_o * df * e},
                          {workspace, l.total}};
    if (any_overlap(outs, ins)) return CGTP_EINVAL;
    rc = current_device_is(plan->device);
    if (rc != CGTP_OK) return rc;
    if (N == 0) {
        // sums over no rows
        hipStream_t s = (hipStream_t)hip_stream;
        if (grad_w_in) rc = status(ffn::launch_zero(grad_w_in, 2 * df * di * e, s));
        if (rc == CGTP_OK && grad_w_out) rc = status(ffn::launch_zero(grad_w_out, d_o * df * e, s));
        return rc;
    }
    char* ws = (char*)workspace;
    const int32_t dt = plan->dtype;
    const bool few_h = few_grad(N, df, dt), few_x = few_grad(N, di, dt);   // their products read the weights as they are
    ffn::PackJobs jobs = {};
    Operand X = {}, Wi = {}, Wo = {}, Gy = {};
    if (!few_h || grad_w_out) Gy = operand(grad_y, ldg, N, d_o, dt, ws + l.gy, &jobs);
    if (!few_h) Wo = operand(w_out, df, d_o, df, dt, ws + l.w_out, &jobs);
    if (grad_x && !few_x) Wi = operand(w_in, di, 2 * df, di, dt, ws + l.w_in, &jobs);
    if (grad_w_in) X = operand(x, ldx, N, di, dt, ws + l.x, &jobs);
    rc = status(ffn::launch_pack(jobs, dt, hip_stream));
    if (rc != CGTP_OK) return rc;
    const Operand H = {ws + l.h, up8(df)}, D = {ws + l.dgu, up8(2 * df)};
    ffn::TileArgs g = {};
    if (few_h) {
        g.a = grad_y; g.lda = ldg; g.b = w_out; g.ldb = df;
    } else {
        g.a = Gy.p; g.lda = Gy.ld;
        g.b = Wo.p; g.ldb = Wo.ld;
    }
    g.M = N; g.N = df; g.K = d_o;
    g.c = ws + l.dgu; g.ldc = D.ld;
    g.h = ws + l.h; g.ldh = H.ld;
    g.act = plan->act; g.saved = (float*)const_cast<void*>(saved);
    rc = few_h ? few_grad_product(g, ffn::kGateGrad, ws + l.partial, hip_stream)
               : product(g, ffn::kGateGrad, false, true, dt, ws + l.partial, hip_stream);
    if (rc == CGTP_OK && grad_x) {
        ffn::TileArgs t = {};
        t.a = D.p; t.lda = D.ld;
        t.M = N; t.N = di; t.K = 2 * df;
        t.c = grad_x; t.ldc = di;
        if (few_x) {
            t.b = w_in; t.ldb = di;
            rc = few_grad_product(t, ffn::kStore, ws + l.partial, hip_stream);
        } else {
            t.b = Wi.p; t.ldb = Wi.ld;
            rc = product(t, ffn::kStore, false, true, dt, ws + l.partial, hip_stream);
        }
    }
    if (rc == CGTP_OK && grad_w_in) {
        ffn::TileArgs t = {};
        t.a = D.p; t.lda = D.ld;
        t.b = X.p; t.ldb = X.ld;
        t.M = 2 * df; t.N = di; t.K = N;
        t.c = grad_w_in; t.ldc = di;
        rc = product(t, ffn::kStore, true, true, plan->dtype, ws + l.partial, hip_stream);
    }
    if (rc == CGTP_OK && grad_w_out) {
        ffn::TileArgs t = {};
        t.a = Gy.p; t.lda = Gy.ld;
        t.b = H.p; t.ldb = H.ld;
        t.M = d_o; t.N = df; t.K = N;
        t.c = grad_w_out; t.ldc = df;
        rc = product(t, ffn::kStore, true, true, plan->dtype, ws + l.partial, hip_stream);
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
    const Range in_x[] = {rows(u == x && ldu == ldx ? nullptr : x, N, ldx, a.width, e), {w, a.width * e}};
    const Range outs[] = {rows(u, N, ldu, a.width, e), {rstd, N * 4}};
    const Range also[] = {rows(x, N, ldx, a.width, e)};
    const Range stat[] = {{rstd, N * 4}};
    if (any_overlap(outs, in_x) || any_overlap(stat, also)) return CGTP_EINVAL;
    a.x = x; a.ldx = ldx;
    a.u = u; a.ldu = ldu; a.wn = w; a.rstd_y = rstd;
    return status(norm_forward(a, norm->dtype, hip_stream));
}

int64_t ffn_norm_workspace_bytes(const ffn_norm* norm, int64_t N, int32_t residual) {
    ffn::NormArgs a;
    if ((residual & ~1) || check_norm(norm, N, &a) != CGTP_OK) return -1;
    return aligned(ffn::norm_workspace_floats(a.width, N, a.rows_per_gate, residual != 0, (int)size_of(norm->dtype)) * 4);
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
    const Range ins[] = {rows(x, N, ldx, a.width, e), {w, a.width * e}, {rstd, N * 4}, rows(grad_u, N, ldg, a.width, e)};
    const Range outs[] = {{grad_x, N * a.width * e}, {grad_w, a.width * e}, {workspace, need}};
    if (any_overlap(outs, ins)) return CGTP_EINVAL;
    a.y = const_cast<void*>(x); a.ldx = ldx; a.wn = w; a.rstd_y = const_cast<float*>(rstd);
    a.gu = grad_u; a.ldg = ldg; a.gx = grad_x; a.gwn = grad_w;
    a.rows_per_gate = 1;   // there is no gate: its rows divide nothing (as the workspace's size has it)
    a.partial = (float*)workspace;
    return status(norm_backward(a, norm->dtype, hip_stream));
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
    return status(norm_forward(a, norm->dtype, hip_stream));
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
    return status(norm_backward(a, norm->dtype, hip_stream));
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
    const Range ins[] = {rows(y == x && ldy == ldx ? nullptr : x, N, ldx, width, e)};
    const Range outs[] = {rows(y, N, ldy, width, e)};
    if (any_overlap(outs, ins)) return CGTP_EINVAL;
    return status(dropout(x, ldx, y, ldy, N, width, dtype, d, hip_stream));
}

}  // extern "C"
