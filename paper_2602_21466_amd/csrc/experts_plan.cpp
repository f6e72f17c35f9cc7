// C ABI of mixtures of feed-forward blocks (include/experts.h): argument checks, workspaces, and the order of the launches.
#include <hip/hip_runtime.h>

#include <new>

#include "experts_internal.h"
#include "ffn_checks.h"

struct ffn_experts_s {
    int64_t d_in, d_ff, d_out;
    int32_t experts, act, dtype, device;
};

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

// ---------------------------------------------------------------- the experts' products

// How products are cut: work-groups of `tile` x `tile` outputs, k in `splits` parts; joined: the parts' sums (also of one
// part) go to memory and a second kernel finishes them.
struct Cut { int32_t tile, splits; bool joined; };

// What a compute unit takes for a step of k (64 values of 16 bits, 32 of 32) of a 256-wide tile, or of two 128-wide ones, in
// microseconds, and the steps that a tile's start and end stand for (16384 x 4096 outputs, k of 64 and 256: bf16 39 and 57.5
// us by 256-wide tiles, 40 and 67.5 by 128-wide ones; fp32 96 and 215, 83 and 219).
struct Cost { double step, ends; };
Cost cost_of(int32_t tile, bool wide) { return wide ? (tile == 256 ? Cost{4.9, 2.8} : Cost{2.8, 1.8}) : tile == 256 ? Cost{1.6, 5.5} : Cost{1.12, 4.0}; }

// The shortest by a count of those, as a single block's products are cut (ffn_plan.cpp), with what the host knows:
// `groups(tile)` work-groups by the mean, of `steps` steps of k each.  256 of 256-wide tiles or 512 of 128-wide ones run at
// one time, and one 128-wide tile alone takes three quarters of what two take; of 16-bit arrays, what is beyond whole rounds
// of 256-wide tiles is cut into 128-wide ones (ffn_experts.h).  Parts of k cost a launch, a tenth of a microsecond a part and
// their sums, written and read once at 4 TB/s; the gate's gradient in the tiles' own epilogue costs ten where they are few.
template <typename Groups> Cut shortest(Groups groups, int64_t steps, double outputs, bool wide, bool gate_grad) {
    Cut best = {128, 1, false};
    double least = 1e300;
    for (int32_t tile : {256, 128}) {
        const double all = groups(tile), slots = tile == 256 ? 256.0 : 512.0;
        const Cost cost = cost_of(tile, wide);
        for (int32_t s = 1; s <= 64 && (s == 1 || steps / s >= 4); ++s) {
            const double n = all * s / slots, full = std::floor(n), rest = n - full;
            const bool cut = tile == 256 && !wide && s == 1 && full > 0.0;
            const double rounds = full + (rest == 0.0 ? 0.0 : tile == 128 && rest <= 0.5 ? 0.75 : cut && rest <= 0.25 ? 0.45 : cut && rest <= 0.5 ? 0.9 : 1.0);
            const double t = rounds * ((double)tiles(steps, s) + cost.ends) * cost.step;
            const double join = 3.0 + 0.1 * s + outputs * s * 8.0 / 4e6, own = gate_grad ? 10.0 : 0.0;
            const bool joined = s > 1 || own > join;
            if (t + (joined ? join : own) < least) { least = t + (joined ? join : own); best = {tile, s, joined}; }
        }
    }
    return best;
}

// One product: R rows over the plan's experts, N columns, K values.
struct Shape { int64_t R, E, N, K; };

// Tiles of rows there may be.
int64_t most_tiles(const Shape& s, int32_t tile) { return s.R / tile + (s.E < s.R ? s.E : s.R); }

// By the mean, and a little more: each expert with a row has a tile or more, and a run of rows ends in half a tile, with a
// third of a tile as the standard deviation.
double mean_tiles(const Shape& s, int32_t tile) {
    if (s.E == 1) return (double)tiles(s.R, tile);
    const double with = (double)(s.E < s.R ? s.E : s.R), each = (double)s.R / (with * tile) + 0.5;
    return each < 1.0 ? with : with * each + 0.3 * std::sqrt(with);
}

// [R, N], B by expert.
Cut cut_rows(const Shape& s, int32_t dtype, int32_t epilogue) {
    const bool wide = dtype == FFN_FP32;
    auto groups = [&](int32_t tile) { return mean_tiles(s, tile) * (double)tiles(s.N, tile); };
    return shortest(groups, tiles(s.K, wide ? 32 : 64), (double)s.R * s.N, wide, epilogue == ffn::kGateGrad);
}

// The gradients' products of one launch: the rows' [R, d_in], whose k is in `splits` parts, and the weights', sums over each
// expert's rows in parts of `chunk` of them (0: one part an expert).  Counted like shortest(): all work-groups' steps over
// those that run at one time, then half of one that comes late, of the shorter kind where these fill what the longer leave;
// a few experts may have three times the mean.
struct GradCut { int32_t tile, splits, chunk; bool sums_first; };
GradCut cut_grads(const ffn_experts_s* p, int64_t R) {
    const bool wide = p->dtype == FFN_FP32;
    const int64_t di = p->d_in, df = p->d_ff, d_o = p->d_out, E = p->experts, kstep = wide ? 32 : 64, steps = tiles(2 * df, kstep);
    const double k = (double)kstep, mean = (double)R / E, longest = 3.0 * mean < (double)R ? 3.0 * mean : (double)R;
    const double outputs = (double)(2 * df * di) + (double)(d_o * df);
    GradCut best = {128, 1, 0, false};
    double least = 1e300;
    for (int32_t tile : {256, 128}) {
        const double slots = tile == 256 ? 256.0 : 512.0, step = cost_of(tile, wide).step, ends = cost_of(tile, wide).ends;
        const double rows = mean_tiles({R, E, di, 0}, tile) * (double)tiles(di, tile);
        const double each = (double)(tiles(2 * df, tile) * tiles(di, tile) + tiles(d_o, tile) * tiles(df, tile));
        auto consider = [&](int32_t chunk) {
            const double parts = chunk ? (double)R / chunk + 0.5 * E : (double)E, sums = each * ((double)R / k + parts * ends);
            const double one = (chunk ? (double)chunk : longest) / k + ends, join = chunk ? 4.0 + parts * outputs * 4.5 / 4e6 : 0.0;
            for (int32_t s = 1; s <= 64 && (s == 1 || steps / s >= 4); s += s < 4 ? 1 : s / 2) {
                const double own = (double)tiles(steps, s) + ends, all = (rows * s * own + sums) / slots;
                const double less = own < one ? own : one, more = own < one ? one : own, fill = (own < one ? rows * s * own : sums) / slots;
                const double late = rows * s + each * parts <= slots ? 0.0 : 0.5 * more - fill > 0.5 * less ? 0.5 * more - fill : 0.5 * less;
                const double t = step * (all + late > more ? all + late : more) + join + 0.1 * s + (double)R * di * s * 8.0 / 4e6;
                if (t < least) { least = t; best = {tile, s, chunk, one > own}; }
            }
        };
        consider(0);
        for (int64_t chunk = tiles(R, 64) * 64; chunk >= 4 * kstep; chunk = (chunk / 2 + 63) & ~63LL)
            if ((double)chunk < longest) consider((int32_t)chunk);
    }
    return best;
}
// Parts of an expert's rows there may be.
int64_t most_parts(int64_t R, int64_t E, const GradCut& c) { return E + (c.chunk ? R / c.chunk : 0); }

int64_t up4(int64_t n) { return (n + 3) & ~3LL; }
int64_t rows_partial(const Shape& s, int32_t dtype, int32_t epilogue) {
    const Cut c = cut_rows(s, dtype, epilogue);
    return c.joined ? aligned(c.splits * s.R * up4(s.N) * 4) : 0;
}
constexpr int64_t kMostGroups = 0x7FFFFFFF / 512;
bool rows_fit(const Shape& s, int32_t dtype, int32_t epilogue) {
    const Cut c = cut_rows(s, dtype, epilogue);
    return most_tiles(s, c.tile) * tiles(s.N, c.tile) * c.splits <= kMostGroups;
}
bool grads_fit(const ffn_experts_s* p, int64_t R) {
    const GradCut c = cut_grads(p, R);
    const int64_t di = p->d_in, df = p->d_ff, d_o = p->d_out, E = p->experts, t = c.tile;
    return most_tiles({R, E, di, 0}, c.tile) * tiles(di, t) * c.splits +
               (tiles(2 * df, t) * tiles(di, t) + tiles(d_o, t) * tiles(df, t) + 16) * most_parts(R, E, c) <= kMostGroups;
}

int launch_rows(const ffn::TileArgs& t, const ffn::Groups& g, int32_t epilogue, bool bc, int32_t dtype, int32_t tile, void* stream) {
    switch (dtype) {
        case FFN_FP32: return ffn::launch_expert_rows_fp32(t, g, epilogue, bc, tile, stream);
        case FFN_BF16: return ffn::launch_expert_rows_bf16(t, g, epilogue, bc, tile, stream);
        default: return ffn::launch_expert_rows_fp16(t, g, epilogue, bc, tile, stream);
    }
}
// Runs the product of rows whose operands, sizes (t.M: the sorted rows) and results t describes; `partial` is scratch of
// rows_partial() (kGate: of 2 N columns).
int rows_product(ffn::TileArgs t, ffn::Groups g, int32_t epilogue, bool bc, int32_t dtype, void* partial, void* stream) {
    const int64_t columns = epilogue == ffn::kGate ? 2 * t.N : t.N;
    const Shape s = {t.M, g.experts, columns, t.K};
    const Cut c = cut_rows(s, dtype, epilogue);
    t.tiles_m = (int32_t)most_tiles(s, c.tile);
    t.tiles_n = (int32_t)tiles(columns, c.tile);
    t.splits = c.splits;
    g.deep = dtype != FFN_FP32 && c.tile == 128 && mean_tiles(s, 128) * t.tiles_n * c.splits <= 256.0;
    if (!c.joined) return status(launch_rows(t, g, epilogue, bc, dtype, c.tile, stream));
    ffn::TileArgs p = t;
    p.c = partial;
    p.N = columns;
    p.ldc = up4(columns);
    const int rc = status(launch_rows(p, g, ffn::kPartial, bc, dtype, c.tile, stream));
    if (rc != CGTP_OK) return rc;
    const int32_t* limit = g.offsets + g.experts;
    if (epilogue == ffn::kStore)
        return status(ffn::launch_join_rows((const float*)partial, p.ldc, c.splits, t.M, t.N, t.c, dtype, limit, stream));
    return status(ffn::launch_join_gate_rows(t, epilogue, (const float*)partial, p.ldc, dtype, limit, stream));
}

// The forward products for few rows an expert, where reading the weights is the time: tiles of 16, 32 or 64 rows, so that
// most experts have one; the work-groups are those of all experts with a row.  What a work-group reads of x beside its weight
// rows comes from the L2: 16 weight rows read as much as 16 of x, 32 half of it a weight (64 rows over 16 experts of 4096 values to
// 2048 in bf16: 61 us by 32 weight rows, 79 by 16; 16 rows, 41 by 16 and 63 by 8).  The gate's products hold two of each.
struct Few { int32_t rows, nr, waves; };
Few few_cut(const Shape& s, bool gate, int32_t dtype) {
    const bool wide = dtype == FFN_FP32;
    const int64_t with = s.E < s.R ? s.E : s.R, mean = tiles(s.R, with), all = with * s.N;
    Few c;
    // (64 rows, two of 16 experts each, 2048 x 4096, 16 weight rows a work-group: bf16 168 us by tiles of 32 rows and 198 of 16;
    // fp32 332 by 16, 399 by 32)
    c.rows = mean <= (wide ? 10 : 6) ? 16 : mean <= 24 || wide ? 32 : 64;
    if (all < 16 * 200 || (gate && c.rows == 16 && !wide)) c.nr = 8;
    else c.nr = all >= 32 * 256 && c.rows > 16 ? 32 : 16;
    const int32_t per = (c.nr > 16 ? 2 : 1) * (gate ? 2 : 1) * (c.rows / 16);
    const int64_t blocks = tiles(s.K, wide ? 64 : 128), groups = tiles(all, c.nr);
    // (gated, 64 rows over 8 experts of 1024 x 2048 in bf16: 15.3 us by four waves, 17.3 by eight)
    c.waves = gate && c.nr == 32 ? 4 : 8;
    while (c.waves > 1 && (c.waves * per > 64 || c.waves > 2 * blocks || (c.waves * 4 > blocks && groups * c.waves > 4096))) c.waves /= 2;
    return c;
}
// Whether these kernels are the faster ones, by the mean of an expert's rows.  Against tiles (both products, experts chosen at
// random), 16 experts of 2048 x 4096 in bf16 take 16 us for one choice (28), 159 for 12 rows an expert (207), 188 for 24 (209), 219
// for 32 (209); 8 of 512 x 1024, whose weights the caches hold, 16 for 40 (23), 24 for 64 (24).  Their 16-byte loads to registers
// take longer where 16-bit rows start on 4 bytes (8 experts of 510 x 1022: 17 and 24 by tiles for 24 rows of each, 26 and 24 at
// random; 16 of 2046 x 4094: 165 and 170 for 2, 196 and 185 for 4, 210 and 187 for 10) and twice as long on 2 (511 x 1023: 25 and
// 26 for 24 of each, 39 and 26 at random; 8 of 1023 x 2047: 48 and 38 for one, 68 and 36 for 16), where tiles' direct loads hardly do; so
// each product goes by the alignment of its own rows, of K values.  In fp32 8 of 1024 x 2048 take 78 for 28 (81), 93 for 40 (83), 121
// for 64 (94).
// The mean does not tell how the rows lie.  With half of them on one expert these kernels stay ahead or within 3 % (16 of 2048 x 4096,
// 24 rows an expert: 206 us and 266; 64 of 2048 x 2048: 391 and 380).  With all on one they read its weights again for each tile of
// rows, from the caches, and tiles are ahead from 12 rows an expert on (67 and 66; 24: 113 and 69; of 64 experts 4: 98 and 64, 24:
// 219 and 68).
bool few_rows(int64_t R, const ffn_experts_s* p, int64_t K) {
    const int64_t with = p->experts < R ? p->experts : R, mean = tiles(R, with);
    const bool small = with * p->d_ff * (2 * p->d_in + p->d_out) * size_of(p->dtype) <= (1 << 25);
    if (p->dtype == FFN_FP32) return mean <= 28;
    return mean <= (K % 4 == 0 ? (small ? 48 : 24) : K % 2 == 0 ? (small ? 24 : 10) : small ? 24 : 0);
}
int few_product(ffn::FewArgs p, const ffn::Groups& g, int32_t epilogue, int32_t dtype, void* stream) {
    const bool gate = epilogue == ffn::kGate;
    const Shape s = {g.rows, g.experts, p.N, p.K};
    const Few c = few_cut(s, gate, dtype);
    const int64_t most = most_tiles(s, c.rows);
    switch (dtype) {
        case FFN_FP32: return status(ffn::launch_expert_few_fp32(p, g, epilogue, c.rows, c.nr, c.waves, most, stream));
        case FFN_BF16: return status(ffn::launch_expert_few_bf16(p, g, epilogue, c.rows, c.nr, c.waves, most, stream));
        default: return status(ffn::launch_expert_few_fp16(p, g, epilogue, c.rows, c.nr, c.waves, most, stream));
    }
}

// A matrix as a product reads it: where it is, and behind its last byte that may be read; of the experts' weights, how far
// from its place the last one's is, where that is a copy.
struct Matrix { const void* p; int64_t ld; const void* end; int64_t shift; };

// Direct loads take four bytes at a time: of 16-bit arrays two bytes more than the last value, which are in the array's own
// four where its rows start on four bytes, and else on its page of memory unless the array ends with a page.
bool direct(const void* p, int64_t rows, int64_t ld, int64_t width, int64_t e) {
    return e == 4 || (((uintptr_t)p & 3) == 0 && (ld % 2 == 0 || rows == 1)) || (((uintptr_t)p + ((rows - 1) * ld + width) * e) & 4095) != 0;
}
Matrix matrix(const void* p, int64_t rows, int64_t ld, int64_t width, int64_t e) {
    return {p, ld, (const char*)p + ((rows - 1) * ld + width) * e + (e == 2 ? 2 : 0), 0};
}
// It, or a copy of it in `scratch`.
Matrix readable(const void* p, int64_t rows, int64_t width, int32_t dtype, void* scratch, ffn::PackJobs* jobs) {
    const int64_t e = size_of(dtype);
    if (direct(p, rows, width, width, e)) return matrix(p, rows, width, width, e);
    jobs->job[jobs->n++] = {p, scratch, width, rows, width, up8(width), 0};
    return matrix(scratch, rows, up8(width), width, e);
}
// The experts' weights, of `rows` rows each: only the last one's reach the end of the array, so these alone are copied, as they
// lie, to scratch of weights_bytes().
int64_t weights_bytes(int64_t rows, int64_t width, int32_t dtype) {
    return dtype != FFN_FP32 && width % 2 ? packed_bytes(1, rows * width + 8, dtype) : 0;   // (what is read behind the last value)
}
Matrix weights(const void* p, int64_t E, int64_t rows, int64_t width, int32_t dtype, void* scratch, ffn::PackJobs* jobs) {
    const int64_t e = size_of(dtype), each = rows * width;
    Matrix m = matrix(p, E * rows, width, width, e);
    if (direct(p, E * rows, width, width, e)) return m;
    const char* last = (const char*)p + (E - 1) * each * e;
    jobs->job[jobs->n++] = {last, scratch, each, 1, each, up8(each), 0};
    m.shift = (int64_t)((uintptr_t)scratch - (uintptr_t)last);
    m.end = (const char*)p + E * each * e;   // (rows of small experts before the last are read up to there)
    return m;
}

// Byte offsets in the workspace: x's rows in the sorted order, intermediates, copies of operands, partial sums.  What a call
// needs copied depends on where its arrays lie and on x's stride, which the query does not know.
struct Layout { int64_t x, h, dgu, gy, w_in, w_out, partial, part_in, part_out, total; };
Layout layout(const ffn_experts_s* p, int64_t R, bool backward) {
    const int64_t di = p->d_in, df = p->d_ff, d_o = p->d_out, E = p->experts;
    const int32_t t = p->dtype;
    const bool narrow = t != FFN_FP32;
    Layout l = {};
    int64_t at = 0;
    auto take = [&](int64_t bytes) { const int64_t o = at; at += bytes; return o; };
    // (the kernels for few rows read everything where it is)
    const bool tiled_gate = backward || (R > 0 && !few_rows(R, p, di)), tiled_down = backward || (R > 0 && !few_rows(R, p, df));
    l.x = take(tiled_gate ? packed_bytes(R, di, t) : 0);
    l.h = take(packed_bytes(R, df, t));
    l.w_in = take(tiled_gate ? weights_bytes(2 * df, di, t) : 0);
    l.w_out = take(tiled_down ? weights_bytes(d_o, df, t) : 0);
    int64_t partial = 0;
    auto also = [&](int64_t bytes) { partial = bytes > partial ? bytes : partial; };
    if (backward) {
        l.dgu = take(packed_bytes(R, 2 * df, t));
        l.gy = take(narrow ? packed_bytes(R, d_o, t) : 0);
        also(rows_partial({R, E, df, d_o}, t, ffn::kGateGrad));
        const GradCut c = cut_grads(p, R);
        also(aligned(c.splits * R * up4(di) * 4));
        if (c.chunk) {
            l.part_in = take(aligned(most_parts(R, E, c) * 2 * df * up4(di) * 4));
            l.part_out = take(aligned(most_parts(R, E, c) * d_o * up4(df) * 4));
        }
    } else {
        if (tiled_gate) also(rows_partial({R, E, 2 * df, di}, t, ffn::kGate));
        if (tiled_down) also(rows_partial({R, E, d_o, df}, t, ffn::kStore));
    }
    l.partial = take(partial);
    l.total = at;
    return l;
}

// x's rows in the sorted order, of up8(d_in) values.
int gather(const ffn_experts_s* plan, const void* x, int64_t ldx, const int32_t* place, void* to, int64_t N, int64_t per_row, void* stream) {
    ffn::RouteArgs a = {};
    a.N = N; a.width = plan->d_in; a.per_row = per_row; a.slots = N * per_row;
    a.place = place; a.rows = x; a.ld = ldx;
    a.out_sorted = to; a.ld_sorted = up8(plan->d_in);
    return status(ffn::launch_gather(a, plan->dtype, stream));
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

int ffn_experts_plan(int32_t experts, int64_t d_in, int64_t d_ff, int64_t d_out, int32_t activation, int32_t dtype,
                     ffn_experts_t* plan_out) {
    if (!plan_out || experts < 1 || d_in < 1 || d_ff < 1 || d_out < 1) return CGTP_EINVAL;
    if (activation < FFN_SILU || activation > FFN_RELU) return CGTP_EINVAL;
    if (!known(dtype)) return CGTP_EDTYPE;
    if (experts > FFN_MAX_EXPERTS || d_in > FFN_MAX_WIDTH || d_ff > FFN_MAX_WIDTH || d_out > FFN_MAX_WIDTH) return CGTP_EUNSUP;
    if (experts * 2 * d_ff > FFN_MAX_ROWS || experts * d_out > FFN_MAX_ROWS) return CGTP_EUNSUP;
    int dev = -1;
    const hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return status((int)e);
    ffn_experts_s* p = new (std::nothrow) ffn_experts_s{d_in, d_ff, d_out, experts, activation, dtype, dev};
    if (!p) return CGTP_ENOMEM;
    *plan_out = p;
    return CGTP_OK;
}

int ffn_experts_destroy(ffn_experts_t plan) {
    delete plan;
    return CGTP_OK;
}

int64_t ffn_experts_workspace_bytes(ffn_experts_t plan, int64_t N, int32_t per_row) {
    if (!plan || check_slots(N, per_row, 1) != CGTP_OK) return -1;
    return layout(plan, N * per_row, false).total;
}

int64_t ffn_experts_backward_workspace_bytes(ffn_experts_t plan, int64_t N, int32_t per_row) {
    if (!plan || check_slots(N, per_row, 1) != CGTP_OK) return -1;
    return layout(plan, N * per_row, true).total;
}

int ffn_experts_forward(ffn_experts_t plan, const void* x, int64_t ldx, const int32_t* place, const int32_t* source,
                        const int32_t* offsets, const void* w_in, const void* w_out, void* y, void* saved, int64_t N,
                        int32_t per_row, void* workspace, int64_t workspace_bytes, void* hip_stream) {
    if (!plan) return CGTP_EINVAL;
    int rc = check_slots(N, per_row, 1);
    if (rc != CGTP_OK) return rc;
    if (N == 0) return CGTP_OK;
    const int64_t e = size_of(plan->dtype), di = plan->d_in, df = plan->d_ff, d_o = plan->d_out, E = plan->experts, R = N * per_row;
    const int32_t dt = plan->dtype;
    if (!x || !place || !source || !offsets || !w_in || !w_out || !y || ldx < di) return CGTP_EINVAL;
    if (ldx > kMaxStride) return CGTP_EUNSUP;
    if (misaligned({x}, e) || misaligned({place, source, offsets}, 4) || misaligned({w_in, w_out, y, saved}, 16)) return CGTP_EINVAL;
    if (!rows_fit({R, E, 2 * df, di}, dt, ffn::kGate) || !rows_fit({R, E, d_o, df}, dt, ffn::kStore)) return CGTP_EUNSUP;
    const Layout l = layout(plan, R, false);
    rc = workspace_ok(workspace, workspace_bytes, l.total);
    if (rc != CGTP_OK) return rc;
    const Range ins[] = {rows(x, N, ldx, di, e), {place, R * 4}, {source, R * 4}, {offsets, (E + 1) * 4}, {w_in, E * 2 * df * di * e}, {w_out, E * d_o * df * e}};
    const Range outs[] = {{y, R * d_o * e}, {saved, R * 2 * df * 4}, {workspace, l.total}};
    if (any_overlap(outs, ins)) return CGTP_EINVAL;
    rc = current_device_is(plan->device);
    if (rc != CGTP_OK) return rc;
    char* ws = (char*)workspace;
    const bool few_gate = few_rows(R, plan, di), few_down = few_rows(R, plan, df);
    ffn::PackJobs jobs = {};
    Matrix Wi = {}, Wo = {};
    if (!few_gate) Wi = weights(w_in, E, 2 * df, di, dt, ws + l.w_in, &jobs);
    if (!few_down) Wo = weights(w_out, E, d_o, df, dt, ws + l.w_out, &jobs);
    if (jobs.n) rc = status(ffn::launch_pack(jobs, dt, hip_stream));
    if (rc != CGTP_OK) return rc;
    const Matrix H = matrix(ws + l.h, R, up8(df), df, e);
    if (few_gate) {
        ffn::FewArgs f = {};
        f.x = x; f.ldx = ldx; f.w = w_in; f.ldw = di;
        f.N = df; f.K = di;
        f.c = ws + l.h; f.ldc = H.ld;
        f.saved = (float*)saved; f.act = plan->act;
        rc = few_product(f, {offsets, plan->experts, R, 2 * df * di * e, nullptr, nullptr, 0, 0, source, per_row}, ffn::kGate, dt, hip_stream);
    } else {
        // x's rows where they are, by 32-bit offsets, or copied in the sorted order
        const bool there = direct(x, N, ldx, di, e) && ((N - 1) * ldx + di) * e < (1LL << 31) - 256;
        if (!there) rc = gather(plan, x, ldx, place, ws + l.x, N, per_row, hip_stream);
        if (rc != CGTP_OK) return rc;
        const Matrix X = there ? matrix(x, N, ldx, di, e) : matrix(ws + l.x, R, up8(di), di, e);
        ffn::TileArgs t = {};
        t.a = X.p; t.lda = X.ld;
        t.b = Wi.p; t.ldb = Wi.ld;
        t.M = R; t.N = df; t.K = di;
        t.c = ws + l.h; t.ldc = H.ld;
        t.act = plan->act; t.saved = (float*)saved;
        const ffn::Groups g = {offsets, plan->experts, R, 2 * df * Wi.ld * e, X.end, Wi.end, Wi.shift, 0, there ? source : nullptr, per_row};
        rc = rows_product(t, g, ffn::kGate, false, dt, ws + l.partial, hip_stream);
    }
    if (rc != CGTP_OK) return rc;
    if (few_down) {
        ffn::FewArgs f = {};
        f.x = ws + l.h; f.ldx = H.ld; f.w = w_out; f.ldw = df;
        f.N = d_o; f.K = df;
        f.c = y; f.ldc = d_o;
        return few_product(f, {offsets, plan->experts, R, d_o * df * e, nullptr, nullptr, 0, 0, nullptr, 1}, ffn::kStore, dt, hip_stream);
    }
    ffn::TileArgs o = {};
    o.a = H.p; o.lda = H.ld;
    o.b = Wo.p; o.ldb = Wo.ld;
    o.M = R; o.N = d_o; o.K = df;
    o.c = y; o.ldc = d_o;
    return rows_product(o, {offsets, plan->experts, R, d_o * Wo.ld * e, H.end, Wo.end, Wo.shift, 0, nullptr, 1}, ffn::kStore, false, dt, ws + l.partial, hip_stream);
}

int ffn_experts_backward(ffn_experts_t plan, const void* x, int64_t ldx, const int32_t* place, const int32_t* source,
                         const int32_t* offsets, const void* w_in, const void* w_out, const void* saved,
                         const void* grad_y, void* grad_x, void* grad_w_in, void* grad_w_out, int64_t N,
                         int32_t per_row, void* workspace, int64_t workspace_bytes, void* hip_stream) {
    if (!plan) return CGTP_EINVAL;
    int rc = check_slots(N, per_row, 1);
    if (rc != CGTP_OK) return rc;
    if (N == 0 && !grad_w_in && !grad_w_out) return CGTP_OK;   // (an empty grad_x may be NULL)
    if (!grad_x && !grad_w_in && !grad_w_out) return CGTP_EINVAL;
    const int64_t e = size_of(plan->dtype), di = plan->d_in, df = plan->d_ff, d_o = plan->d_out, E = plan->experts, R = N * per_row;
    const int32_t dt = plan->dtype;
    if (N > 0 && (!x || !place || !source || !offsets || !w_in || !w_out || !saved || !grad_y || ldx < di)) return CGTP_EINVAL;
    if (ldx > kMaxStride) return CGTP_EUNSUP;
    if (misaligned({x, grad_y}, e) || misaligned({place, source, offsets}, 4) ||
        misaligned({w_in, w_out, saved, grad_x, grad_w_in, grad_w_out}, 16))
        return CGTP_EINVAL;
    if (!rows_fit({R, E, df, d_o}, dt, ffn::kGateGrad) || !grads_fit(plan, R)) return CGTP_EUNSUP;
    const Layout l = layout(plan, R, true);
    rc = workspace_ok(workspace, workspace_bytes, l.total);
    if (rc != CGTP_OK) return rc;
    const Range ins[] = {rows(x, N, ldx, di, e), {place, R * 4}, {source, R * 4}, {offsets, (E + 1) * 4}, {w_in, E * 2 * df * di * e}, {w_out, E * d_o * df * e},
                         {saved, R * 2 * df * 4}, {grad_y, R * d_o * e}};
    const Range outs[] = {{grad_x, N * di * e}, {grad_w_in, E * 2 * df * di * e}, {grad_w_out, E * d_o * df * e}, {workspace, l.total}};
    if (any_overlap(outs, ins)) return CGTP_EINVAL;
    rc = current_device_is(plan->device);
    if (rc != CGTP_OK) return rc;
    if (N == 0) {
        // sums over no rows
        if (grad_w_in) rc = status(ffn::launch_zero(grad_w_in, E * 2 * df * di * e, hip_stream));
        if (rc == CGTP_OK && grad_w_out) rc = status(ffn::launch_zero(grad_w_out, E * d_o * df * e, hip_stream));
        return rc;
    }
    char* ws = (char*)workspace;
    ffn::PackJobs jobs = {};
    const Matrix Gy = readable(grad_y, R, d_o, dt, ws + l.gy, &jobs), Wo = weights(w_out, E, d_o, df, dt, ws + l.w_out, &jobs);
    Matrix Wi = {};
    if (grad_x) Wi = weights(w_in, E, 2 * df, di, dt, ws + l.w_in, &jobs);
    rc = status(ffn::launch_pack(jobs, dt, hip_stream));
    if (rc == CGTP_OK && grad_w_in) rc = gather(plan, x, ldx, place, ws + l.x, N, per_row, hip_stream);
    if (rc != CGTP_OK) return rc;
    const Matrix H = matrix(ws + l.h, R, up8(df), df, e), D = matrix(ws + l.dgu, R, up8(2 * df), 2 * df, e), X = matrix(ws + l.x, R, up8(di), di, e);
    ffn::Groups g = {offsets, plan->experts, R, d_o * Wo.ld * e, Gy.end, Wo.end, Wo.shift, 0, nullptr, 1};
    ffn::TileArgs t = {};
    t.a = Gy.p; t.lda = Gy.ld;
    t.b = Wo.p; t.ldb = Wo.ld;
    t.M = R; t.N = df; t.K = d_o;
    t.c = ws + l.dgu; t.ldc = D.ld;
    t.h = ws + l.h; t.ldh = H.ld;
    t.act = plan->act; t.saved = (float*)const_cast<void*>(saved);
    rc = rows_product(t, g, ffn::kGateGrad, true, dt, ws + l.partial, hip_stream);
    if (rc != CGTP_OK) return rc;
    const GradCut c = cut_grads(plan, R);
    ffn::ExpertGrads a = {};
    for (int k = 0; k < 3; ++k) a.order[k] = c.sums_first ? (k + 1) % 3 : k;
    auto sums = [&](int k, const Matrix& A, const Matrix& B, int64_t M, int64_t columns, void* to, int64_t part) {
        ffn::TileArgs& w = a.t[k];
        w.a = A.p; w.lda = A.ld; w.b = B.p; w.ldb = B.ld;
        w.M = M; w.N = columns; w.c = to; w.ldc = columns;
        w.tiles_m = (int32_t)tiles(M, c.tile);
        w.tiles_n = (int32_t)tiles(columns, c.tile);
        w.splits = (int32_t)most_parts(R, E, c);
        a.g[k] = {offsets, plan->experts, R, 0, A.end, B.end, 0, c.chunk, nullptr, 1};
        a.partial[k - 1] = (float*)(ws + part);
    };
    if (grad_x) {
        // its sums stay in 32 bits until a row's choices are added
        ffn::TileArgs& d = a.t[0];
        d.a = D.p; d.lda = D.ld; d.b = Wi.p; d.ldb = Wi.ld;
        d.M = R; d.N = di; d.K = 2 * df;
        d.c = ws + l.partial; d.ldc = up4(di);
        d.tiles_m = (int32_t)most_tiles({R, E, di, 0}, c.tile);
        d.tiles_n = (int32_t)tiles(di, c.tile);
        d.splits = c.splits;
        a.g[0] = {offsets, plan->experts, R, 2 * df * Wi.ld * e, D.end, Wi.end, Wi.shift, 0, nullptr, 1};
    }
    if (grad_w_in) sums(1, D, X, 2 * df, di, grad_w_in, l.part_in);
    if (grad_w_out) sums(2, Gy, H, d_o, df, grad_w_out, l.part_out);
    rc = status(dt == FFN_FP32   ? ffn::launch_expert_grads_fp32(a, c.tile, hip_stream)
                : dt == FFN_BF16 ? ffn::launch_expert_grads_bf16(a, c.tile, hip_stream)
                                 : ffn::launch_expert_grads_fp16(a, c.tile, hip_stream));
    if (rc == CGTP_OK && grad_x) {
        ffn::RouteArgs r = {};
        r.N = N; r.width = di; r.per_row = per_row; r.slots = R;
        r.place = place; r.sorted = ws + l.partial; r.out_rows = grad_x; r.ld_out = di;
        rc = status(ffn::launch_combine_parts(r, c.splits, dt, hip_stream));
    }
    if (rc == CGTP_OK && c.chunk && (grad_w_in || grad_w_out)) rc = status(ffn::launch_join_sums(a, dt, hip_stream));
    return rc;
}

}  // extern "C"
