// The host code of the experts' operators and of the layer norm (experts_plan.cpp, ffn_layer.cpp: checks, workspace
// layouts, cutting of the products, order of the launches) under ASan/UBSan without a GPU.  The launchers are stand-ins
// that do on the host what a launch is asked for, plainly.  Arrays are as long as the headers say and the workspace as the
// query says, filled with NaN before every call, so a wrong offset, stride, size or order ends the run or shows in the
// results, which are held against the definitions in 64 bits.  16-bit arrays are bf16 here, cut off.
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <limits>
#include <vector>

#include "../../paper_2602_21466_amd/csrc/cgtp_internal.h"
#include "../../paper_2602_21466_amd/csrc/experts_internal.h"

static int fails = 0, launches = 0, parts_seen = 0, few_seen = 0, deep_seen = 0;
#define EXPECT(cond)                                                \
    do {                                                            \
        if (!(cond)) {                                              \
            std::printf("FAILED %s at line %d\n", #cond, __LINE__); \
            ++fails;                                                \
        }                                                           \
    } while (0)

extern "C" hipError_t hipGetDevice(int* d) {
    *d = 0;
    return hipSuccess;
}
namespace cgtp {
void set_last_hip_error(int) {}
}

struct F32 {
    static constexpr int size = 4;
    static double get(const void* p, int64_t i) {
        float f;
        std::memcpy(&f, (const char*)p + 4 * i, 4);
        return f;
    }
    static void put(void* p, int64_t i, double v) {
        const float f = (float)v;
        std::memcpy((char*)p + 4 * i, &f, 4);
    }
};
struct B16 {
    static constexpr int size = 2;
    static double get(const void* p, int64_t i) {
        uint16_t h;
        std::memcpy(&h, (const char*)p + 2 * i, 2);
        const uint32_t u = (uint32_t)h << 16;
        float f;
        std::memcpy(&f, &u, 4);
        return f;
    }
    static void put(void* p, int64_t i, double v) {
        const float f = (float)v;
        uint32_t u;
        std::memcpy(&u, &f, 4);
        const uint16_t h = (uint16_t)(u >> 16);
        std::memcpy((char*)p + 2 * i, &h, 2);
    }
};

static double act(int a, double g) { return a == FFN_RELU ? std::fmax(g, 0.0) : a == FFN_SILU ? g / (1 + std::exp(-g)) : 0.5 * g * (1 + std::erf(g * std::sqrt(0.5))); }
static double dact(int a, double g) {
    if (a == FFN_RELU) return g > 0;
    if (a == FFN_SILU) { const double s = 1 / (1 + std::exp(-g)); return s * (1 + g * (1 - s)); }
    return 0.5 * (1 + std::erf(g * std::sqrt(0.5))) + g * std::exp(-0.5 * g * g) * 0.3989422804014327;
}

// ---------------------------------------------------------------- launches

template <typename T> void finish(const ffn::TileArgs& t, int epi, int64_t m, int64_t n, double v, double u) {
    if (epi == ffn::kStore) { T::put(t.c, m * t.ldc + n, v); return; }
    if (epi == ffn::kGate) {
        T::put(t.c, m * t.ldc + n, act(t.act, v) * u);
        if (t.saved) { t.saved[m * 2 * t.N + n] = (float)v; t.saved[m * 2 * t.N + t.N + n] = (float)u; }
        return;
    }
    const double g = t.saved[m * 2 * t.N + n], up = t.saved[m * 2 * t.N + t.N + n];
    T::put(t.c, m * t.ldc + n, v * up * dact(t.act, g));
    T::put(t.c, m * t.ldc + t.N + n, v * act(t.act, g));
    T::put(t.h, m * t.ldh + n, act(t.act, g) * up);
}

// The last byte that may be read is the array's own (two more of 16-bit arrays, which are the last value's four).
template <typename T> void last(const void* end) {
    volatile char c = *((const char*)end - (T::size == 2 ? 2 : 0) - 1);
    (void)c;
}

template <typename T> int rows_launch(const ffn::TileArgs& t, const ffn::Groups& g, int epi, bool bc, int side) {
    ++launches;
    deep_seen += g.deep;
    EXPECT(side == 128 || side == 256);
    EXPECT(t.M == g.rows && t.K >= 1);
    const int64_t brows = epi == ffn::kGate ? 2 * t.N : t.N, step = 128 / T::size, steps = (t.K + step - 1) / step;
    EXPECT(t.tiles_n == (brows + side - 1) / side && (epi == ffn::kPartial || t.splits == 1));
    int64_t tiles = 0;
    for (int e = 0; e < g.experts; ++e) tiles += (g.offsets[e + 1] - g.offsets[e] + side - 1) / side;
    EXPECT(tiles <= t.tiles_m && (int64_t)t.tiles_m * t.tiles_n * t.splits <= 0x7FFFFFFF / 512);
    last<T>(g.a_end);
    last<T>(g.b_end);
    for (int e = 0; e < g.experts; ++e)
        for (int64_t m = g.offsets[e]; m < g.offsets[e + 1]; ++m) {
            const char* b = (const char*)t.b + e * g.b_step;
            const int64_t row = g.source ? g.source[m] / g.per_row : m;
            auto sum = [&](int64_t n, int64_t k0, int64_t k1) {
                double v = 0;
                for (int64_t k = k0; k < k1 && k < t.K; ++k) v += T::get(t.a, row * t.lda + k) * T::get(b, bc ? k * t.ldb + n : n * t.ldb + k);
                return v;
            };
            for (int64_t n = 0; n < t.N; ++n) {
                if (epi == ffn::kPartial)
                    for (int64_t s = 0; s < t.splits; ++s)
                        ((float*)t.c)[(s * t.M + m) * t.ldc + n] = (float)sum(n, steps * s / t.splits * step, steps * (s + 1) / t.splits * step);
                else finish<T>(t, epi, m, n, sum(n, 0, t.K), epi == ffn::kGate ? sum(t.N + n, 0, t.K) : 0);
            }
        }
    return 0;
}

template <typename T> int few_launch(const ffn::FewArgs& p, const ffn::Groups& g, int epi, int rows, int nr, int waves, int64_t most) {
    ++launches;
    ++few_seen;
    const bool gate = epi == ffn::kGate;
    const int mt = rows / 16;
    EXPECT((rows == 16 || rows == 32 || (rows == 64 && T::size == 2)) && (epi == ffn::kStore || gate));
    EXPECT(nr == 8 || (nr == 16 && (mt > 1 || T::size == 4 || !gate)) || (nr == 32 && mt > 1));
    EXPECT(waves >= 1 && waves <= 8 && waves * (nr > 16 ? 2 : 1) * (gate ? 2 : 1) * mt <= 64 && most <= 65535);
    int64_t tiles = 0;
    for (int e = 0; e < g.experts; ++e) tiles += (g.offsets[e + 1] - g.offsets[e] + rows - 1) / rows;
    EXPECT(tiles <= most);
    ffn::TileArgs t = {};
    t.N = p.N; t.act = p.act; t.c = p.c; t.ldc = p.ldc; t.saved = p.saved;
    for (int e = 0; e < g.experts; ++e)
        for (int64_t m = g.offsets[e]; m < g.offsets[e + 1]; ++m) {
            const int64_t row = g.source ? g.source[m] / g.per_row : m;
            const char* w = (const char*)p.w + e * g.b_step;
            for (int64_t n = 0; n < p.N; ++n) {
                double v = 0, u = 0;
                for (int64_t k = 0; k < p.K; ++k) {
                    v += T::get(p.x, row * p.ldx + k) * T::get(w, n * p.ldw + k);
                    if (gate) u += T::get(p.x, row * p.ldx + k) * T::get(w, (p.N + n) * p.ldw + k);
                }
                finish<T>(t, epi, m, n, v, u);
                if (gate && n == p.N - 1) for (int64_t c = p.N; c < p.ldc; ++c) T::put(p.c, m * p.ldc + c, 0);
            }
        }
    return 0;
}

template <typename T> int grads_launch(const ffn::ExpertGrads& a, int side) {
    int seen = 0;
    for (int k : {0, 1, 2}) seen |= 1 << a.order[k];
    EXPECT(seen == 7);
    if (a.t[0].a) rows_launch<T>(a.t[0], a.g[0], ffn::kPartial, true, side);
    ++launches;
    for (int k : {1, 2}) {
        const ffn::TileArgs& t = a.t[k];
        const ffn::Groups& g = a.g[k];
        if (!t.a) continue;
        last<T>(g.a_end);
        last<T>(g.b_end);
        EXPECT(t.tiles_m == (t.M + side - 1) / side && t.tiles_n == (t.N + side - 1) / side);
        int64_t unit = 0;
        const int64_t ld = (t.N + 3) & ~3LL;
        for (int e = 0; e < g.experts; ++e) {
            const int64_t b = g.offsets[e], end = g.offsets[e + 1], n = g.chunk && end - b > g.chunk ? (end - b + g.chunk - 1) / g.chunk : 1;
            for (int64_t part = 0; part < n; ++part, ++unit) {
                const int64_t r0 = n > 1 ? b + part * g.chunk : b, r1 = n > 1 && r0 + g.chunk < end ? r0 + g.chunk : end;
                parts_seen += n > 1;
                for (int64_t i = 0; i < t.M; ++i)
                    for (int64_t j = 0; j < t.N; ++j) {
                        double v = 0;
                        for (int64_t r = r0; r < r1; ++r) v += T::get(t.a, r * t.lda + i) * T::get(t.b, r * t.ldb + j);
                        if (n > 1) a.partial[k - 1][(unit * t.M + i) * ld + j] = (float)v;
                        else T::put(t.c, (e * t.M + i) * t.ldc + j, v);
                    }
            }
        }
        EXPECT(unit <= t.splits);
    }
    return 0;
}

template <typename T> int join_sums(const ffn::ExpertGrads& a) {
    ++launches;
    for (int k : {1, 2}) {
        const ffn::TileArgs& t = a.t[k];
        const ffn::Groups& g = a.g[k];
        if (!t.a) continue;
        int64_t unit = 0;
        const int64_t ld = (t.N + 3) & ~3LL;
        for (int e = 0; e < g.experts; ++e) {
            const int64_t rows = g.offsets[e + 1] - g.offsets[e], n = rows > g.chunk ? (rows + g.chunk - 1) / g.chunk : 1;
            if (n > 1)
                for (int64_t i = 0; i < t.M; ++i)
                    for (int64_t j = 0; j < t.N; ++j) {
                        double v = 0;
                        for (int64_t s = 0; s < n; ++s) v += a.partial[k - 1][((unit + s) * t.M + i) * ld + j];
                        T::put(t.c, (e * t.M + i) * t.N + j, v);
                    }
            unit += n;
        }
    }
    return 0;
}

template <typename T> int gather(const ffn::RouteArgs& a) {
    ++launches;
    for (int64_t n = 0; n < a.N; ++n)
        for (int64_t k = 0; k < a.per_row; ++k) {
            const int64_t p = a.place[n * a.per_row + k];
            for (int64_t c = 0; p >= 0 && c < a.ld_sorted; ++c) T::put(a.out_sorted, p * a.ld_sorted + c, c < a.width ? T::get(a.rows, n * a.ld + c) : 0);
        }
    if (a.offsets)
        for (int64_t p = a.offsets[a.experts]; p < a.slots; ++p)
            for (int64_t c = 0; c < a.ld_sorted; ++c) T::put(a.out_sorted, p * a.ld_sorted + c, 0);
    return 0;
}
template <typename T> int combine(const ffn::RouteArgs& a) {
    ++launches;
    for (int64_t n = 0; n < a.N; ++n)
        for (int64_t c = 0; c < a.width; ++c) {
            double v = 0;
            for (int64_t k = 0; k < a.per_row; ++k) {
                const int64_t s = n * a.per_row + k;
                if (a.place[s] >= 0) v += (a.weights ? a.weights[s] : 1.0) * T::get(a.sorted, a.place[s] * a.width + c);
            }
            T::put(a.out_rows, n * a.ld_out + c, v);
        }
    return 0;
}
template <typename T> int combine_backward(const ffn::RouteArgs& a) {
    ++launches;
    for (int64_t s = 0; s < a.slots; ++s) {
        double dot = 0;
        for (int64_t c = 0; a.place[s] >= 0 && c < a.width; ++c) {
            const double g = T::get(a.rows, s / a.per_row * a.ld + c);
            if (a.grad_weights) dot += g * T::get(a.sorted, a.place[s] * a.width + c);
            if (a.out_sorted) T::put(a.out_sorted, a.place[s] * a.ld_sorted + c, (a.weights ? a.weights[s] : 1.0) * g);
        }
        if (a.grad_weights) a.grad_weights[s] = (float)dot;
    }
    if (a.out_sorted)
        for (int64_t p = a.offsets[a.experts]; p < a.slots; ++p)
            for (int64_t c = 0; c < a.width; ++c) T::put(a.out_sorted, p * a.ld_sorted + c, 0);
    return 0;
}

static void touch(const void* p, int64_t rows, int64_t ld, int64_t width, int size, bool write) {
    if (!p) return;
    volatile unsigned char sink = 0;
    for (int64_t r = 0; r < rows; ++r) {
        char* row = (char*)p + r * ld * size;
        if (write) std::memset(row, 0, width * size);
        else for (int64_t c = 0; c < width * size; ++c) sink = sink + (unsigned char)row[c];
    }
}
static int layer(const ffn::LayerArgs& a, int size, bool backward) {
    ++launches;
    const int64_t D = a.width;
    touch(a.x, a.N, a.ldx, D, size, false);
    for (const void* p : {a.w, a.b}) touch(p, 1, D, D, size, false);
    touch(a.stats, 2, a.N, a.N, 4, !backward);
    touch(a.u, a.N, a.ldu, D, size, true);
    touch(a.gu, a.N, a.ldg, D, size, false);
    touch(a.gx, a.N, D, D, size, true);
    for (void* p : {a.gw, a.gb}) touch(p, 1, D, D, size, true);
    if (backward) touch(a.partial, 1, 0, ffn::layer_workspace_floats(D, a.N, size), 4, true);
    return 0;
}

namespace ffn {
#define BY_TYPE(NAME, PARAMS, CALL)               \
    int NAME##_fp32 PARAMS { return CALL(F32); }  \
    int NAME##_bf16 PARAMS { return CALL(B16); }  \
    int NAME##_fp16 PARAMS { return CALL(B16); }
#define ROWS(T) rows_launch<T>(t, g, e, b, side)
BY_TYPE(launch_expert_rows, (const TileArgs& t, const Groups& g, int32_t e, bool b, int32_t side, void*), ROWS)
#define FEW(T) few_launch<T>(p, g, e, rows, nr, waves, most)
BY_TYPE(launch_expert_few, (const FewArgs& p, const Groups& g, int32_t e, int32_t rows, int32_t nr, int32_t waves, int64_t most, void*), FEW)
#define GRADS(T) grads_launch<T>(a, side)
BY_TYPE(launch_expert_grads, (const ExpertGrads& a, int32_t side, void*), GRADS)
#define LF(T) layer(a, T::size, false)
BY_TYPE(launch_layer_forward, (const LayerArgs& a, void*), LF)
#define LB(T) layer(a, T::size, true)
BY_TYPE(launch_layer_backward, (const LayerArgs& a, void*), LB)
// (any number that the caller cannot know: the launch writes all of it)
int64_t layer_workspace_floats(int64_t width, int64_t N, int bytes) { return 2 * width + N % 5 + bytes; }

#define OF_TYPE(CALL) dtype == FFN_FP32 ? CALL<F32> : CALL<B16>
int launch_join_sums(const ExpertGrads& a, int32_t dtype, void*) { return (OF_TYPE(join_sums))(a); }
int launch_gather(const RouteArgs& a, int32_t dtype, void*) { return (OF_TYPE(gather))(a); }
int launch_combine(const RouteArgs& a, int32_t dtype, void*) { return (OF_TYPE(combine))(a); }
int launch_combine_backward(const RouteArgs& a, int32_t dtype, void*) { return (OF_TYPE(combine_backward))(a); }
int launch_combine_parts(const RouteArgs& a, int32_t splits, int32_t dtype, void*) {
    ++launches;
    const int64_t ld = (a.width + 3) & ~3LL;
    for (int64_t n = 0; n < a.N; ++n)
        for (int64_t c = 0; c < a.width; ++c) {
            double v = 0;
            for (int64_t k = 0; k < a.per_row; ++k)
                for (int64_t s = 0; a.place[n * a.per_row + k] >= 0 && s < splits; ++s)
                    v += ((const float*)a.sorted)[(s * a.slots + a.place[n * a.per_row + k]) * ld + c];
            if (dtype == FFN_FP32) F32::put(a.out_rows, n * a.ld_out + c, v);
            else B16::put(a.out_rows, n * a.ld_out + c, v);
        }
    return 0;
}
int launch_join_rows(const float* from, int64_t ld, int32_t splits, int64_t M, int64_t N, void* out, int32_t dtype, const int32_t* limit, void*) {
    ++launches;
    for (int64_t m = 0; m < (limit ? *limit : M); ++m)
        for (int64_t n = 0; n < N; ++n) {
            double v = 0;
            for (int s = 0; s < splits; ++s) v += from[(s * M + m) * ld + n];
            if (dtype == FFN_FP32) F32::put(out, m * N + n, v);
            else B16::put(out, m * N + n, v);
        }
    return 0;
}
int launch_join_gate_rows(const TileArgs& t, int32_t epi, const float* from, int64_t ld, int32_t dtype, const int32_t* limit, void*) {
    ++launches;
    for (int64_t m = 0; m < (limit ? *limit : t.M); ++m)
        for (int64_t n = 0; n < t.N; ++n) {
            double v = 0, u = 0;
            for (int s = 0; s < t.splits; ++s) {
                v += from[(s * t.M + m) * ld + n];
                if (epi == kGate) u += from[(s * t.M + m) * ld + t.N + n];
            }
            if (dtype == FFN_FP32) finish<F32>(t, epi, m, n, v, u);
            else finish<B16>(t, epi, m, n, v, u);
        }
    return 0;
}
int launch_pack(PackJobs jobs, int32_t dtype, void*) {
    EXPECT(jobs.n >= 0 && jobs.n <= 4);
    for (int j = 0; j < jobs.n; ++j) {
        const PackJob& q = jobs.job[j];
        for (int64_t r = 0; r < q.rows; ++r)
            for (int64_t c = 0; c < q.to_ld; ++c) {
                if (dtype == FFN_FP32) F32::put(q.to, r * q.to_ld + c, c < q.width ? F32::get(q.from, r * q.ld + c) : 0);
                else B16::put(q.to, r * q.to_ld + c, c < q.width ? B16::get(q.from, r * q.ld + c) : 0);
            }
    }
    return 0;
}
int launch_zero(void* p, int64_t bytes, void*) {
    std::memset(p, 0, bytes);
    return 0;
}
int launch_sort(const SortArgs& a, void*) {
    ++launches;
    EXPECT(a.groups * a.chunk >= a.slots && (a.groups == 1 || (a.groups - 1) * a.chunk < a.slots));
    if (a.groups > 1) std::memset(a.counts, 0, (size_t)a.groups * a.experts * 4);
    int32_t at = 0;
    for (int64_t s = 0; s < a.slots; ++s) a.place[s] = a.source[s] = -1;
    for (int e = 0; e < a.experts; ++e) {
        a.offsets[e] = at;
        for (int64_t s = 0; s < a.slots; ++s) {
            const int64_t v = a.index_bytes == 8 ? ((const int64_t*)a.index)[s] : ((const int32_t*)a.index)[s];
            if (v != e) continue;
            a.place[s] = at;
            a.source[at++] = (int32_t)s;
        }
    }
    a.offsets[a.experts] = at;
    return 0;
}
}  // namespace ffn

// ---------------------------------------------------------------- arrays

// Rows `ld` apart, from `off` elements behind a 256-byte boundary, exactly as long as they have to be; with `page`, ending
// where a page of memory ends.
template <typename T> struct Array {
    char* base = nullptr;
    void* p = nullptr;
    int64_t rows, width, ld;
    Array(int64_t rows, int64_t width, int64_t ld = 0, int64_t off = 0) : rows(rows), width(width), ld(ld ? ld : width) {
        const int64_t bytes = (off + (rows > 0 ? (rows - 1) * this->ld + width : 0)) * T::size;
        if (posix_memalign((void**)&base, 256, bytes ? bytes : 1)) std::abort();
        p = base + off * T::size;
        for (int64_t i = 0; i < bytes / T::size; ++i) T::put(base, i, std::numeric_limits<double>::quiet_NaN());
    }
    Array(const Array&) = delete;
    ~Array() { std::free(base); }
    double at(int64_t r, int64_t c) const { return T::get(p, r * ld + c); }
    void draw(uint32_t seed, double size) {
        uint32_t x = seed * 2654435761u + 1;
        for (int64_t r = 0; r < rows; ++r)
            for (int64_t c = 0; c < width; ++c) {
                x = x * 1664525u + 1013904223u;
                T::put(p, r * ld + c, ((int32_t)x / 2147483648.0) * size);
            }
    }
};

template <typename T> bool near(const Array<T>& got, const std::vector<double>& want, double tol, int64_t rows = -1) {
    double d = 0, w = 0;
    for (int64_t r = 0; r < (rows < 0 ? got.rows : rows); ++r)
        for (int64_t c = 0; c < got.width; ++c) {
            const double e = got.at(r, c) - want[r * got.width + c];
            d += e * e;
            w += want[r * got.width + c] * want[r * got.width + c];
        }
    if (!(d <= tol * tol * w)) std::printf("  off by %.3g\n", std::sqrt(d / w));
    return d <= tol * tol * w;
}

// kind: 0 even, 1 some choices of no expert, 2 all of one expert, 3 none
template <typename T> void experts(int dtype, int64_t N, int K, int E, int64_t di, int64_t df, int64_t d_o, int act_, int kind, int64_t gap, int64_t off) {
    const int64_t S = N * K;
    std::vector<int64_t> index(S);
    uint32_t r = (uint32_t)(N * 31 + K * 7 + E);
    for (int64_t s = 0; s < S; ++s) {
        r = r * 1664525u + 1013904223u;
        index[s] = kind == 2 ? E - 1 : kind == 3 ? -1 : (int64_t)((r >> 8) % (uint32_t)E);
        if (kind == 1 && (r >> 4) % 3 == 0) index[s] = (r & 1) ? -5 : E + 3;
    }
    std::vector<int32_t> place(S), source(S), offsets(E + 1);
    {
        const int64_t need = ffn_route_workspace_bytes(N, K, E);
        Array<F32> ws(1, need / 4);
        EXPECT(ffn_route(index.data(), 8, N, K, E, place.data(), source.data(), offsets.data(), need ? ws.p : nullptr, need, nullptr) == CGTP_OK);
        if (need) EXPECT(ffn_route(index.data(), 8, N, K, E, place.data(), source.data(), offsets.data(), ws.p, need - 1, nullptr) == CGTP_EINVAL);
    }
    const int64_t M = offsets[E];
    ffn_experts_t plan = nullptr;
    EXPECT(ffn_experts_plan(E, di, df, d_o, act_, dtype, &plan) == CGTP_OK && plan);
    Array<T> x(N, di, di + gap, off), wi(E * 2 * df, di), wo(E * d_o, df), gy(S, d_o, 0, off), y(S, d_o), gx(N, di), gwi(E * 2 * df, di), gwo(E * d_o, df);
    Array<F32> saved(S, 2 * df);
    x.draw(1, 1); wi.draw(2, 1.5 / std::sqrt((double)di)); wo.draw(3, 1.5 / std::sqrt((double)df)); gy.draw(4, 1);
    std::vector<double> want(S * d_o), wx(N * di), wwi(E * 2 * df * di), wwo(E * d_o * df);
    for (int e = 0; e < E; ++e)
        for (int64_t p = offsets[e]; p < offsets[e + 1]; ++p) {
            const int64_t n = source[p] / K;
            for (int64_t j = 0; j < df; ++j) {
                double g = 0, u = 0, dh = 0;
                for (int64_t k = 0; k < di; ++k) {
                    g += x.at(n, k) * wi.at(e * 2 * df + j, k);
                    u += x.at(n, k) * wi.at(e * 2 * df + df + j, k);
                }
                const double h = act(act_, g) * u;
                for (int64_t o = 0; o < d_o; ++o) {
                    want[p * d_o + o] += h * wo.at(e * d_o + o, j);
                    dh += gy.at(p, o) * wo.at(e * d_o + o, j);
                    wwo[(e * d_o + o) * df + j] += gy.at(p, o) * h;
                }
                const double dg = dh * u * dact(act_, g), du = dh * act(act_, g);
                for (int64_t k = 0; k < di; ++k) {
                    wx[n * di + k] += dg * wi.at(e * 2 * df + j, k) + du * wi.at(e * 2 * df + df + j, k);
                    wwi[(e * 2 * df + j) * di + k] += dg * x.at(n, k);
                    wwi[(e * 2 * df + df + j) * di + k] += du * x.at(n, k);
                }
            }
        }
    const double tol = T::size == 4 ? 1e-5 : 5e-2;
    for (int save = 0; save < 2; ++save) {
        const int64_t need = ffn_experts_workspace_bytes(plan, N, K);
        EXPECT(need >= 0 && need % 256 == 0);
        Array<F32> ws(1, need / 4);
        EXPECT(ffn_experts_forward(plan, x.p, x.ld, place.data(), source.data(), offsets.data(), wi.p, wo.p, y.p, save ? saved.p : nullptr, N, K, ws.p, need, nullptr) == CGTP_OK);
        EXPECT(near(y, want, tol, M));
        for (int64_t p = M; p < S; ++p) EXPECT(std::isnan(y.at(p, 0)));   // left as they were
        EXPECT(ffn_experts_forward(plan, x.p, x.ld, place.data(), source.data(), offsets.data(), wi.p, wo.p, y.p, nullptr, N, K, ws.p, need - 1, nullptr) == CGTP_EINVAL);
        EXPECT(ffn_experts_forward(plan, x.p, x.ld, place.data(), source.data(), offsets.data(), wi.p, wo.p, wi.p, nullptr, N, K, ws.p, need, nullptr) == CGTP_EINVAL);
    }
    for (int which = 1; which < 8; ++which) {
        const int64_t need = ffn_experts_backward_workspace_bytes(plan, N, K);
        Array<F32> ws(1, need / 4);
        EXPECT(ffn_experts_backward(plan, x.p, x.ld, place.data(), source.data(), offsets.data(), wi.p, wo.p, saved.p, gy.p, which & 1 ? gx.p : nullptr,
                                    which & 2 ? gwi.p : nullptr, which & 4 ? gwo.p : nullptr, N, K, ws.p, need, nullptr) == CGTP_OK);
        if (which & 1) EXPECT(near(gx, wx, tol));
        if (which & 2) EXPECT(near(gwi, wwi, tol));
        if (which & 4) EXPECT(near(gwo, wwo, tol));
    }
    // rows there and back
    Array<T> xs(S, di), back(N, di, di + gap, off), gs(S, di);
    Array<F32> w(1, S), gw(1, S);
    w.draw(9, 1);
    EXPECT(ffn_route_gather(x.p, x.ld, place.data(), offsets.data(), xs.p, N, K, E, di, dtype, nullptr) == CGTP_OK);
    EXPECT(ffn_route_combine(xs.p, place.data(), (float*)w.p, back.p, back.ld, N, K, di, dtype, nullptr) == CGTP_OK);
    EXPECT(ffn_route_combine_backward(xs.p, place.data(), offsets.data(), (float*)w.p, x.p, x.ld, gs.p, (float*)gw.p, N, K, E, di, dtype, nullptr) == CGTP_OK);
    std::vector<double> wb(N * di), wgw(S);
    for (int64_t s = 0; s < S; ++s)
        for (int64_t c = 0; place[s] >= 0 && c < di; ++c) {
            wb[s / K * di + c] += w.at(0, s) * x.at(s / K, c);
            wgw[s] += x.at(s / K, c) * x.at(s / K, c);
        }
    EXPECT(near(back, wb, tol) && near(gw, wgw, tol));
    for (int64_t p = M; p < S; ++p) EXPECT(xs.at(p, 0) == 0 && gs.at(p, di - 1) == 0);
    ffn_experts_destroy(plan);
}

template <typename T> void layers(int dtype, int64_t N, int64_t D, int64_t gap) {
    ffn_norm n{D, 1, dtype, 1e-6f, 0.0, 0, 0};
    Array<T> x(N, D, D + gap, 1), u(N, D, D + 2 * gap, 3), gu(N, D, D + gap, 1), w(1, D), b(1, D), gx(N, D), gw(1, D), gb(1, D);
    Array<F32> stats(2, N);
    EXPECT(ffn_layer_forward(&n, x.p, x.ld, w.p, b.p, u.p, u.ld, (float*)stats.p, N, nullptr) == CGTP_OK);
    EXPECT(ffn_layer_forward(&n, x.p, x.ld, w.p, nullptr, x.p, x.ld, nullptr, N, nullptr) == CGTP_OK);
    const int64_t need = ffn_layer_workspace_bytes(&n, N);
    Array<F32> ws(1, need / 4);
    EXPECT(ffn_layer_backward(&n, x.p, x.ld, w.p, (float*)stats.p, gu.p, gu.ld, gx.p, gw.p, gb.p, N, ws.p, need, nullptr) == CGTP_OK);
    EXPECT(ffn_layer_backward(&n, x.p, x.ld, w.p, (float*)stats.p, gu.p, gu.ld, gx.p, gw.p, gx.p, N, ws.p, need, nullptr) == CGTP_EINVAL);
    EXPECT(ffn_layer_backward(&n, x.p, x.ld, w.p, (float*)stats.p, gu.p, gu.ld, gx.p, gw.p, gb.p, N, ws.p, need - 1, nullptr) == CGTP_EINVAL);
}

int main() {
    // rows, choices, experts, sizes: few rows and many, chunks whole and broken, k in parts, long runs in parts
    const int64_t sizes[][6] = {{1, 1, 1, 1, 1, 1},     {1, 2, 4, 17, 9, 5},    {5, 3, 3, 64, 24, 40},   {60, 1, 2, 33, 40, 9},  {150, 2, 3, 24, 16, 20},
                                {90, 2, 3, 9, 33, 30},  {400, 1, 2, 40, 8, 12}, {70, 4, 70, 5, 6, 3},    {80, 1, 1, 700, 6, 9},  {100, 1, 1, 5, 300, 8},
                                {1500, 2, 2, 9, 6, 10}, {64, 2, 2, 8, 6, 900}};
    for (const auto& s : sizes)
        for (int kind = 0; kind < 4; ++kind) {
            const int64_t gap = kind % 2 ? 3 : 0, off = kind / 2;
            experts<F32>(FFN_FP32, s[0], (int)s[1], (int)s[2], s[3], s[4], s[5], (int)(s[0] % 3), kind, gap, off);
            experts<B16>(s[3] % 2 ? FFN_FP16 : FFN_BF16, s[0], (int)s[1], (int)s[2], s[3], s[4], s[5], (int)(s[0] % 3), kind, gap, off);
        }
    EXPECT(parts_seen > 0 && few_seen > 0 && deep_seen > 0);
    std::printf("experts OK, %d launches\n", launches);
    for (int64_t N : {1, 3, 130})
        for (int64_t D : {1, 7, 64, 1401}) {
            layers<F32>(FFN_FP32, N, D, 0);
            layers<B16>(FFN_BF16, N, D, 5);
        }
    std::printf("layers OK\n");
    // the queries over the whole range: no overflow
    for (int64_t w : {1, 7, 4096, 65537, 1 << 20})
        for (int dtype : {FFN_FP32, FFN_BF16, FFN_FP16})
            for (int E : {1, 3, 100}) {
                ffn_experts_t p = nullptr;
                const int64_t df = (1 << 20) / E / (w > 4096 ? 1 : 3);
                EXPECT(ffn_experts_plan(E, w, df, w, FFN_GELU, dtype, &p) == CGTP_OK);
                for (int64_t N : {0LL, 1LL, 64LL, 65LL, 100001LL, 1LL << 30})
                    EXPECT(ffn_experts_workspace_bytes(p, N, 1) >= 0 && ffn_experts_backward_workspace_bytes(p, N, 1) >= 0);
                EXPECT(ffn_experts_workspace_bytes(p, 1LL << 29, 3) == -1 && ffn_experts_backward_workspace_bytes(p, 1, 1025) == -1);
                ffn_experts_destroy(p);
            }
    // more tiles than one launch takes: refused before anything is read
    ffn_experts_t p = nullptr;
    EXPECT(ffn_experts_plan(2, 1 << 20, 1 << 20, 1 << 20, FFN_SILU, FFN_BF16, &p) == CGTP_OK);
    EXPECT(ffn_experts_forward(p, (void*)256, 1 << 20, (int32_t*)512, (int32_t*)512, (int32_t*)512, (void*)512, (void*)1024, (void*)2048, nullptr, 1LL << 30, 1, (void*)4096, 1LL << 62, nullptr) == CGTP_EUNSUP);
    ffn_experts_destroy(p);
    if (fails) return 1;
    std::printf("sanitized host code OK\n");
    return 0;
}
