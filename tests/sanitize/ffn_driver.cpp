// The feed-forward sublayer's plan source (ffn_plan.cpp: checks, workspace layouts, cutting of the products, order of
// the launches) under ASan/UBSan without a GPU.  The launchers are stand-ins that do on the host what a launch is asked
// for, plainly, reading and writing the elements that the kernels read and write: whole 16-byte chunks of operands,
// zeros behind rows, parts of k in their order.  Arrays are as long as the header says and the workspace as the query
// says, filled with NaN before every call, so a wrong offset, stride, size or order ends the run or shows in the
// results, which are held against the definition in 64 bits.  16-bit arrays are bf16 here, cut off (fp16 takes the same
// code on the host).
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <limits>
#include <vector>

#include "../../paper_2602_21466_amd/csrc/cgtp_internal.h"
#include "../../paper_2602_21466_amd/csrc/ffn_internal.h"

static int fails = 0, launches = 0;
#define EXPECT(cond)                                                       \
    do {                                                                   \
        if (!(cond)) {                                                     \
            std::printf("FAILED %s at line %d\n", #cond, __LINE__);        \
            ++fails;                                                       \
        }                                                                  \
    } while (0)

extern "C" hipError_t hipGetDevice(int* d) {
    *d = 0;
    return hipSuccess;
}
namespace cgtp {
void set_last_hip_error(int) {}
}

// ---------------------------------------------------------------- values and launches

struct F32 {
    static constexpr int size = 4;
    static double get(const void* p, int64_t i) { return ((const float*)p)[i]; }
    static void put(void* p, int64_t i, double v) { ((float*)p)[i] = (float)v; }
};
struct B16 {
    static constexpr int size = 2;
    static double get(const void* p, int64_t i) {
        const uint32_t u = (uint32_t)((const uint16_t*)p)[i] << 16;
        float f;
        std::memcpy(&f, &u, 4);
        return f;
    }
    static void put(void* p, int64_t i, double v) {
        const float f = (float)v;
        uint32_t u;
        std::memcpy(&u, &f, 4);
        ((uint16_t*)p)[i] = (uint16_t)(u >> 16);
    }
};

static double act(int a, double g) { return a == FFN_RELU ? std::fmax(g, 0.0) : a == FFN_SILU ? g / (1 + std::exp(-g)) : 0.5 * g * (1 + std::erf(g * std::sqrt(0.5))); }
static double dact(int a, double g) {
    if (a == FFN_RELU) return g > 0;
    if (a == FFN_SILU) { const double s = 1 / (1 + std::exp(-g)); return s * (1 + g * (1 - s)); }
    return 0.5 * (1 + std::erf(g * std::sqrt(0.5))) + g * std::exp(-0.5 * g * g) * 0.3989422804014327;
}

template <typename T> void finish(const ffn::TileArgs& t, int epi, int64_t m, int64_t n, double v, double u) {
    if (epi == ffn::kStore) { T::put(t.c, m * t.ldc + n, v); return; }
    if (epi == ffn::kGate) {
        T::put(t.c, m * t.ldc + n, act(t.act, v) * u);
        if (n == t.N - 1) for (int64_t c = t.N; c < t.ldc; ++c) T::put(t.c, m * t.ldc + c, 0);
        if (t.saved) { t.saved[m * 2 * t.N + n] = (float)v; t.saved[m * 2 * t.N + t.N + n] = (float)u; }
        return;
    }
    const double g = t.saved[m * 2 * t.N + n], up = t.saved[m * 2 * t.N + t.N + n];
    T::put(t.c, m * t.ldc + n, v * up * dact(t.act, g));
    T::put(t.c, m * t.ldc + t.N + n, v * act(t.act, g));
    T::put(t.h, m * t.ldh + n, act(t.act, g) * up);
    if (n == t.N - 1) {
        for (int64_t c = 2 * t.N; c < t.ldc; ++c) T::put(t.c, m * t.ldc + c, 0);
        for (int64_t c = t.N; c < t.ldh; ++c) T::put(t.h, m * t.ldh + c, 0);
    }
}

template <typename T> int tile(const ffn::TileArgs& t, int epi, bool ac, bool bc, int side) {
    ++launches;
    const int64_t per = 16 / T::size, step = 128 / T::size, rows_b = epi == ffn::kGate ? 2 * t.N : t.N;
    EXPECT(side == 128 || side == 256);
    EXPECT(t.tiles_m == (t.M + side - 1) / side && t.tiles_n == (rows_b + side - 1) / side);
    EXPECT((int64_t)t.tiles_m * t.tiles_n * t.splits <= 0x7FFFFFFF / 512);
    EXPECT(((uintptr_t)t.a & 15) == 0 && ((uintptr_t)t.b & 15) == 0 && t.lda % per == 0 && t.ldb % per == 0);
    EXPECT(epi == ffn::kPartial || t.splits == 1);
    auto up = [&](int64_t n) { return (n + per - 1) / per * per; };
    auto value = [&](const void* p, int64_t ld, bool cols, int64_t r, int64_t k) { return T::get(p, cols ? k * ld + r : r * ld + k); };
    // chunks that end behind the last row (columns) or behind K (rows; there zeros are read)
    double touched = 0;
    for (int64_t k = 0; k < t.K; ++k) {
        if (ac) for (int64_t r = t.M; r < up(t.M); ++r) touched += value(t.a, t.lda, true, r, k);
        if (bc) for (int64_t r = rows_b; r < up(rows_b); ++r) touched += value(t.b, t.ldb, true, r, k);
    }
    volatile double keep = touched;
    (void)keep;
    auto sum = [&](int64_t m, int64_t n, int64_t k0, int64_t k1) {
        double v = 0;
        for (int64_t k = k0; k < k1; ++k) {
            if (k >= t.K) {
                if (!ac) EXPECT(value(t.a, t.lda, false, m, k) == 0);
                if (!bc) EXPECT(value(t.b, t.ldb, false, n, k) == 0);
                continue;
            }
            v += value(t.a, t.lda, ac, m, k) * value(t.b, t.ldb, bc, n, k);
        }
        return v;
    };
    const int64_t steps = (t.K + step - 1) / step, end = up(t.K);
    for (int64_t m = 0; m < t.M; ++m)
        for (int64_t n = 0; n < t.N; ++n) {
            if (epi == ffn::kPartial) {
                for (int64_t s = 0; s < t.splits; ++s) {
                    const int64_t k0 = steps * s / t.splits * step, k1 = steps * (s + 1) / t.splits * step;
                    ((float*)t.c)[(s * t.M + m) * t.ldc + n] = (float)sum(m, n, k0, k1 < end ? k1 : end);
                }
            } else {
                finish<T>(t, epi, m, n, sum(m, n, 0, end), epi == ffn::kGate ? sum(m, t.N + n, 0, end) : 0);
            }
        }
    return 0;
}

template <typename T> int few(const ffn::FewArgs& p, int epi, int nr, int waves) {
    ++launches;
    const bool gate = epi == ffn::kGate;
    const int mt = p.M <= 16 ? 1 : p.M <= 32 ? 2 : 4;
    EXPECT(p.M <= ffn::kFewRows && (epi == ffn::kStore || gate));
    EXPECT(nr == 8 || (nr == 16 && (mt > 1 || T::size == 4)) || (nr == 32 && mt > 1 && gate));
    EXPECT(waves >= 1 && waves <= 8 && waves * (nr > 16 ? 2 : 1) * (gate ? 2 : 1) * mt <= 64);
    ffn::TileArgs t = {};
    t.N = p.N; t.act = p.act; t.c = p.c; t.ldc = p.ldc; t.saved = p.saved;
    for (int64_t m = 0; m < p.M; ++m)
        for (int64_t n = 0; n < p.N; ++n) {
            double v = 0, u = 0;
            for (int64_t k = 0; k < p.K; ++k) {
                v += T::get(p.x, m * p.ldx + k) * T::get(p.w, n * p.ldw + k);
                if (gate) u += T::get(p.x, m * p.ldx + k) * T::get(p.w, (p.N + n) * p.ldw + k);
            }
            finish<T>(t, epi, m, n, v, u);
        }
    return 0;
}

template <typename T> void pack(const ffn::PackJobs& jobs) {
    for (int j = 0; j < jobs.n; ++j) {
        const ffn::PackJob& q = jobs.job[j];
        EXPECT(q.to_ld % 8 == 0 && ((uintptr_t)q.to & 15) == 0);
        for (int64_t r = 0; r < q.rows; ++r)
            for (int64_t c = 0; c < q.to_ld; ++c) T::put(q.to, r * q.to_ld + c, c < q.width ? T::get(q.from, r * q.ld + c) : 0);
    }
}
template <typename T> void join(const float* partial, int64_t ld, int splits, int64_t M, int64_t N, void* out) {
    EXPECT(ld % 4 == 0);
    for (int64_t m = 0; m < M; ++m)
        for (int64_t n = 0; n < ld; ++n) {
            double v = 0;
            for (int s = 0; s < splits; ++s) v += partial[(s * M + m) * ld + n];   // (whole quads are read)
            if (n < N) T::put(out, m * N + n, v);
        }
}
template <typename T> void join_gate(const ffn::TileArgs& t, int epi, const float* partial, int64_t ld) {
    EXPECT(ld % 4 == 0);
    for (int64_t m = 0; m < t.M; ++m)
        for (int64_t n = 0; n < t.N; ++n) {
            double v = 0, u = 0;
            for (int s = 0; s < t.splits; ++s) {
                v += partial[(s * t.M + m) * ld + n];
                if (epi == ffn::kGate) u += partial[(s * t.M + m) * ld + t.N + n];
            }
            finish<T>(t, epi, m, n, v, u);
        }
}

// Norms: every array of a launch from its first to its last element.
static void touch(const void* p, int64_t rows, int64_t ld, int64_t width, int size, bool write) {
    if (!p) return;
    volatile unsigned char sink = 0;
    for (int64_t r = 0; r < rows; ++r) {
        char* row = (char*)p + r * ld * size;
        if (write) std::memset(row, 0, width * size);
        else for (int64_t c = 0; c < width * size; ++c) sink = sink + (unsigned char)row[c];
    }
}
static int norm(const ffn::NormArgs& a, int size, bool backward) {
    ++launches;
    const int64_t D = a.width, gates = (a.N + a.rows_per_gate - 1) / a.rows_per_gate;
    EXPECT(a.h || a.rows_per_gate == 1 || !backward);   // without a gate it divides nothing
    for (const void* p : {a.w, a.scale, a.wn}) touch(p, 1, D, D, size, false);
    touch(a.gate, gates, D, D, size, false);
    touch(a.h, a.N, D, D, size, false);
    if (backward) {
        touch(a.y, a.N, a.ldx, D, size, false);
        touch(a.gy, a.N, D, D, size, false);
        touch(a.gu, a.N, a.ldg, D, size, false);
        touch(a.h ? a.rstd_h : nullptr, a.N, 1, 1, 4, false);
        touch(a.gu ? a.rstd_y : nullptr, a.N, 1, 1, 4, false);
        for (void* p : {a.gx, a.gh}) touch(p, a.N, D, D, size, true);
        for (void* p : {a.gw, a.gscale, a.gwn}) touch(p, 1, D, D, size, true);
        touch(a.ggate, gates, D, D, size, true);
        touch(a.partial, 1, 0, ffn::norm_workspace_floats(D, a.N, a.rows_per_gate, a.h != nullptr, size), 4, true);
    } else {
        touch(a.x, a.N, a.ldx, D, size, false);
        touch(a.y, a.N, D, D, size, true);
        touch(a.u, a.N, a.ldu, D, size, true);
        touch(a.h ? a.rstd_h : nullptr, a.N, 1, 1, 4, true);
        touch(a.u ? a.rstd_y : nullptr, a.N, 1, 1, 4, true);
    }
    return 0;
}
static int drop(const void* x, int64_t ldx, void* y, int64_t ldy, int64_t N, int64_t width, int size) {
    ++launches;
    touch(x, N, ldx, width, size, false);
    touch(y, N, ldy, width, size, true);
    return 0;
}

namespace ffn {
int launch_tile_fp32(const TileArgs& p, int32_t e, bool a, bool b, int32_t t, void*) { return tile<F32>(p, e, a, b, t); }
int launch_tile_bf16(const TileArgs& p, int32_t e, bool a, bool b, int32_t t, void*) { return tile<B16>(p, e, a, b, t); }
int launch_tile_fp16(const TileArgs& p, int32_t e, bool a, bool b, int32_t t, void*) { return tile<B16>(p, e, a, b, t); }
int launch_few_fp32(const FewArgs& p, int32_t e, int32_t nr, int32_t w, void*) { return few<F32>(p, e, nr, w); }
int launch_few_bf16(const FewArgs& p, int32_t e, int32_t nr, int32_t w, void*) { return few<B16>(p, e, nr, w); }
int launch_few_fp16(const FewArgs& p, int32_t e, int32_t nr, int32_t w, void*) { return few<B16>(p, e, nr, w); }
int launch_few_grad(const FewGradArgs& p, void*) {
    ++launches;
    EXPECT(p.M <= kFewRows && p.N >= 4 && p.splits >= 1 && p.splits <= 65535);
    EXPECT(p.waves * 4 * (p.M <= 16 ? 1 : p.M <= 32 ? 2 : 4) <= 64);
    // a wave takes blocks of 32 k (16 above 32 rows of x), the waves of all parts in turn
    const int64_t block = p.M <= 32 ? 32 : 16;
    for (int64_t s = 0; s < p.splits; ++s)
        for (int64_t m = 0; m < p.M; ++m)
            for (int64_t n = 0; n < p.N; ++n) {
                double v = 0;
                for (int64_t k = 0; k < p.K; ++k)
                    if (k / block / p.waves % p.splits == s) v += F32::get(p.x, m * p.ldx + k) * F32::get(p.w, k * p.ldw + n);
                p.c[(s * p.M + m) * p.ldc + n] = (float)v;
            }
    return 0;
}
int launch_join(const float* from, int64_t ld, int32_t splits, int64_t M, int64_t N, void* out, int32_t dtype, void*) {
    ++launches;
    if (dtype == FFN_FP32) join<F32>(from, ld, splits, M, N, out);
    else join<B16>(from, ld, splits, M, N, out);
    return 0;
}
int launch_join_gate(const TileArgs& p, int32_t epi, const float* from, int64_t ld, int32_t dtype, void*) {
    ++launches;
    if (dtype == FFN_FP32) join_gate<F32>(p, epi, from, ld);
    else join_gate<B16>(p, epi, from, ld);
    return 0;
}
int launch_pack(PackJobs jobs, int32_t dtype, void*) {
    EXPECT(jobs.n >= 0 && jobs.n <= 4);
    if (dtype == FFN_FP32) pack<F32>(jobs);
    else pack<B16>(jobs);
    return 0;
}
int launch_zero(void* p, int64_t bytes, void*) {
    std::memset(p, 0, bytes);
    return 0;
}
int launch_norm_forward_fp32(const NormArgs& a, void*) { return norm(a, 4, false); }
int launch_norm_forward_bf16(const NormArgs& a, void*) { return norm(a, 2, false); }
int launch_norm_forward_fp16(const NormArgs& a, void*) { return norm(a, 2, false); }
int launch_norm_backward_fp32(const NormArgs& a, void*) { return norm(a, 4, true); }
int launch_norm_backward_bf16(const NormArgs& a, void*) { return norm(a, 2, true); }
int launch_norm_backward_fp16(const NormArgs& a, void*) { return norm(a, 2, true); }
int launch_dropout_fp32(const void* x, int64_t ldx, void* y, int64_t ldy, int64_t N, int64_t w, const DropArgs&, void*) { return drop(x, ldx, y, ldy, N, w, 4); }
int launch_dropout_bf16(const void* x, int64_t ldx, void* y, int64_t ldy, int64_t N, int64_t w, const DropArgs&, void*) { return drop(x, ldx, y, ldy, N, w, 2); }
int launch_dropout_fp16(const void* x, int64_t ldx, void* y, int64_t ldy, int64_t N, int64_t w, const DropArgs&, void*) { return drop(x, ldx, y, ldy, N, w, 2); }
// (any number that the caller cannot know: the launch writes all of it)
int64_t norm_workspace_floats(int64_t width, int64_t N, int64_t rows_per_gate, bool residual, int bytes) {
    return 3 * width + (residual ? 2 * N + rows_per_gate % 7 : N % 5) + bytes;
}
}  // namespace ffn

// ---------------------------------------------------------------- arrays

// Rows `ld` apart, from `off` elements behind a 256-byte boundary, exactly as long as they have to be.
template <typename T> struct Array {
    char* base = nullptr;
    void* p = nullptr;
    int64_t rows, width, ld, off;
    Array(int64_t rows, int64_t width, int64_t ld = 0, int64_t off = 0) : rows(rows), width(width), ld(ld ? ld : width), off(off) {
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

template <typename T> bool near(const Array<T>& got, const std::vector<double>& want, double tol) {
    double d = 0, w = 0;
    for (int64_t r = 0; r < got.rows; ++r)
        for (int64_t c = 0; c < got.width; ++c) {
            const double e = got.at(r, c) - want[r * got.width + c];
            d += e * e;
            w += want[r * got.width + c] * want[r * got.width + c];
        }
    if (!(d <= tol * tol * w)) std::printf("  off by %.3g\n", std::sqrt(d / w));
    return d <= tol * tol * w;
}

template <typename T> void block(int dtype, int64_t N, int64_t di, int64_t df, int64_t d_o, int act_, int64_t gap, int64_t off) {
    ffn_plan_t plan = nullptr;
    EXPECT(ffn_plan(di, df, d_o, act_, dtype, &plan) == CGTP_OK && plan);
    Array<T> x(N, di, di + gap, off), wi(2 * df, di), wo(d_o, df), gy(N, d_o, d_o + gap, off), y(N, d_o), gx(N, di), gwi(2 * df, di), gwo(d_o, df);
    Array<F32> saved(N, 2 * df);
    x.draw(1, 1); wi.draw(2, 1.5 / std::sqrt((double)di)); wo.draw(3, 1.5 / std::sqrt((double)df)); gy.draw(4, 1);
    // the definition
    std::vector<double> g(N * df), u(N * df), h(N * df), want(N * d_o), wx(N * di), wwi(2 * df * di), wwo(d_o * df);
    for (int64_t n = 0; n < N; ++n) {
        for (int64_t j = 0; j < df; ++j) {
            for (int64_t k = 0; k < di; ++k) {
                g[n * df + j] += x.at(n, k) * wi.at(j, k);
                u[n * df + j] += x.at(n, k) * wi.at(df + j, k);
            }
            h[n * df + j] = act(act_, g[n * df + j]) * u[n * df + j];
        }
        for (int64_t o = 0; o < d_o; ++o)
            for (int64_t j = 0; j < df; ++j) want[n * d_o + o] += h[n * df + j] * wo.at(o, j);
        for (int64_t j = 0; j < df; ++j) {
            double dh = 0;
            for (int64_t o = 0; o < d_o; ++o) {
                dh += gy.at(n, o) * wo.at(o, j);
                wwo[o * df + j] += gy.at(n, o) * h[n * df + j];
            }
            const double G = g[n * df + j], dg = dh * u[n * df + j] * dact(act_, G), du = dh * act(act_, G);
            for (int64_t k = 0; k < di; ++k) {
                wx[n * di + k] += dg * wi.at(j, k) + du * wi.at(df + j, k);
                wwi[j * di + k] += dg * x.at(n, k);
                wwi[(df + j) * di + k] += du * x.at(n, k);
            }
        }
    }
    const double tol = T::size == 4 ? 1e-5 : 5e-2;
    for (int save = 0; save < 2; ++save) {
        const int64_t need = ffn_workspace_bytes(plan, N);
        EXPECT(need >= 0 && need % 256 == 0);
        Array<F32> ws(1, need / 4);
        EXPECT(ffn_forward(plan, x.p, x.ld, wi.p, wo.p, y.p, save ? saved.p : nullptr, N, ws.p, need, nullptr) == CGTP_OK);
        EXPECT(near(y, want, tol));
        EXPECT(ffn_forward(plan, x.p, x.ld, wi.p, wo.p, y.p, nullptr, N, ws.p, need - 1, nullptr) == CGTP_EINVAL);
    }
    for (int which = 1; which < 8; ++which) {
        const int64_t need = ffn_backward_workspace_bytes(plan, N);
        Array<F32> ws(1, need / 4);
        EXPECT(ffn_backward(plan, x.p, x.ld, wi.p, wo.p, saved.p, gy.p, gy.ld, which & 1 ? gx.p : nullptr, which & 2 ? gwi.p : nullptr,
                            which & 4 ? gwo.p : nullptr, N, ws.p, need, nullptr) == CGTP_OK);
        if (which & 1) EXPECT(near(gx, wx, tol));
        if (which & 2) EXPECT(near(gwi, wwi, tol));
        if (which & 4) EXPECT(near(gwo, wwo, tol));
    }
    ffn_destroy(plan);
}

template <typename T> void norms(int dtype, int64_t N, int64_t D, int64_t rpg, int64_t gap) {
    ffn_norm n{D, rpg, dtype, 1e-6f, 0.25, 1, 2};
    const int64_t gates = (N + rpg - 1) / rpg;
    Array<T> x(N, D, D + gap, 1), u(N, D, D + 2 * gap, 3), gu(N, D, D + gap, 1), w(1, D), gx(N, D), gw(1, D);
    Array<F32> rstd(1, N);
    EXPECT(ffn_norm_forward(&n, x.p, x.ld, w.p, u.p, u.ld, (float*)rstd.p, N, nullptr) == CGTP_OK);
    {
        const int64_t need = ffn_norm_workspace_bytes(&n, N, 0);
        Array<F32> ws(1, need / 4);
        EXPECT(ffn_norm_backward(&n, x.p, x.ld, w.p, (float*)rstd.p, gu.p, gu.ld, gx.p, gw.p, N, ws.p, need, nullptr) == CGTP_OK);
        EXPECT(ffn_norm_backward(&n, x.p, x.ld, w.p, (float*)rstd.p, gu.p, gu.ld, gx.p, gw.p, N, ws.p, need - 1, nullptr) == CGTP_EINVAL);
    }
    Array<T> a(N, D), h(N, D), y(N, D), v(N, D), gate(gates, D), sc(1, D), wn(1, D), gh(N, D), gg(gates, D), gs(1, D), gn(1, D);
    Array<F32> stats(2, N);
    EXPECT(ffn_residual_forward(&n, a.p, h.p, w.p, gate.p, sc.p, wn.p, y.p, v.p, (float*)stats.p, N, nullptr) == CGTP_OK);
    EXPECT(ffn_residual_forward(&n, a.p, h.p, nullptr, nullptr, nullptr, nullptr, a.p, nullptr, nullptr, N, nullptr) == CGTP_OK);
    EXPECT(ffn_residual_forward(&n, a.p, h.p, w.p, gate.p, sc.p, wn.p, h.p, v.p, (float*)stats.p, N, nullptr) == CGTP_EINVAL);
    const int64_t need = ffn_norm_workspace_bytes(&n, N, 1);
    Array<F32> ws(1, need / 4);
    EXPECT(ffn_residual_backward(&n, h.p, y.p, w.p, gate.p, sc.p, wn.p, (float*)stats.p, a.p, v.p, a.p, gh.p, gw.p, gg.p, gs.p, gn.p, N,
                                 ws.p, need, nullptr) == CGTP_OK);
    EXPECT(ffn_residual_backward(&n, h.p, y.p, w.p, gate.p, sc.p, wn.p, (float*)stats.p, a.p, v.p, v.p, gh.p, gw.p, gg.p, gs.p, gn.p, N,
                                 ws.p, need, nullptr) == CGTP_EINVAL);
}

// Two views of one buffer are refused if and only if they share a byte.
void overlaps() {
    ffn_norm n{5, 1, FFN_BF16, 1e-6f, 0.0, 0, 0};
    Array<B16> buf(1, 200);
    for (int64_t N : {1, 2, 4})
        for (int64_t ldx : {5, 9, 12, 17})
            for (int64_t ldu : {5, 9, 12, 17})
                for (int64_t at = 0; at < 200; ++at) {
                    const int64_t x0 = 70;
                    if (at + (N - 1) * ldu + 5 > 200 || x0 + (N - 1) * ldx + 5 > 200) continue;
                    bool meet = false, span = !(at >= x0 + (N - 1) * ldx + 5 || x0 >= at + (N - 1) * ldu + 5);
                    for (int64_t i = 0; i < N; ++i)
                        for (int64_t j = 0; j < N; ++j) {
                            const int64_t d = at + j * ldu - x0 - i * ldx;
                            meet = meet || (d > -5 && d < 5);
                        }
                    void *x = (uint16_t*)buf.p + x0, *u = (uint16_t*)buf.p + at;
                    const bool same = at == x0 && ldu == ldx;
                    const bool taken = ffn_norm_forward(&n, x, ldx, nullptr, u, ldu, nullptr, N, nullptr) == CGTP_OK;
                    const bool dropped = ffn_dropout(x, ldx, u, ldu, N, 5, FFN_BF16, 0.5, 1, 2, nullptr) == CGTP_OK;
                    EXPECT(taken == dropped);
                    if (meet && !same) EXPECT(!taken);
                    if (!span || same) EXPECT(taken);
                    // rows of one stride: to the element, where all rows of both are side by side
                    if (ldx == ldu && !meet && at > x0 - ldx && at < x0 + ldx) EXPECT(taken);
                }
    // results as a block in the gap of strided rows
    Array<F32> wide(3, 40);
    ffn_plan_t plan = nullptr;
    EXPECT(ffn_plan(8, 8, 4, FFN_SILU, FFN_FP32, &plan) == CGTP_OK);
    Array<F32> wi(16, 8), wo(4, 8), ws(1, ffn_workspace_bytes(plan, 3) / 4);
    float* f = (float*)wide.p;
    for (int64_t at : {0, 4, 8, 28, 32, 36}) {
        const int rc = ffn_forward(plan, f + 0, 40, wi.p, wo.p, f + at, nullptr, 3, ws.p, ffn_workspace_bytes(plan, 3), nullptr);
        EXPECT(rc == (at >= 8 && at + 12 <= 40 ? CGTP_OK : CGTP_EINVAL));
    }
    ffn_destroy(plan);
}

int main() {
    // one row, few rows, many; chunks whole and broken; k in parts; strides and odd first elements
    const int64_t sizes[][4] = {{1, 1, 1, 1},    {1, 17, 9, 5},    {3, 64, 24, 40},  {16, 40, 70, 9},  {17, 33, 64, 130}, {40, 100, 36, 7},
                                {64, 8, 130, 3}, {65, 24, 40, 16}, {70, 33, 21, 19}, {130, 9, 66, 30}, {66, 700, 10, 9},  {300, 5, 12, 3},
                                {66, 5, 900, 20}, {33, 5, 900, 6}};
    for (const auto& s : sizes)
        for (int64_t gap : {0, 8, 3})
            for (int64_t off : {0, 1}) {
                block<F32>(FFN_FP32, s[0], s[1], s[2], s[3], (int)(s[0] % 3), gap, off);
                block<B16>(s[1] % 2 ? FFN_FP16 : FFN_BF16, s[0], s[1], s[2], s[3], (int)(s[0] % 3), gap, off);
            }
    std::printf("block OK, %d launches\n", launches);
    for (int64_t N : {1, 3, 130})
        for (int64_t D : {1, 7, 64, 1401})
            for (int64_t rpg : {1, 2, 1000}) {
                norms<F32>(FFN_FP32, N, D, rpg, 0);
                norms<B16>(FFN_BF16, N, D, rpg, 5);
            }
    std::printf("norms OK\n");
    overlaps();
    std::printf("overlaps OK\n");
    // the queries over the whole range: no overflow, and larger sizes need no less
    for (int64_t w : {1, 7, 4096, 65537, 1 << 20})
        for (int dtype : {FFN_FP32, FFN_BF16, FFN_FP16}) {
            ffn_plan_t p = nullptr;
            EXPECT(ffn_plan(w, (1 << 20) / (w > 4096 ? 1 : 3), w, FFN_GELU, dtype, &p) == CGTP_OK);
            for (int64_t N : {0LL, 1LL, 64LL, 65LL, 100001LL, 1LL << 30})
                EXPECT(ffn_workspace_bytes(p, N) >= 0 && ffn_backward_workspace_bytes(p, N) >= 0);
            EXPECT(ffn_workspace_bytes(p, (1LL << 30) + 1) == -1);
            // more tiles than one launch takes: refused before anything is read
            EXPECT(ffn_forward(p, (void*)256, w, (void*)512, (void*)1024, (void*)2048, nullptr, 1LL << 30, (void*)4096, 1LL << 62, nullptr) == CGTP_EUNSUP);
            ffn_destroy(p);
        }
    if (fails) return 1;
    std::printf("sanitized host code OK\n");
    return 0;
}
