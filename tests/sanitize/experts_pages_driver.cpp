// The workspaces that the experts' blocks ask for (experts_plan.cpp), and what their products read of weights that end with a page
// of memory: without a GPU.  The launchers are stand-ins that look at what they are asked for; the page behind each array cannot be
// read, so a byte read there ends the run.
#include <sys/mman.h>

#include <cstdio>
#include <cstdlib>
#include <cstring>

#include "../../paper_2602_21466_amd/csrc/cgtp_internal.h"
#include "../../paper_2602_21466_amd/csrc/experts_internal.h"

static int fails = 0, tiled = 0, copies = 0, few = 0;
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

static const char *ws_begin, *ws_end;
static volatile unsigned char sink;
static void read_all(const void* from, const void* end) {
    for (const char* p = (const char*)from; p < (const char*)end; ++p) sink = sink + (unsigned char)*p;
}
// Every byte that a product reads of B; the last expert's, where they are a copy, are its own values.
static int rows_seen(const ffn::TileArgs& t, const ffn::Groups& g, int size, int epi, bool cols) {
    ++tiled;
    // as the loads go: 16 bytes of a row at a time, of which the words that are wholly before the end
    const int64_t rows = cols ? t.K : epi == ffn::kGate ? 2 * t.N : t.N, width = (cols ? t.N : t.K) * size;
    for (int e = 0; e < g.experts; ++e) {
        const int64_t shift = e == g.experts - 1 ? g.b_shift : 0;
        const uintptr_t base = (uintptr_t)t.b + e * g.b_step + shift, end = (uintptr_t)g.b_end + (shift ? shift + ffn::kCopyRoom : 0);
        for (int64_t r = 0; r < rows; ++r)
            for (int64_t at = 0; at < (width + 15) / 16 * 16; at += 4) {
                const uintptr_t word = base + r * t.ldb * size + at;
                if (word + 4 <= end) read_all((const void*)word, (const void*)(word + 4));
            }
    }
    if (g.b_shift == 0) return 0;
    ++copies;
    const char *b = (const char*)t.b + (g.experts - 1) * g.b_step, *last = (const char*)((uintptr_t)b + g.b_shift);
    EXPECT(last >= ws_begin && last + g.b_step + 2 <= ws_end && (const char*)g.b_end == b + g.b_step + 2 - ffn::kCopyRoom);
    EXPECT(std::memcmp(last, b, g.b_step) == 0);
    return 0;
}
namespace ffn {
#define BY_TYPE(NAME, PARAMS, RUN)                                     \
    int NAME##_fp32 PARAMS { constexpr int kSize = 4; RUN; return kSize - 4; }  \
    int NAME##_bf16 PARAMS { constexpr int kSize = 2; RUN; return kSize - 2; }  \
    int NAME##_fp16 PARAMS { constexpr int kSize = 2; RUN; return kSize - 2; }
BY_TYPE(launch_expert_rows, (const TileArgs& t, const Groups& g, int32_t epi, bool cols, int32_t, void*), rows_seen(t, g, kSize, epi, cols))
BY_TYPE(launch_expert_few, (const FewArgs&, const Groups&, int32_t, int32_t, int32_t, int32_t, int64_t, void*), ++few)
BY_TYPE(launch_expert_grads, (const ExpertGrads& a, int32_t, void*), if (a.t[0].a) rows_seen(a.t[0], a.g[0], kSize, kPartial, true))
int launch_pack(PackJobs jobs, int32_t dtype, void*) {
    for (int k = 0; k < jobs.n; ++k)
        for (int64_t r = 0, e = dtype == FFN_FP32 ? 4 : 2; r < jobs.job[k].rows; ++r) {
            const PackJob& j = jobs.job[k];
            std::memset((char*)j.to + r * j.to_ld * e, 0, j.to_ld * e);
            std::memcpy((char*)j.to + r * j.to_ld * e, (const char*)j.from + r * j.ld * e, j.width * e);
        }
    return 0;
}
int launch_join_sums(const ExpertGrads&, int32_t, void*) { return 0; }
int launch_gather(const RouteArgs&, int32_t, void*) { return 0; }
int launch_combine(const RouteArgs&, int32_t, void*) { return 0; }
int launch_combine_backward(const RouteArgs&, int32_t, void*) { return 0; }
int launch_combine_parts(const RouteArgs&, int32_t, int32_t, void*) { return 0; }
int launch_join_rows(const float*, int64_t, int32_t, int64_t, int64_t, void*, int32_t, const int32_t*, void*) { return 0; }
int launch_join_gate_rows(const TileArgs&, int32_t, const float*, int64_t, int32_t, const int32_t*, void*) { return 0; }
int launch_sort(const SortArgs&, void*) { return 0; }
int launch_zero(void*, int64_t, void*) { return 0; }
}  // namespace ffn

// `bytes` of memory that end with a page, behind which nothing can be read.
static char* at_page_end(int64_t bytes) {
    const int64_t whole = (bytes + 4095) / 4096 * 4096;
    char* p = (char*)mmap(nullptr, whole + 4096, PROT_READ | PROT_WRITE, MAP_PRIVATE | MAP_ANONYMOUS, -1, 0);
    if (p == MAP_FAILED || mprotect(p + whole, 4096, PROT_NONE)) std::exit(2);
    for (int64_t i = 0; i < whole; ++i) p[i] = (char)(i * 7 + 3);
    return p + whole - bytes;
}

static int64_t asked(int E, int64_t di, int64_t df, int64_t d_o, int dtype, int64_t N, int K, bool backward) {
    ffn_experts_t p = nullptr;
    EXPECT(ffn_experts_plan(E, di, df, d_o, FFN_SILU, dtype, &p) == CGTP_OK);
    const int64_t n = backward ? ffn_experts_backward_workspace_bytes(p, N, K) : ffn_experts_workspace_bytes(p, N, K);
    ffn_experts_destroy(p);
    return n;
}

static void page_ends(int E, int64_t di, int64_t df, int64_t d_o, int64_t N) {
    ffn_experts_t plan = nullptr;
    EXPECT(ffn_experts_plan(E, di, df, d_o, FFN_GELU, FFN_BF16, &plan) == CGTP_OK);
    char *wi = at_page_end(E * 2 * df * di * 2), *wo = at_page_end(E * d_o * df * 2), *x = at_page_end(N * di * 2), *gy = at_page_end(N * d_o * 2);
    EXPECT(((uintptr_t)wi & 15) == 0 && ((uintptr_t)wo & 15) == 0);
    char *y = (char*)aligned_alloc(256, (N * d_o * 2 + 255) / 256 * 256), *saved = (char*)aligned_alloc(256, N * 2 * df * 4 + 256 - N * 2 * df * 4 % 256);
    char *gx = (char*)aligned_alloc(256, (N * di * 2 + 255) / 256 * 256), *gwi = (char*)aligned_alloc(256, (E * 2 * df * di * 2 + 255) / 256 * 256);
    char* gwo = (char*)aligned_alloc(256, (E * d_o * df * 2 + 255) / 256 * 256);
    int32_t *place = (int32_t*)calloc(N, 4), *source = (int32_t*)calloc(N, 4), *offsets = (int32_t*)calloc(E + 1, 4);
    int64_t need = ffn_experts_workspace_bytes(plan, N, 1);
    char* ws = (char*)aligned_alloc(256, need);
    ws_begin = ws; ws_end = ws + need;
    EXPECT(ffn_experts_forward(plan, x, di, place, source, offsets, wi, wo, y, saved, N, 1, ws, need, nullptr) == CGTP_OK);
    need = ffn_experts_backward_workspace_bytes(plan, N, 1);
    char* wb = (char*)aligned_alloc(256, need);
    ws_begin = wb; ws_end = wb + need;
    EXPECT(ffn_experts_backward(plan, x, di, place, source, offsets, wi, wo, saved, gy, gx, gwi, gwo, N, 1, wb, need, nullptr) == CGTP_OK);
    ffn_experts_destroy(plan);
}

int main() {
    // odd sizes ask for a copy of one expert's weights at the most, whatever the number of experts, beside 64 rows' intermediates
    // and sums
    for (int E : {1, 16, 64})
        for (bool backward : {false, true}) {
            const int64_t one = (2 * 4097 * 2049 + 2049 * 4097) * 2LL, odd = asked(E, 2049, 4097, 2049, FFN_BF16, 64, 1, backward);
            EXPECT(odd <= one + (16 << 20));
        }
    // the kernels for few rows: the hidden rows alone
    EXPECT(asked(8, 2048, 4096, 2048, FFN_BF16, 1, 2, false) == 2 * 4096 * 2);
    EXPECT(asked(8, 1024, 2048, 1024, FFN_FP32, 24, 1, false) == 24 * 2048 * 4);
    page_ends(3, 9, 256, 8, 300);      // odd rows of w_in
    page_ends(2, 8, 257, 64, 300);     // of w_out
    page_ends(4, 7, 9, 48, 1000);      // of both
    page_ends(1, 64, 64, 8, 300);      // of none
    page_ends(8, 1, 1, 8, 1000);       // of experts whose weights are less than what is read at a time
    page_ends(16, 3, 1, 1, 2000);
    page_ends(8, 8, 3, 1, 1000);
    EXPECT(tiled > 0 && copies >= 8);
    if (fails) return 1;
    std::printf("workspaces OK\n");
    return 0;
}
