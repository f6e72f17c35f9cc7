// The experts' forward products for few rows each: those of ffn_few.h, a tile of an expert's rows a work-group, whose
// weights are read once for it.  Internal; instantiated once per array type (ffn_experts_few_*.hip).
#pragma once

#include "experts_device.h"
#include "ffn_few.h"

namespace ffn {
namespace dev {

// Bound by HBM, the weights (64 rows, two of 16 experts of 2048 x 4096 each, bf16: gated 99 us, 5.5 TB/s, down 57, 4.9; one row:
// 14.2 and 8.1, 4.7 and 4.1).
template <typename T, int MT, int NR, int EPI>
__global__ __launch_bounds__(512) void expert_few_kernel(FewArgs p, Groups g) {
    const int lane = threadIdx.x & 63, t = blockIdx.y;
    Scan first;
    if (t >= count_tiles(g, lane, 16 * MT, 0, first)) return;
    const Run r = find_tile(g, lane, 16 * MT, 0, first, t);
    const int begin = r.begin + r.tile * 16 * MT, rows = r.end - begin;
    few_body<T, MT, NR, EPI>(p, FewWork{(const char*)p.w + r.expert * g.b_step, rows < 16 * MT ? rows : 16 * MT, (int64_t)blockIdx.x * NR, begin, g.source,
                                        (uint32_t)g.per_row, (uint32_t)g.rows});
}

template <typename T, int MT, int EPI> int run_expert_few(const FewArgs& p, const Groups& g, int nr, int waves, int64_t most, hipStream_t s) {
    const dim3 grid((unsigned)((p.N + nr - 1) / nr), (unsigned)most);
    const int lds = waves * (nr > 16 ? 2 : 1) * (EPI == kGate ? 2 : 1) * MT * 1024;
    if (lds > 64 * 1024 || most > 65535) return (int)hipErrorInvalidValue;
    // (those that few_cut() asks for)
    constexpr bool k16 = MT > 1 || EPI == kStore || sizeof(T) == 4, k32 = MT > 1;
    if (nr == 8) {
        expert_few_kernel<T, MT, 8, EPI><<<grid, waves * 64, lds, s>>>(p, g);
        return (int)hipGetLastError();
    }
    if constexpr (k16) {
        if (nr == 16) {
            expert_few_kernel<T, MT, 16, EPI><<<grid, waves * 64, lds, s>>>(p, g);
            return (int)hipGetLastError();
        }
    }
    if constexpr (k32) {
        if (nr == 32) {
            expert_few_kernel<T, MT, 32, EPI><<<grid, waves * 64, lds, s>>>(p, g);
            return (int)hipGetLastError();
        }
    }
    return (int)hipErrorInvalidValue;
}

template <typename T> int expert_few(const FewArgs& p, const Groups& g, int32_t epilogue, int32_t rows, int nr, int waves, int64_t most, hipStream_t s) {
    // (fp32 takes tiles of 64 rows by the other kernels)
    constexpr int kMost = sizeof(T) == 4 ? 2 : 4;
    if (rows > 16 * kMost) return (int)hipErrorInvalidValue;
#define FFN_RUN(EPI)                                                       \
    (rows == 16   ? run_expert_few<T, 1, EPI>(p, g, nr, waves, most, s)    \
     : rows == 32 ? run_expert_few<T, 2, EPI>(p, g, nr, waves, most, s)    \
                  : run_expert_few<T, kMost, EPI>(p, g, nr, waves, most, s))
    return epilogue == kGate ? FFN_RUN(kGate) : FFN_RUN(kStore);
#undef FFN_RUN
}

}  // namespace dev
}  // namespace ffn
