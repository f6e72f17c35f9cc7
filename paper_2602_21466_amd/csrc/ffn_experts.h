// The tiled products of the experts' blocks: those of ffn_tile.h, with the rows of A in runs of one expert each.  Internal;
// instantiated once per array type (ffn_experts_*.hip).
//
// The lengths of the runs are on the device.  A launch has work-groups for every tile that there could be; each finds its
// own by a scan of the runs' tiles over the lanes of a wave, and those beyond the last end at once.  A tile's rows are of one
// expert, so that its B is that expert's.
#pragma once

#include "experts_internal.h"
#include "ffn_tile.h"

namespace ffn {
namespace dev {

struct Run { int expert, begin, end, tile; };   // sorted rows begin .. end - 1, and which of its tiles

// The runs' tiles of `side` rows, 64 experts at a time, one a lane.
struct Scan {
    int begin, end, upto;                         // of this lane's expert: its run, and the tiles of these 64 up to it
    __device__ __forceinline__ void read(const Groups& g, int e0, int lane, int side) {
        const int e = e0 + lane, R = (int)g.rows;
        begin = end = 0;
        if (e < g.experts) {
            begin = g.offsets[e];
            end = g.offsets[e + 1];
        }
        begin = begin < 0 ? 0 : begin < R ? begin : R;
        end = end < begin ? begin : end < R ? end : R;
        upto = (end - begin + side - 1) / side;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int v = __shfl_up(upto, o, 64);
            if (lane >= o) upto += v;
        }
    }
    __device__ __forceinline__ int total() const { return __builtin_amdgcn_readlane(upto, 63); }
};

// All tiles of all runs.
__device__ __forceinline__ int count_tiles(const Groups& g, int lane, int side, Scan& first) {
    first.read(g, 0, lane, side);
    int total = first.total();
    for (int e0 = 64; e0 < g.experts; e0 += 64) {
        Scan s;
        s.read(g, e0, lane, side);
        total += s.total();
    }
    return total;
}

// The run of tile t, which is one of them.
__device__ __forceinline__ Run find_tile(const Groups& g, int lane, int side, Scan s, int t) {
    int e0 = 0;
    while (t >= s.total() && e0 + 64 < g.experts) {
        t -= s.total();
        e0 += 64;
        s.read(g, e0, lane, side);
    }
    const int at = __builtin_ctzll(__ballot(s.upto > t) | 1ull << 63);
    Run r;
    r.expert = e0 + at;
    r.begin = __builtin_amdgcn_readlane(s.begin, at);
    r.end = __builtin_amdgcn_readlane(s.end, at);
    r.tile = t - (__builtin_amdgcn_readlane(s.upto, at) - (r.end - r.begin + side - 1) / side);
    return r;
}

template <typename T, int BM, int WM, int WN, bool BC, int EPI>
__global__ __launch_bounds__(64 * WM * WN) void expert_rows_kernel(TileArgs p, Groups g) {
    const int lane = threadIdx.x & 63;
    Scan first;
    const int total = count_tiles(g, lane, BM, first);
    if ((int64_t)blockIdx.x >= (int64_t)total * p.tiles_n * p.splits) return;
    int tm, tn, split;
    place(blockIdx.x, total, p.tiles_n, p.splits, tm, tn, split);
    const Run r = find_tile(g, lane, BM, first, tm);
    const Exact xa = {(const char*)g.a_end, g.source, (uint32_t)g.per_row, (uint32_t)g.rows}, xb = {(const char*)g.b_end, nullptr, 1, 0};
    tile_body<T, BM, BM, WM, WN, false, BC, EPI, true>(p, Work{p.a, (const char*)p.b + r.expert * g.b_step, (int64_t)r.begin + (int64_t)r.tile * BM, r.end, p.K, 0, p.M,
                                                              tn, split, xa, xb});
}

// Each expert's tiles go round the eight dies, as its rows may be many more than another's.
template <typename T, int BM, int WM, int WN, int EPI>
__global__ __launch_bounds__(64 * WM * WN) void expert_sums_kernel(TileArgs p, Groups g) {
    const int tiles = p.tiles_m * p.tiles_n * p.splits, step = (tiles + 7) & ~7;
    const int e = blockIdx.x / step, id = blockIdx.x - e * step, R = (int)g.rows;
    if (id >= tiles) return;
    int tm, tn, split, begin = g.offsets[e], end = g.offsets[e + 1];
    begin = begin < 0 ? 0 : begin < R ? begin : R;
    end = end < begin ? begin : end < R ? end : R;
    place(id, p.tiles_m, p.tiles_n, p.splits, tm, tn, split);
    constexpr int64_t ES = (int64_t)sizeof(T);
    const Exact xa = {(const char*)g.a_end, nullptr, 1, 0}, xb = {(const char*)g.b_end, nullptr, 1, 0};
    tile_body<T, BM, BM, WM, WN, true, true, EPI, true>(p, Work{(const char*)p.a + begin * p.lda * ES, (const char*)p.b + begin * p.ldb * ES, (int64_t)tm * BM, p.M, end - begin,
                                                                (int64_t)e * p.M, g.experts * p.M, tn, split, xa, xb});
}

template <typename T, int BM, bool BC, int EPI> int run_rows(const TileArgs& p, const Groups& g, hipStream_t s) {
    constexpr int WM = 2, WN = BM == 256 ? 4 : 2;
    expert_rows_kernel<T, BM, WM, WN, BC, EPI><<<dim3((unsigned)(p.tiles_m * p.tiles_n * p.splits)), 64 * WM * WN, 0, s>>>(p, g);
    return (int)hipGetLastError();
}
template <typename T, int BM, int EPI> int run_sums(const TileArgs& p, const Groups& g, hipStream_t s) {
    constexpr int WM = 2, WN = BM == 256 ? 4 : 2;
    const int64_t step = ((int64_t)p.tiles_m * p.tiles_n * p.splits + 7) & ~7LL;
    expert_sums_kernel<T, BM, WM, WN, EPI><<<dim3((unsigned)(step * g.experts)), 64 * WM * WN, 0, s>>>(p, g);
    return (int)hipGetLastError();
}

template <typename T> int expert_rows(const TileArgs& p, const Groups& g, int32_t epilogue, bool bc, int32_t tile, hipStream_t s) {
#define FFN_RUN(BC, EPI) (tile == 256 ? run_rows<T, 256, BC, EPI>(p, g, s) : run_rows<T, 128, BC, EPI>(p, g, s))
    if (epilogue == kGate && !bc) return FFN_RUN(false, kGate);
    if (epilogue == kGateGrad && bc) return FFN_RUN(true, kGateGrad);
    if (epilogue == kStore && !bc) return FFN_RUN(false, kStore);
    if (epilogue == kPartial) return bc ? FFN_RUN(true, kPartial) : FFN_RUN(false, kPartial);
#undef FFN_RUN
    return (int)hipErrorInvalidValue;
}
template <typename T> int expert_sums(const TileArgs& p, const Groups& g, int32_t epilogue, int32_t tile, hipStream_t s) {
    if (epilogue == kStore) return tile == 256 ? run_sums<T, 256, kStore>(p, g, s) : run_sums<T, 128, kStore>(p, g, s);
    if (epilogue == kPartial) return tile == 256 ? run_sums<T, 256, kPartial>(p, g, s) : run_sums<T, 128, kPartial>(p, g, s);
    return (int)hipErrorInvalidValue;
}

}  // namespace dev
}  // namespace ffn
