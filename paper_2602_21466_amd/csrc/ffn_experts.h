// The tiled products of the experts' blocks: those of ffn_tile.h, with the rows of A in runs of one expert each.  Internal;
// instantiated once per array type (ffn_experts_*.hip).
//
// A launch has work-groups for every tile that there could be; each finds its own, and those beyond the last end at once.
// A tile's rows are of one expert, so that its B is that expert's.
#pragma once

#include "experts_device.h"
#include "ffn_tile.h"

namespace ffn {
namespace dev {

// Tiles of 256 that run at one time, and how many beyond a multiple of them are cut into four of 128 each: one of those alone
// takes 0.45 of a tile's time, so that up to 64 tiles take that and up to 128 twice that (16384 rows over 16 experts, 4096
// values to 2048, bf16: a seventh less time with it).
constexpr int kRound = 256, kCutTiles = 128;

// Work-group `block` of C = A B^T by expert.  CUT: see above.
template <typename T, int BM, bool BC, int EPI, bool CUT, int NB>
__device__ __forceinline__ void rows_group(const TileArgs& p, const Groups& g, int block, const TileLds<NB>& lds) {
    constexpr int WM = 2, WN = BM == 256 ? 4 : 2;
    const int lane = threadIdx.x & 63;
    Scan first;
    const int total = count_tiles(g, lane, BM, 0, first), tiles = total * p.tiles_n;
    // (the whole rounds' tiles are dealt to the dies apart from what is cut)
    const int over = tiles % kRound, rest = CUT && p.splits == 1 && tiles > kRound && over <= kCutTiles ? over : 0, whole = tiles - rest;
    if ((int64_t)block >= (int64_t)whole * p.splits + 4 * rest) return;
    // as place() does, but expert by expert, so that tiles side by side share an expert's B (16384 rows over 16 experts of 2048 x
    // 4096, a training step in bf16: 2.87 ms, 2.91 by rows of tiles across experts)
    const bool quarter = block >= whole * p.splits;
    int t = quarter ? by_die(block - whole, 4 * rest) : by_die(block, whole * p.splits), tm, tn;
    const int q = t & 3, split = quarter ? 0 : t / whole;
    t = quarter ? whole + (t >> 2) : t - split * whole;
    Run r = find_tile(g, lane, BM, 0, first, t / p.tiles_n);
    const int its = Scan::tiles_of(r.end - r.begin, BM, 0), bands = (its + 7) >> 3;
    walk(t % p.tiles_n + r.tile * p.tiles_n, its, p.tiles_n, (its + bands - 1) / bands, tm, tn);
    const int64_t shift = r.expert == g.experts - 1 ? g.b_shift : 0, behind = shift ? shift + kCopyRoom : 0;
    const Exact xa = {(const char*)g.a_end, g.source, (uint32_t)g.per_row, (uint32_t)g.rows}, xb = {(const char*)g.b_end + behind, nullptr, 1, 0};
    Work w = {p.a, (const char*)p.b + r.expert * g.b_step + shift, (int64_t)r.begin + (int64_t)tm * BM, r.end, p.K, 0, p.M, tn, split, xa, xb, nullptr};
    if constexpr (CUT) {
        if (quarter) {
            static_assert(BM == 256 && NB == 2, "a step's buffers of the smaller tiles in each of the larger's");
            w.m0 += (q >> 1) * 128;
            w.tn = tn * 2 + (q & 1);
            if (w.m0 >= r.end || (int64_t)w.tn * (EPI == kGate ? 64 : 128) >= p.N) return;
            const TileLds<4> four = {{lds.a[0], lds.b[0], lds.a[1], lds.b[1]}, {lds.a[0] + 16384, lds.b[0] + 16384, lds.a[1] + 16384, lds.b[1] + 16384}};
            tile_body<T, 128, 128, 2, 2, false, BC, EPI, true, 4>(p, w, four);
            return;
        }
    }
    tile_body<T, BM, BM, WM, WN, false, BC, EPI, true, NB>(p, w, lds);
}
// (16384 rows over 16 experts of 2048 x 4096 in bf16: the gated product with G and U kept 673 us, 0.82 PFLOP/s; 279 down, 0.98;
// dG, dU and H 436, 0.63, where G and U are read.)
template <typename T, int BM, bool BC, int EPI>
__global__ __launch_bounds__(BM == 256 ? 512 : 256) void expert_rows_kernel(TileArgs p, Groups g) {
    FFN_TILE_LDS(BM, BM);
    rows_group<T, BM, BC, EPI, BM == 256 && sizeof(T) == 2>(p, g, blockIdx.x, lds);
}
// The same for launches of no more tiles than compute units, where a step waits for memory and for the steps of its own
// work: deeper buffers, and two waves a SIMD (2002 rows of 1089 values over 6 experts to 2 x 725 gated columns and back to
// 1089, fp16: 22.7 and 15.0 us; 27.2 and 18.4 with a wave a SIMD, which reads and multiplies in turn).
template <typename T, bool BC, int EPI>
__global__ __launch_bounds__(512) void expert_rows_deep_kernel(TileArgs p, Groups g) {
    FFN_TILE_LDS4(128, 128);
    rows_group<T, 128, BC, EPI, false>(p, g, blockIdx.x, lds);
}

constexpr int kManyTiles = 64;
__host__ __device__ __forceinline__ constexpr int64_t sums_step(int64_t tiles) { return tiles >= kManyTiles ? (tiles + 7) & ~7LL : tiles; }

// Work-groups go to the eight dies in turn.  A part's tiles, where they are many, are dealt to the dies in runs (as place()
// does), each part's to all dies, as its rows may be many more than another's; where they are few, one after the other.  An
// expert of many rows is cut into parts of them, so that no work-group has many times another's steps (5 experts, the largest of 8192 rows' half, 3281 x 512 in fp32: 160 us, 294 without).
template <typename T, int BM, int NB>
__device__ __forceinline__ void sums_group(TileArgs p, const Groups& g, float* partial, int block, const TileLds<NB>& lds) {
    constexpr int WM = 2, WN = BM == 256 ? 4 : 2;
    const int lane = threadIdx.x & 63, tiles = p.tiles_m * p.tiles_n, step = (int)sums_step(tiles);
    const int unit = block / step, id = block - unit * step;
    if (id >= tiles) return;
    Run r = {unit, 0, 0, 0};
    bool whole = true;
    if (g.chunk == 0) {
        Scan s;
        s.read(g, unit & ~63, lane, 1, 0);
        r.begin = __builtin_amdgcn_readlane(s.begin, unit & 63);
        r.end = __builtin_amdgcn_readlane(s.end, unit & 63);
    } else {
        Scan first;
        if (unit >= count_tiles(g, lane, g.chunk, 1, first)) return;
        r = find_tile(g, lane, g.chunk, 1, first, unit);
        whole = r.end - r.begin <= g.chunk;
        r.begin += r.tile * g.chunk;
        if (r.end > r.begin + g.chunk) r.end = r.begin + g.chunk;
    }
    int tm = id % p.tiles_m, tn = id / p.tiles_m, split;
    if (tiles >= kManyTiles) place(id, p.tiles_m, p.tiles_n, 1, tm, tn, split);
    constexpr int64_t ES = (int64_t)sizeof(T);
    const Exact xa = {(const char*)g.a_end, nullptr, 1, 0}, xb = {(const char*)g.b_end, nullptr, 1, 0};
    p.splits = 1;
    tile_body<T, BM, BM, WM, WN, true, true, kEither, true, NB>(p, Work{(const char*)p.a + r.begin * p.lda * ES, (const char*)p.b + r.begin * p.ldb * ES, (int64_t)tm * BM, p.M,
                                                                    r.end - r.begin, r.expert * p.M, 0, tn, 0, xa, xb,
                                                                    whole ? nullptr : partial + (int64_t)unit * p.M * ((p.N + 3) & ~3LL)}, lds);
}

// The three products of the gradients that need dG, dU and H alone, in one launch, those of the longest sums first: the
// others take the places that these leave.  (The same sizes: 1374 us, 1.00 PFLOP/s; a
// training step takes a twentieth less than with three launches.)
template <typename T, int BM>
__global__ __launch_bounds__(BM == 256 ? 512 : 256) void expert_grads_kernel(ExpertGrads a) {
    FFN_TILE_LDS(BM, BM);
    const int at = (int)blockIdx.x < a.end[0] ? 0 : (int)blockIdx.x < a.end[1] ? 1 : 2, k = a.order[at];
    const int block = at ? blockIdx.x - a.end[at - 1] : blockIdx.x;
    if (k == 0) rows_group<T, BM, true, kPartial, false>(a.t[0], a.g[0], block, lds);
    else sums_group<T, BM>(a.t[k], a.g[k], a.partial[k - 1], block, lds);
}

template <typename T, int BM, bool BC, int EPI> int run_rows(const TileArgs& p, const Groups& g, hipStream_t s) {
    const dim3 grid((unsigned)(p.tiles_m * p.tiles_n * p.splits + (BM == 256 && sizeof(T) == 2 ? 3 * kCutTiles : 0)));
    if constexpr (BM == 128 && sizeof(T) == 2)
        if (g.deep) {
            expert_rows_deep_kernel<T, BC, EPI><<<grid, 512, 0, s>>>(p, g);
            return (int)hipGetLastError();
        }
    expert_rows_kernel<T, BM, BC, EPI><<<grid, BM == 256 ? 512 : 256, 0, s>>>(p, g);
    return (int)hipGetLastError();
}
template <typename T, int BM> int run_grads(ExpertGrads a, hipStream_t s) {
    int64_t end = 0;
    for (int at = 0; at < 3; ++at) {
        const int k = a.order[at];
        const TileArgs& t = a.t[k];
        if (t.a) end += (k == 0 ? (int64_t)t.tiles_m * t.tiles_n : sums_step((int64_t)t.tiles_m * t.tiles_n)) * t.splits;
        a.end[at] = (int32_t)end;
    }
    expert_grads_kernel<T, BM><<<dim3((unsigned)end), BM == 256 ? 512 : 256, 0, s>>>(a);
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
template <typename T> int expert_grads(const ExpertGrads& a, int32_t tile, hipStream_t s) { return tile == 256 ? run_grads<T, 256>(a, s) : run_grads<T, 128>(a, s); }

}  // namespace dev
}  // namespace ffn
