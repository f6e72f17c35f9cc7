// How the kernels of the experts find their rows: the runs' lengths are on the device, and each work-group looks for its
// own by a scan over the lanes of a wave.  Internal.
#pragma once

#include <hip/hip_runtime.h>

#include "experts_internal.h"

namespace ffn {
namespace dev {

struct Run { int expert, begin, end, tile; };   // sorted rows begin .. end - 1, and which of its tiles

// The runs' tiles of `side` rows, `least` or more of each, 64 experts at a time, one a lane.
struct Scan {
    int begin, end, upto;                         // of this lane's expert: its run, and the tiles of these 64 up to it
    __device__ __forceinline__ void read(const Groups& g, int e0, int lane, int side, int least) {
        const int e = e0 + lane, R = (int)g.rows;
        begin = end = 0;
        if (e < g.experts) {
            begin = g.offsets[e];
            end = g.offsets[e + 1];
        }
        begin = begin < 0 ? 0 : begin < R ? begin : R;
        end = end < begin ? begin : end < R ? end : R;
        upto = tiles_of(end - begin, side, least);
        if (e >= g.experts) upto = 0;
        // within 16 lanes, then the rows' sums to the rows behind them
        upto += __builtin_amdgcn_update_dpp(0, upto, 0x111, 0xf, 0xf, false);   // one lane up
        upto += __builtin_amdgcn_update_dpp(0, upto, 0x112, 0xf, 0xf, false);
        upto += __builtin_amdgcn_update_dpp(0, upto, 0x114, 0xf, 0xf, false);
        upto += __builtin_amdgcn_update_dpp(0, upto, 0x118, 0xf, 0xf, false);
        upto += __builtin_amdgcn_update_dpp(0, upto, 0x142, 0xa, 0xf, false);   // a row's last lane to the next row
        upto += __builtin_amdgcn_update_dpp(0, upto, 0x143, 0xc, 0xf, false);   // lane 31 to the last two
    }
    static __device__ __forceinline__ int tiles_of(int rows, int side, int least) {
        const int n = (int)((uint32_t)(rows + side - 1) / (uint32_t)side);
        return n < least ? least : n;
    }
    __device__ __forceinline__ int total() const { return __builtin_amdgcn_readlane(upto, 63); }
};

// All tiles of all runs.
__device__ __forceinline__ int count_tiles(const Groups& g, int lane, int side, int least, Scan& first) {
    first.read(g, 0, lane, side, least);
    int total = first.total();
    for (int e0 = 64; e0 < g.experts; e0 += 64) {
        Scan s;
        s.read(g, e0, lane, side, least);
        total += s.total();
    }
    return total;
}

// The run of tile t, which is one of them.
__device__ __forceinline__ Run find_tile(const Groups& g, int lane, int side, int least, Scan s, int t) {
    int e0 = 0;
    while (t >= s.total() && e0 + 64 < g.experts) {
        t -= s.total();
        e0 += 64;
        s.read(g, e0, lane, side, least);
    }
    const int at = __builtin_ctzll(__ballot(s.upto > t) | 1ull << 63);
    Run r;
    r.expert = e0 + at;
    r.begin = __builtin_amdgcn_readlane(s.begin, at);
    r.end = __builtin_amdgcn_readlane(s.end, at);
    r.tile = t - (__builtin_amdgcn_readlane(s.upto, at) - Scan::tiles_of(r.end - r.begin, side, least));
    return r;
}

}  // namespace dev
}  // namespace ffn
