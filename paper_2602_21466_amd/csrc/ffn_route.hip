// Rows sorted by expert and brought back (include/experts.h).
#include "experts_internal.h"
#include "ffn_tile.h"

namespace ffn {
namespace {

using namespace dev;

constexpr int kThreads = 256;

// ---------------------------------------------------------------- sorting
//
// A stable counting sort.  Work-group g takes the slots [g chunk, (g + 1) chunk), its waves consecutive parts of them, 64
// slots at a time: lanes with the same expert find each other by one ballot a bit of the expert's number, and the wave's
// count of the expert, in LDS, gives the first of them its place.  Sums are of whole numbers: any order gives the same.
constexpr int kSort = 512;

__device__ __forceinline__ int expert_of(const SortArgs& a, int64_t slot) {
    const int64_t e = a.index_bytes == 8 ? ((const int64_t*)a.index)[slot] : ((const int32_t*)a.index)[slot];
    return e >= 0 && e < a.experts ? (int)e : -1;
}

__global__ __launch_bounds__(kSort) void sort_count_kernel(SortArgs a) {
    __shared__ int count[FFN_MAX_EXPERTS];
    for (int e = threadIdx.x; e < a.experts; e += kSort) count[e] = 0;
    __syncthreads();
    const int64_t first = (int64_t)blockIdx.x * a.chunk, end = first + a.chunk < a.slots ? first + a.chunk : a.slots;
    for (int64_t i = first + threadIdx.x; i < end; i += kSort) {
        const int e = expert_of(a, i);
        if (e >= 0) atomicAdd(&count[e], 1);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < a.experts; e += kSort) a.counts[(int64_t)blockIdx.x * a.experts + e] = count[e];
}

__global__ __launch_bounds__(kSort) void sort_place_kernel(SortArgs a) {
    constexpr int kWaves = kSort / 64, kPer = FFN_MAX_EXPERTS / kSort;
    extern __shared__ int count[];                       // [waves][experts]
    __shared__ int total[FFN_MAX_EXPERTS], before[FFN_MAX_EXPERTS], sums[kWaves];
    const int E = a.experts, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    for (int e = threadIdx.x; e < E; e += kSort) total[e] = before[e] = 0;
    for (int i = threadIdx.x; i < kWaves * E; i += kSort) count[i] = 0;
    __syncthreads();

    const int64_t first = (int64_t)blockIdx.x * a.chunk, end = first + a.chunk < a.slots ? first + a.chunk : a.slots;
    const int64_t part = ((end - first + kWaves - 1) / kWaves + 63) & ~63LL;
    const int64_t w0 = first + wave * part, w1 = w0 + part < end ? w0 + part : end;
    for (int64_t i = w0 + lane; i < w1; i += 64) {
        const int e = expert_of(a, i);
        if (e >= 0) atomicAdd(&count[wave * E + e], 1);
    }
    // the other work-groups' counts
    if (a.groups > 1)
        for (int i = threadIdx.x; i < a.groups * E; i += kSort) {
            const int g = i / E, e = i - g * E, n = a.counts[i];
            atomicAdd(&total[e], n);
            if (g < (int)blockIdx.x) atomicAdd(&before[e], n);
        }
    __syncthreads();
    // where each expert's rows begin: thread t sums experts kPer t .. kPer t + kPer - 1
    int mine[kPer], sum = 0;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        const int e = threadIdx.x * kPer + j;
        int n = 0;
        if (e < E) {
            n = total[e];
            if (a.groups == 1)
                for (int w = 0; w < kWaves; ++w) n += count[w * E + e];
        }
        mine[j] = n;
        sum += n;
    }
    int scan = sum;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int v = __shfl_up(scan, o, 64);
        if (lane >= o) scan += v;
    }
    if (lane == 63) sums[wave] = scan;
    __syncthreads();
    int at = scan - sum, all = 0;
    for (int w = 0; w < kWaves; ++w) {
        if (w < wave) at += sums[w];
        all += sums[w];
    }
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        const int e = threadIdx.x * kPer + j;
        if (e < E) {
            if (blockIdx.x == 0) a.offsets[e] = at;
            int next = at + before[e];
            for (int w = 0; w < kWaves; ++w) {
                const int n = count[w * E + e];
                count[w * E + e] = next;
                next += n;
            }
            at += mine[j];
        }
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) a.offsets[E] = all;
    __syncthreads();

    const int bits = 32 - __builtin_clz(E);
    for (int64_t i = w0; i < w1; i += 64) {
        const int64_t slot = i + lane;
        const int e = slot < w1 ? expert_of(a, slot) : -1;
        uint64_t same = __ballot(e >= 0);
        for (int b = 0; b < bits; ++b) {
            const uint64_t set = __ballot(e >> b & 1);
            same &= (e >> b & 1) ? set : ~set;
        }
        const int rank = __popcll(same & ((1ull << lane) - 1));
        int p = -1;
        if (e >= 0) p = count[wave * E + e] + rank;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        if (e >= 0 && rank == 0) count[wave * E + e] = p + __popcll(same);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        if (slot < w1) a.place[slot] = p;
        if (p >= 0) a.source[p] = (int)slot;
    }
    for (int64_t p = all + (int64_t)blockIdx.x * kSort + threadIdx.x; p < a.slots; p += (int64_t)a.groups * kSort) a.source[p] = -1;
}

// ---------------------------------------------------------------- rows
//
// TPR threads take a row, 16 values a thread and turn in chunks of 16 bytes, side by side over the threads: x's rows
// (grad_y's) are read once for all of their choices, and the loads of four choices are in flight together.

template <typename T> struct Chunk {
    static constexpr int kVals = 16 / sizeof(T), kTurn = 16 / kVals;   // values, chunks a turn
    typedef T V __attribute__((ext_vector_type(kVals)));
};
template <typename T> __device__ __forceinline__ typename Chunk<T>::V load_chunk(const T* row, int64_t c, int64_t D) {
    constexpr int kVals = Chunk<T>::kVals;
    typename Chunk<T>::V v;
    if (c + kVals <= D) {
        __builtin_memcpy(&v, row + c, sizeof(v));
    } else {
#pragma unroll
        for (int j = 0; j < kVals; ++j) v[j] = c + j < D ? row[c + j] : (T)0.0f;
    }
    return v;
}
// Chunk i of a turn: those beyond the row repeat the turn's first, in whose branch they are read with it.
template <typename T, int TPR> __device__ __forceinline__ typename Chunk<T>::V load_turn(const T* row, int64_t c, int i, int64_t D) {
    const int64_t at = c + i * TPR * Chunk<T>::kVals;
    return load_chunk(row, i == 0 || at < D ? at : c, D);
}
template <typename T> __device__ __forceinline__ void store_chunk(T* row, int64_t c, int64_t D, typename Chunk<T>::V v) {
    constexpr int kVals = Chunk<T>::kVals;
    if (c + kVals <= D) {
        __builtin_memcpy(row + c, &v, sizeof(v));
    } else if (c < D) {
#pragma unroll
        for (int j = 0; j < kVals; ++j)
            if (c + j < D) row[c + j] = v[j];
    }
}

// A result: past the caches where all of them are more than these hold, as what stays there is written to memory during
// the next kernel (16384 x 4096 in bf16, two choices a row, gather and combine after each other and their gradients: 346 us;
// 366 with all kept, 366 with gather's alone kept).
template <typename T> __device__ __forceinline__ void put_chunk(T* row, int64_t c, int64_t D, typename Chunk<T>::V v, bool past) {
    typedef typename Chunk<T>::V U __attribute__((aligned(sizeof(T))));
    if (past && c + Chunk<T>::kVals <= D) __builtin_nontemporal_store(v, (U*)(row + c));
    else store_chunk(row, c, D, v);
}
template <typename T> __device__ __forceinline__ bool large(const RouteArgs& p) { return p.slots * p.width * (int64_t)sizeof(T) >= 16 << 20; }

// Walks the chunks of `rows` rows, one a thread and turn, without a division a turn.
struct Chunks {
    int64_t row, at, rows, chunks, dr, da;
    __device__ Chunks(int64_t rows_, int64_t chunks_, int64_t block, int64_t blocks) : rows(rows_), chunks(chunks_) {
        const int64_t i = block * blockDim.x + threadIdx.x, stride = blocks * blockDim.x;
        row = i / chunks;
        at = i - row * chunks;
        dr = stride / chunks;
        da = stride - dr * chunks;
    }
    __device__ bool more() const { return row < rows; }
    __device__ void next() {
        row += dr;
        at += da;
        if (at >= chunks) { at -= chunks; ++row; }
    }
};

// Zeros in the sorted rows from offsets[experts] on, by the work-groups behind those of the rows.
constexpr unsigned kZeroGroups = 64;
template <typename T> __device__ __forceinline__ void zero_behind(const RouteArgs& p) {
    int64_t held = p.offsets[p.experts];
    held = held < 0 ? 0 : held < p.slots ? held : p.slots;
    const typename Chunk<T>::V zero = {};
    constexpr int kVals = Chunk<T>::kVals;
    for (Chunks k(p.slots - held, (p.ld_sorted + kVals - 1) / kVals, blockIdx.x - (gridDim.x - kZeroGroups), kZeroGroups); k.more(); k.next())
        store_chunk((T*)p.out_sorted + (held + k.row) * p.ld_sorted, k.at * kVals, p.ld_sorted, zero);
}

// This thread's first row, its place among the row's threads, and from a row to its next one (of `groups` work-groups).
template <int TPR> __device__ __forceinline__ int64_t own_row(int& t) {
    t = threadIdx.x % TPR;
    const int sub = TPR >= 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x / TPR) : threadIdx.x / TPR;
    return (int64_t)blockIdx.x * (kThreads / TPR) + sub;
}
template <int TPR> __device__ __forceinline__ int64_t row_step(unsigned groups) { return (int64_t)groups * (kThreads / TPR); }

template <typename T, int TPR>
__global__ __launch_bounds__(kThreads) void gather_kernel(RouteArgs p) {
    if (p.offsets && blockIdx.x >= gridDim.x - kZeroGroups) return zero_behind<T>(p);
    constexpr int kVals = Chunk<T>::kVals, kTurn = Chunk<T>::kTurn;
    int t;
    const int64_t D = p.width;
    const bool past = large<T>(p);
    for (int64_t n = own_row<TPR>(t); n < p.N; n += row_step<TPR>(gridDim.x - (p.offsets ? kZeroGroups : 0))) {
        const T* row = (const T*)p.rows + n * p.ld;
        const int32_t* place = p.place + n * p.per_row;
        for (int64_t c = t * kVals; c < p.ld_sorted; c += TPR * 16) {
            typename Chunk<T>::V v[kTurn];
#pragma unroll
            for (int i = 0; i < kTurn; ++i) {
                v[i] = load_turn<T, TPR>(row, c, i, D);
                if (i > 0 && c + i * TPR * kVals >= D) v[i] = {};   // (stored where rows have room behind D)
            }
            for (int j = 0; j < p.per_row; ++j) {
                const uint32_t to = (uint32_t)place[j];
                if (to >= (uint64_t)p.slots) continue;
                T* out = (T*)p.out_sorted + (int64_t)to * p.ld_sorted;
#pragma unroll
                for (int i = 0; i < kTurn; ++i) put_chunk(out, c + i * TPR * kVals, p.ld_sorted, v[i], past);
            }
        }
    }
}

template <typename T, int TPR>
__global__ __launch_bounds__(kThreads) void combine_kernel(RouteArgs p) {
    constexpr int kVals = Chunk<T>::kVals, kTurn = Chunk<T>::kTurn;
    int t;
    const int64_t D = p.width;
    const bool past = large<T>(p);
    for (int64_t n = own_row<TPR>(t); n < p.N; n += row_step<TPR>(gridDim.x)) {
        const int32_t* place = p.place + n * p.per_row;
        const float* weights = p.weights ? p.weights + n * p.per_row : nullptr;
        for (int64_t c = t * kVals; c < D; c += TPR * 16) {
            float sum[kTurn][kVals] = {};
            for (int k = 0; k < p.per_row; k += 4) {
                typename Chunk<T>::V v[4][kTurn] = {};
                float w[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t from = k + j < p.per_row ? (uint32_t)place[k + j] : ~0u;
                    w[j] = 0.0f;
                    if (from >= (uint64_t)p.slots) continue;
                    w[j] = weights ? weights[k + j] : 1.0f;
                    const T* row = (const T*)p.sorted + (int64_t)from * D;
#pragma unroll
                    for (int i = 0; i < kTurn; ++i) v[j][i] = load_turn<T, TPR>(row, c, i, D);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int i = 0; i < kTurn; ++i)
#pragma unroll
                        for (int e = 0; e < kVals; ++e) sum[i][e] += w[j] * to_f32(v[j][i][e]);
            }
#pragma unroll
            for (int i = 0; i < kTurn; ++i) {
                typename Chunk<T>::V o;
#pragma unroll
                for (int e = 0; e < kVals; ++e) o[e] = (T)sum[i][e];
                put_chunk((T*)p.out_rows + n * p.ld_out, c + i * TPR * kVals, D, o, past);
            }
        }
    }
}

// The same of 32-bit sums in parts, four columns a thread.
template <typename T>
__global__ __launch_bounds__(kThreads) void combine_parts_kernel(RouteArgs p, int splits) {
    const int64_t ld = (p.width + 3) & ~3LL;
    for (Chunks k(p.N, ld >> 2, blockIdx.x, gridDim.x); k.more(); k.next()) {
        const int32_t* place = p.place + k.row * p.per_row;
        f32x4 sum = {};
        for (int j = 0; j < p.per_row; ++j) {
            const uint32_t from = (uint32_t)place[j];
            if (from >= (uint64_t)p.slots) continue;
            f32x4 v = {};
#pragma unroll 8
            for (int s = 0; s < splits; ++s) v += *(const f32x4*)((const float*)p.sorted + ((int64_t)s * p.slots + from) * ld + k.at * 4);
            sum += v;
        }
        store4<T>((T*)p.out_rows + k.row * p.ld_out, k.at * 4, p.width, 0, sum);
    }
}

// grad_y's row times the weights into its places, and its products with the rows there.
template <typename T, int TPR>
__global__ __launch_bounds__(kThreads) void combine_backward_kernel(RouteArgs p) {
    if (p.out_sorted && blockIdx.x >= gridDim.x - kZeroGroups) return zero_behind<T>(p);
    __shared__ float s[4 * (kThreads / 64)];
    constexpr int kVals = Chunk<T>::kVals, kTurn = Chunk<T>::kTurn / 2;   // (eight values a turn)
    int t;
    const int64_t D = p.width, first = own_row<TPR>(t), step = row_step<TPR>(gridDim.x - (p.out_sorted ? kZeroGroups : 0));
    const bool past = large<T>(p);
    for (int64_t start = (int64_t)blockIdx.x * (kThreads / TPR); start < p.N; start += step) {   // (the same turns for all threads)
        const int64_t row = first + (start - (int64_t)blockIdx.x * (kThreads / TPR)), n = row < p.N ? row : p.N - 1;
        const bool mine = row < p.N;
        const T* gy = (const T*)p.rows + n * p.ld;
        for (int k0 = 0; k0 < p.per_row; k0 += 4) {
            uint32_t at[4];
            float w[4], dot[4] = {};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                at[j] = k0 + j < p.per_row && mine ? (uint32_t)p.place[n * p.per_row + k0 + j] : ~0u;
                w[j] = k0 + j < p.per_row && p.weights ? p.weights[n * p.per_row + k0 + j] : 1.0f;
            }
            for (int64_t c = t * kVals; c < D; c += TPR * 8) {
                typename Chunk<T>::V g[kTurn], v[4][kTurn] = {};
#pragma unroll
                for (int i = 0; i < kTurn; ++i) g[i] = load_turn<T, TPR>(gy, c, i, D);
                if (p.grad_weights) {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
#pragma unroll
                        for (int i = 0; i < kTurn; ++i)
                            if (at[j] < (uint64_t)p.slots) v[j][i] = load_turn<T, TPR>((const T*)p.sorted + (int64_t)at[j] * D, c, i, D);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (at[j] >= (uint64_t)p.slots) continue;
                    if (p.grad_weights) {
#pragma unroll
                        for (int i = 0; i < kTurn; ++i) {
                            float sum = dot[j];
#pragma unroll
                            for (int e = 0; e < kVals; ++e) sum += to_f32(g[i][e]) * to_f32(v[j][i][e]);   // (zeros beyond the rows)
                            if (i == 0 || c + i * TPR * kVals < D) dot[j] = sum;
                        }
                    }
                    if (p.out_sorted) {
#pragma unroll
                        for (int i = 0; i < kTurn; ++i) {
                            typename Chunk<T>::V o;
#pragma unroll
                            for (int e = 0; e < kVals; ++e) o[e] = (T)(w[j] * to_f32(g[i][e]));
                            put_chunk((T*)p.out_sorted + (int64_t)at[j] * p.ld_sorted, c + i * TPR * kVals, p.ld_sorted, o, past);
                        }
                    }
                }
            }
            if (!p.grad_weights) continue;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
#pragma unroll
                for (int o = TPR < 64 ? TPR / 2 : 32; o; o >>= 1) dot[j] += __shfl_xor(dot[j], o, 64);
            }
            if constexpr (TPR > 64) {
                constexpr int W = TPR / 64;
                __syncthreads();
                if ((t & 63) == 0)
#pragma unroll
                    for (int j = 0; j < 4; ++j) s[(t >> 6) * 4 + j] = dot[j];
                __syncthreads();
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    dot[j] = s[j];
#pragma unroll
                    for (int w2 = 1; w2 < W; ++w2) dot[j] += s[w2 * 4 + j];
                }
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (t == j % TPR && mine && k0 + j < p.per_row) p.grad_weights[n * p.per_row + k0 + j] = dot[j];
        }
    }
}

unsigned chunk_groups(int64_t rows, int64_t width) {
    const int64_t chunks = (width + 7) / 8, n = (rows * chunks + kThreads - 1) / kThreads;
    return (unsigned)(n < 1 ? 1 : n < 8192 ? n : 8192);
}

}  // namespace

int launch_sort(const SortArgs& a, void* stream) {
    hipStream_t s = (hipStream_t)stream;
    if (a.groups > 1) sort_count_kernel<<<dim3((unsigned)a.groups), kSort, 0, s>>>(a);
    sort_place_kernel<<<dim3((unsigned)a.groups), kSort, kSort / 64 * a.experts * 4, s>>>(a);
    return (int)hipGetLastError();
}

#define FFN_BY_TYPE(RUN)                       \
    if (dtype == FFN_FP32) { RUN(float); }     \
    else if (dtype == FFN_BF16) { RUN(bf16); } \
    else { RUN(fp16); }

// Threads a row: one for two chunks, in steps of four.
#define FFN_BY_WIDTH(RUN, T)                   \
    const int64_t chunks = (a.width + 7) / 8;  \
    if (chunks <= 8) { RUN(T, 4); }            \
    else if (chunks <= 32) { RUN(T, 16); }     \
    else if (chunks <= 256) { RUN(T, 64); }    \
    else { RUN(T, 256); }
unsigned row_blocks(int64_t N, int tpr, bool zeros) {
    const int64_t n = (N * tpr + kThreads - 1) / kThreads;
    return (unsigned)(n < (1 << 22) ? n : 1 << 22) + (zeros ? kZeroGroups : 0);   // (a launch has fewer than 2^32 threads)
}

template <typename T> void run_gather(const RouteArgs& a, hipStream_t s) {
#define FFN_RUN(T, TPR) gather_kernel<T, TPR><<<dim3(row_blocks(a.N, TPR, a.offsets != nullptr)), kThreads, 0, s>>>(a)
    FFN_BY_WIDTH(FFN_RUN, T)
#undef FFN_RUN
}
template <typename T> void run_combine(const RouteArgs& a, hipStream_t s) {
#define FFN_RUN(T, TPR) combine_kernel<T, TPR><<<dim3(row_blocks(a.N, TPR, false)), kThreads, 0, s>>>(a)
    FFN_BY_WIDTH(FFN_RUN, T)
#undef FFN_RUN
}
template <typename T> void run_combine_backward(const RouteArgs& a, hipStream_t s) {
#define FFN_RUN(T, TPR) combine_backward_kernel<T, TPR><<<dim3(row_blocks(a.N, TPR, a.out_sorted != nullptr)), kThreads, 0, s>>>(a)
    FFN_BY_WIDTH(FFN_RUN, T)
#undef FFN_RUN
}

int launch_gather(const RouteArgs& a, int32_t dtype, void* stream) {
    if (dtype == FFN_FP32) run_gather<float>(a, (hipStream_t)stream);
    else run_gather<bf16>(a, (hipStream_t)stream);   // bits alone
    return (int)hipGetLastError();
}

int launch_combine(const RouteArgs& a, int32_t dtype, void* stream) {
#define FFN_RUN(T) run_combine<T>(a, (hipStream_t)stream)
    FFN_BY_TYPE(FFN_RUN)
#undef FFN_RUN
    return (int)hipGetLastError();
}

int launch_combine_parts(const RouteArgs& a, int32_t splits, int32_t dtype, void* stream) {
    const dim3 grid(chunk_groups(a.N, 2 * a.width));
#define FFN_RUN(T) combine_parts_kernel<T><<<grid, kThreads, 0, (hipStream_t)stream>>>(a, splits)
    FFN_BY_TYPE(FFN_RUN)
#undef FFN_RUN
    return (int)hipGetLastError();
}

int launch_combine_backward(const RouteArgs& a, int32_t dtype, void* stream) {
#define FFN_RUN(T) run_combine_backward<T>(a, (hipStream_t)stream)
    FFN_BY_TYPE(FFN_RUN)
#undef FFN_RUN
    return (int)hipGetLastError();
}

}  // namespace ffn
