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
// A thread takes chunks of eight values of a row: every row is read once and written to, or gathered from, its places.

template <typename T> struct Chunk { typedef T V __attribute__((ext_vector_type(8))); };
template <typename T> __device__ __forceinline__ typename Chunk<T>::V load_chunk(const T* row, int64_t c, int64_t D) {
    typename Chunk<T>::V v;
    if (c + 8 <= D) {
        __builtin_memcpy(&v, row + c, sizeof(v));
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = c + j < D ? row[c + j] : (T)0.0f;
    }
    return v;
}
template <typename T> __device__ __forceinline__ void store_chunk(T* row, int64_t c, int64_t D, typename Chunk<T>::V v) {
    if (c + 8 <= D) {
        __builtin_memcpy(row + c, &v, sizeof(v));
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (c + j < D) row[c + j] = v[j];
    }
}

// Walks the chunks of `rows` rows, one a thread and turn, without a division a turn.
struct Chunks {
    int64_t row, at, rows, chunks, dr, da;
    __device__ Chunks(int64_t rows_, int64_t chunks_) : rows(rows_), chunks(chunks_) {
        const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x, stride = (int64_t)gridDim.x * blockDim.x;
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

// Sorted rows from offsets[experts] on.
__device__ __forceinline__ int64_t held_rows(const RouteArgs& p) {
    const int64_t n = p.offsets[p.experts];
    return n < 0 ? 0 : n < p.slots ? n : p.slots;
}
template <typename T> __device__ __forceinline__ void zero_behind(const RouteArgs& p) {
    if (!p.offsets) return;
    const int64_t held = held_rows(p);
    const typename Chunk<T>::V zero = {};
    for (Chunks k(p.slots - held, (p.ld_sorted + 7) >> 3); k.more(); k.next())
        store_chunk((T*)p.out_sorted + (held + k.row) * p.ld_sorted, k.at * 8, p.ld_sorted, zero);
}

template <typename T>
__global__ __launch_bounds__(kThreads) void gather_kernel(RouteArgs p) {
    for (Chunks k(p.N, (p.width + 7) >> 3); k.more(); k.next()) {
        const auto v = load_chunk((const T*)p.rows + k.row * p.ld, k.at * 8, p.width);
        const int32_t* place = p.place + k.row * p.per_row;
        for (int j = 0; j < p.per_row; ++j) {
            const uint32_t to = (uint32_t)place[j];
            if (to < (uint64_t)p.slots) store_chunk((T*)p.out_sorted + (int64_t)to * p.ld_sorted, k.at * 8, p.ld_sorted, v);
        }
    }
    zero_behind<T>(p);
}

template <typename T>
__global__ __launch_bounds__(kThreads) void combine_kernel(RouteArgs p) {
    for (Chunks k(p.N, (p.width + 7) >> 3); k.more(); k.next()) {
        const int32_t* place = p.place + k.row * p.per_row;
        float sum[8] = {};
        for (int j = 0; j < p.per_row; ++j) {
            const uint32_t from = (uint32_t)place[j];
            if (from >= (uint64_t)p.slots) continue;
            const float w = p.weights ? p.weights[k.row * p.per_row + j] : 1.0f;
            const auto v = load_chunk((const T*)p.sorted + (int64_t)from * p.width, k.at * 8, p.width);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] += w * to_f32(v[e]);
        }
        typename Chunk<T>::V o;
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = (T)sum[e];
        store_chunk((T*)p.out_rows + k.row * p.ld_out, k.at * 8, p.width, o);
    }
}

// The same of 32-bit sums in parts, four columns a thread.
template <typename T>
__global__ __launch_bounds__(kThreads) void combine_parts_kernel(RouteArgs p, int splits) {
    const int64_t ld = (p.width + 3) & ~3LL;
    for (Chunks k(p.N, ld >> 2); k.more(); k.next()) {
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

// TPR threads a row: they read grad_y's row once for four of its choices, and add up the products with those rows.
template <typename T, int TPR>
__global__ __launch_bounds__(kThreads) void combine_backward_kernel(RouteArgs p) {
    __shared__ float s[4 * (kThreads / 64)];
    constexpr int kRows = kThreads / TPR;
    const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR;
    const int64_t D = p.width;
    for (int64_t n0 = (int64_t)blockIdx.x * kRows; n0 < p.N; n0 += (int64_t)gridDim.x * kRows) {
        const int64_t n = n0 + sub < p.N ? n0 + sub : p.N - 1;
        const bool mine = n0 + sub < p.N;
        for (int k0 = 0; k0 < p.per_row; k0 += 4) {
            uint32_t at[4];
            float w[4], dot[4] = {};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                at[j] = k0 + j < p.per_row && mine ? (uint32_t)p.place[n * p.per_row + k0 + j] : ~0u;
                w[j] = k0 + j < p.per_row && p.weights ? p.weights[n * p.per_row + k0 + j] : 1.0f;
            }
            for (int64_t c = t * 8; c < D; c += TPR * 8) {
                const auto g = load_chunk((const T*)p.rows + n * p.ld, c, D);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (at[j] >= (uint64_t)p.slots) continue;
                    if (p.grad_weights) {
                        const auto v = load_chunk((const T*)p.sorted + (int64_t)at[j] * D, c, D);
#pragma unroll
                        for (int e = 0; e < 8; ++e) dot[j] += c + e < D ? to_f32(g[e]) * to_f32(v[e]) : 0.0f;
                    }
                    if (p.out_sorted) {
                        typename Chunk<T>::V o;
#pragma unroll
                        for (int e = 0; e < 8; ++e) o[e] = (T)(w[j] * to_f32(g[e]));
                        store_chunk((T*)p.out_sorted + (int64_t)at[j] * p.ld_sorted, c, p.ld_sorted, o);
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
                if (t == j && mine && k0 + j < p.per_row) p.grad_weights[n * p.per_row + k0 + j] = dot[j];
        }
    }
    if (p.out_sorted) zero_behind<T>(p);
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

int launch_gather(const RouteArgs& a, int32_t dtype, void* stream) {
    const dim3 grid(chunk_groups(a.N, a.width));
#define FFN_RUN(T) gather_kernel<T><<<grid, kThreads, 0, (hipStream_t)stream>>>(a)
    if (dtype == FFN_FP32) FFN_RUN(float);
    else FFN_RUN(bf16);   // bits alone
#undef FFN_RUN
    return (int)hipGetLastError();
}

int launch_combine(const RouteArgs& a, int32_t dtype, void* stream) {
    const dim3 grid(chunk_groups(a.N, a.width));
#define FFN_RUN(T) combine_kernel<T><<<grid, kThreads, 0, (hipStream_t)stream>>>(a)
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
    const dim3 grid((unsigned)(a.N < 4096 ? a.N : 4096));
#define FFN_RUN(T) combine_backward_kernel<T, 256><<<grid, kThreads, 0, (hipStream_t)stream>>>(a)
    FFN_BY_TYPE(FFN_RUN)
#undef FFN_RUN
    return (int)hipGetLastError();
}

}  // namespace ffn
