// Tiled matrix product on the 16-bit matrix instructions, with the feed-forward
// block's epilogues.  Internal; instantiated once per array type (ffn_tile_*.hip).
//
// C(m, n) = sum_k A(m, k) B(n, k), A and B each stored with k adjacent ("rows")
// or with m / n adjacent ("columns").  A work-group of BM x BN outputs walks k in
// steps of 64: operands go from memory to LDS directly (16 bytes a lane, no
// registers), one step ahead of the step that is multiplied, in two buffers.
// Each of the WM x WN waves holds the 16 x 16 accumulators of a (BM / WM) x (BN / WN) block.  A step is two halves of
// 32 k: while the matrix instructions of one half run, the fragments of the next are read from LDS.  Between the halves
// all waves meet: by then each has read the last of this step's buffer, which takes the step after next from memory,
// and the next step's data, asked for a whole step earlier, is there.
//
// LDS layouts, chosen so that the direct loads write whole 1 KB runs and the
// reads meet no bank twice:
//   rows:    [row][64 k], 16-byte chunk c of row r kept at chunk c ^ (r & 7);
//            fragments by 16-byte reads
//   columns: [k][BM or BN], 32-byte unit u of row k kept at u ^ s(k),
//            s(k) = (k & 3) | ((k >> 3) & 1) << 2; fragments by the transposing
//            8-byte read (16 lanes give four k-rows of 16 values and get back one
//            column of four k each)
//
// 32-bit arrays run as three bf16 planes, x = x0 + x1 + x2 exactly (8 bits of the
// significand each, cut, not rounded, so that no plane overflows), by the six
// products x_i y_j with i + j <= 2: what is left out is below 2^-24 of |x| |y|.
#pragma once

#include "ffn_device.h"

namespace ffn {

namespace dev {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef fp16 fp16x4 __attribute__((ext_vector_type(4)));
typedef fp16 fp16x8 __attribute__((ext_vector_type(8)));
#define FFN_LDS __attribute__((address_space(3)))

__device__ __forceinline__ f32x4 mfma16(s16x8 a, s16x8 b, f32x4 c, bf16) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma16(s16x8 a, s16x8 b, f32x4 c, fp16) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(fp16x8, a), __builtin_bit_cast(fp16x8, b), c, 0, 0, 0);
}

// x cut to its upper 16 bits; the rest follows exactly.  What is not finite goes to the first plane alone.
__device__ __forceinline__ float cut(float x) { return __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, x) & 0xFFFF0000u); }
__device__ __forceinline__ void planes_of(float x, uint16_t (&p)[3]) {
    if ((__builtin_bit_cast(uint32_t, x) & 0x7F800000u) == 0x7F800000u) {
        // a NaN whose set bits are all cut away would read as infinite
        p[0] = (uint16_t)((__builtin_bit_cast(uint32_t, x) >> 16) | (x != x ? 0x40u : 0u));
        p[1] = p[2] = 0;
        return;
    }
    const float x0 = cut(x), r1 = x - x0, x1 = cut(r1), x2 = cut(r1 - x1);
    p[0] = (uint16_t)(__builtin_bit_cast(uint32_t, x0) >> 16);
    p[1] = (uint16_t)(__builtin_bit_cast(uint32_t, x1) >> 16);
    p[2] = (uint16_t)(__builtin_bit_cast(uint32_t, x2) >> 16);
}

// Four adjacent values of a row, columns n .. n + 3, in the arrays' type, by one store where all are inside (rows may
// start on any element: memory takes wide accesses at any address); whoever stores column N - 1 also writes zeros up to
// column `pad`, for products that read whole 16-byte chunks of the row.
template <typename Out> __device__ __forceinline__ void store4(Out* p, int64_t n, int64_t N, int64_t pad, f32x4 v) {
    typedef Out Out4 __attribute__((ext_vector_type(4)));
    if (n + 3 < N) {
        Out4 o;
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] = (Out)v[j];
        __builtin_memcpy(p + n, &o, sizeof(o));
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (n + j < N) p[n + j] = (Out)v[j];
    }
    if (n < N && n + 4 >= N)
        for (int64_t c = N; c < pad; ++c) p[c] = (Out)0.0f;
}

// The same for a 32-bit intermediate kept as three planes.
__device__ __forceinline__ void store4_planes(uint16_t* p, int64_t plane, int64_t n, int64_t N, int64_t pad, f32x4 v) {
    uint16_t q[4][3];
#pragma unroll
    for (int j = 0; j < 4; ++j) planes_of(v[j], q[j]);
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        uint16_t* r = p + i * plane;
        if (n + 3 < N) {
            const s16x4 o = {(short)q[0][i], (short)q[1][i], (short)q[2][i], (short)q[3][i]};
            __builtin_memcpy(r + n, &o, sizeof(o));
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (n + j < N) r[n + j] = q[j][i];
        }
        if (n < N && n + 4 >= N)
            for (int64_t c = N; c < pad; ++c) r[c] = 0;
    }
}

// An intermediate (H, dG, dU): in T, or as planes of T where the arrays hold 32 bits.
template <typename T, typename Out> __device__ __forceinline__ void store_mid(void* base, int64_t row, int64_t ld, int64_t plane, int64_t n,
                                                                              int64_t N, int64_t pad, f32x4 v) {
    if constexpr (sizeof(Out) == 4) store4_planes((uint16_t*)base + row * ld, plane, n, N, pad, v);
    else store4<T>((T*)base + row * ld, n, N, pad, v);
}

// dG and dU side by side (zeros behind dU), and H
template <typename T, typename Out> __device__ __forceinline__ void store_gate_grad(const TileArgs& p, int64_t m, int64_t n, f32x4 dg,
                                                                                   f32x4 du, f32x4 h) {
    store_mid<T, Out>(p.c, m, p.ldc, p.plane_c, n, p.N, 0, dg);
    if constexpr (sizeof(Out) == 4)
        store4_planes((uint16_t*)p.c + m * p.ldc + p.N, p.plane_c, n, p.N, p.ldc - p.N, du);
    else
        store4<T>((T*)p.c + m * p.ldc + p.N, n, p.N, p.ldc - p.N, du);
    store_mid<T, Out>(p.h, m, p.ldh, p.plane_h, n, p.N, p.ldh, h);
}

__device__ __forceinline__ f32x4 load4(const float* p, int64_t n, int64_t N) {
    f32x4 v = {};
    if (n + 3 < N) {
        __builtin_memcpy(&v, p + n, sizeof(v));
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (n + j < N) v[j] = p[n + j];
    }
    return v;
}

constexpr uint32_t kOut = 0x80000000u;    // beyond every buffer: a direct load from there writes zeros

// The direct loads of one operand: `R` rows of C's index a tile, 64 k a step, by NW waves.  GATE: in blocks of GATE
// tile rows, half of the gate's rows, then the same half of the up projection's.
template <int R, int NW, bool COLS, int GATE> struct Loader {
    static constexpr int kLoads = R * 128 / 1024 / NW;
    __amdgpu_buffer_rsrc_t rsrc[GATE ? 2 : 1];
    const char* base[GATE ? 2 : 1];
    uint32_t voff[kLoads];
    uint32_t kpos;       // first k of this lane's chunk (rows) or k row of its first load (columns)
    int64_t step;

    static __device__ __forceinline__ int swizzle(int k) {
        const int s = (k & 3) | ((k >> 3) & 1) << 2;
        return R >= 128 ? s : s & (R / 16 - 1);
    }

    __device__ __forceinline__ void init(const void* p, int64_t ld, int64_t r0, int64_t rows, int64_t half, int wave, int lane) {
        if constexpr (!COLS) {
            const int sub = lane >> 3, c = (lane & 7) ^ sub;
            kpos = c * 8;
            step = 128;
            if constexpr (GATE) {
                base[0] = (const char*)p + r0 * ld * 2;
                base[1] = base[0] + half * ld * 2;
#pragma unroll
                for (int i = 0; i < kLoads; ++i) {
                    const int t = (i * NW + wave) * 8 + sub;
                    int64_t r = t / GATE * (GATE / 2) + t % (GATE / 2);
                    if (r0 + r >= rows) r = rows - 1 - r0;
                    voff[i] = (uint32_t)(r * ld * 2 + c * 16);
                }
            } else {
                base[0] = (const char*)p + r0 * ld * 2;
#pragma unroll
                for (int i = 0; i < kLoads; ++i) {
                    int64_t r = (i * NW + wave) * 8 + sub;
                    if (r0 + r >= rows) r = rows - 1 - r0;
                    voff[i] = (uint32_t)(r * ld * 2 + c * 16);
                }
            }
        } else {
            constexpr int kRows = 1024 / (R * 2) ? 1024 / (R * 2) : 1;   // k rows a load
            constexpr int kChunks = 64 / kRows;
            base[0] = (const char*)p + r0 * 2;
            step = 64 * ld * 2;
            kpos = wave * kRows + lane / kChunks;
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int k = i * NW * kRows + (int)kpos, pos = lane % kChunks;
                int c = (((pos >> 1) ^ swizzle(k)) << 1) | (pos & 1);
                if (r0 + c * 8 >= rows) c = 0;
                voff[i] = (uint32_t)(k * ld * 2 + c * 16);
            }
        }
    }

    __device__ __forceinline__ void seek(int64_t bytes) {
#pragma unroll
        for (int g = 0; g < (GATE ? 2 : 1); ++g)
            rsrc[g] = __builtin_amdgcn_make_buffer_rsrc((void*)(base[g] + bytes), 0, (int)0x7FFFFFFF, 0x00020000);
    }

    // k left from this step's first on; `whole`: at least 64 of them
    __device__ __forceinline__ void issue(char* lds, int wave, int left) const {
        constexpr int kRows = COLS ? (1024 / (R * 2) ? 1024 / (R * 2) : 1) : 0;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int k = COLS ? (int)kpos + i * NW * kRows : (int)kpos;
            const uint32_t v = k < left ? voff[i] : kOut;
            FFN_LDS void* to = (FFN_LDS void*)(lds + (i * NW + wave) * 1024);
            if constexpr (GATE) {
                if ((i * NW + wave) * 8 % GATE < GATE / 2) __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc[0], to, 16, v, 0, 0, 0);
                else __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc[1], to, 16, v, 0, 0, 0);
            } else {
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc[0], to, 16, v, 0, 0, 0);
            }
        }
    }
};

// Fragments: 16 rows and 32 k (half kk of the step) of an operand; lane l gets row l % 16, k = 8 (l / 16) .. + 7.  The
// swizzles are exclusive ors of fields that hold nothing else, so that one lane offset serves all fragments: base()
// for the wave's first row r0, then an exclusive or and a constant.
template <int R, bool COLS> struct Fragments {
    static __device__ __forceinline__ int base(int r0, int lane) {
        const int q = lane >> 4, i = lane & 15;
        if constexpr (!COLS) return (r0 + i) * 128 + ((q ^ (i & 7)) << 4);
        const int k = q * 8 + (i >> 2);
        return k * R * 2 + (((r0 >> 4) ^ Loader<R, 1, true, 0>::swizzle(k)) << 5) + (i & 3) * 8;
    }
    // tile i of the wave's; r0 is a multiple of its tiles' rows
    static __device__ __forceinline__ s16x8 get(const char* lds, int base, int i, int kk) {
        if constexpr (!COLS) return *(const s16x8*)(lds + (base ^ (kk << 6)) + i * 2048);
        const char* at = lds + (base ^ (i << 5)) + kk * 64 * R;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((FFN_LDS s16x4*)at);
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((FFN_LDS s16x4*)(at + 8 * R));
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    }
};

// Which part of k and which tile a work-group takes.  Consecutive work-groups go to the eight dies in turn; each die gets
// a run of consecutive tiles of one part, and a run walks down eight rows of tiles before it moves one column on, so
// that a die's L2 holds what its tiles share (down projection, 8192 x 4096 x 16384: 1.28 against 0.99 PFLOP/s without).
__device__ __forceinline__ void place(int id, int tm, int tn, int splits, int& m, int& n, int& split) {
    const int tiles = tm * tn, total = tiles * splits, die = id & 7, per = total >> 3, more = total & 7;
    int t = die * per + (die < more ? die : more) + (id >> 3);
    if (tm == 1) {   // nothing shared but x: a tile's parts side by side read its rows of B through (24 rows, 4096 x 16384: 29 us against 32)
        split = t % splits;
        m = 0;
        n = t / splits;
        return;
    }
    split = t / tiles;
    t -= split * tiles;
    constexpr int kGroup = 8;
    const int band = t / (kGroup * tn), r = t - band * kGroup * tn;
    const int rows = tm - band * kGroup < kGroup ? tm - band * kGroup : kGroup;
    m = band * kGroup + r % rows;
    n = r / rows;
}

template <typename T, typename Out, int BM, int BN, int WM, int WN, bool AC, bool BC, int EPI>
__global__ __launch_bounds__(64 * WM * WN) void tile_kernel(TileArgs p) {
#ifdef __HIP_DEVICE_COMPILE__   // (the host's pass needs the launch stub alone)
    constexpr int NW = WM * WN, MT = BM / WM / 16, CW = BN / WN, NT = CW / 16;
    __shared__ __align__(1024) char sa0[BM * 128], sb0[BN * 128];
    __shared__ __align__(1024) char sa1[BM * 128], sb1[BN * 128];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int wm = (wave / WN) * (BM / WM), wn = (wave % WN) * CW;
    int tm, tn, split;
    place(blockIdx.x, p.tiles_m, p.tiles_n, p.splits, tm, tn, split);
    constexpr int kCols = EPI == kGate ? BN / 2 : BN;      // columns of C a tile covers
    const int64_t m0 = (int64_t)tm * BM, n0 = (int64_t)tn * kCols;

    Loader<BM, NW, AC, 0> la;
    Loader<BN, NW, BC, EPI == kGate ? CW : 0> lb;
    la.init(p.a, p.lda, m0, p.M, 0, wave, lane);
    lb.init(p.b, p.ldb, n0, p.N, p.N, wave, lane);

    // this split's steps, of 64 k each; the six products of planes of one 64 follow each other, while their operands are
    // in L2
    const int nk = (int)((p.K + 63) >> 6), pairs = p.planes == 3 ? 6 : 1, steps = nk * pairs;
    const int s0 = (int)((int64_t)steps * split / p.splits), s1 = (int)((int64_t)steps * (split + 1) / p.splits);
    int ks = s0 / pairs, pair = s0 - ks * pairs;

    auto issue = [&](char* a, char* b) {
        // planes (0, 2), (2, 0), (1, 1), (0, 1), (1, 0), (0, 0)
        const int pa = p.planes == 3 ? (0x010120 >> (4 * pair)) & 3 : 0, pb = p.planes == 3 ? (0x001102 >> (4 * pair)) & 3 : 0;
        la.seek(pa * p.plane_a * 2 + ks * la.step);
        lb.seek(pb * p.plane_b * 2 + ks * lb.step);
        const int64_t rest = p.K - (int64_t)ks * 64;
        const int left = rest < 64 ? (int)rest : 64;
        la.issue(a, wave, left);
        lb.issue(b, wave, left);
        if (++pair == pairs) { pair = 0; ++ks; }
    };

    f32x4 acc[MT][NT] = {};
    s16x8 fa[2][MT], fb[2][NT];
    const int base_a = Fragments<BM, AC>::base(wm, lane), base_b = Fragments<BN, BC>::base(wn, lane);
    auto read = [&](const char* a, const char* b, int kk) {
        // (the offsets are made anew at every reading: kept over the loop they would not fit the registers)
        int oa = base_a, ob = base_b;
        asm volatile("" : "+v"(oa), "+v"(ob));
#pragma unroll
        for (int j = 0; j < NT; ++j) fb[kk][j] = Fragments<BN, BC>::get(b, ob, j, kk);
#pragma unroll
        for (int i = 0; i < MT; ++i) fa[kk][i] = Fragments<BM, AC>::get(a, oa, i, kk);
    };
    auto multiply = [&](int kk) {
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j) acc[i][j] = mfma16(fb[kk][j], fa[kk][i], acc[i][j], T());
    };
    // one step out of (a, b), the next one's first half out of (an, bn)
    auto step = [&](char* a, char* b, char* an, char* bn, bool more) {
        read(a, b, 1);
        multiply(0);
        __syncthreads();
        if (more) issue(a, b);
        read(an, bn, 0);
        multiply(1);
    };

    const int n = s1 - s0;
    if constexpr (NW == 8) {
        // Two waves a SIMD, of which one reads fragments while the other multiplies: waves 4 - 7 run one phase behind.
        auto meet = [] {
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_barrier();
            __builtin_amdgcn_sched_barrier(0);
        };
        auto phases = [&](char* a, char* b, char* an, char* bn, bool more) {
            if (more) issue(an, bn);
            read(a, b, 0);
            __builtin_amdgcn_s_waitcnt(0xC07F);     // own LDS reads done
            meet();
            __builtin_amdgcn_s_setprio(1);
            multiply(0);
            __builtin_amdgcn_s_setprio(0);
            meet();
            read(a, b, 1);
            __builtin_amdgcn_s_waitcnt(0x0070);     // own LDS reads done, own direct loads landed
            meet();
            __builtin_amdgcn_s_setprio(1);
            multiply(1);
            __builtin_amdgcn_s_setprio(0);
            meet();
        };
        if (n > 0) issue(sa0, sb0);
        __syncthreads();
        if (wave >= 4) meet();
        int s = 0;
        for (; s + 1 < n; s += 2) {
            phases(sa0, sb0, sa1, sb1, true);
            phases(sa1, sb1, sa0, sb0, s + 2 < n);
        }
        if (s < n) phases(sa0, sb0, sa1, sb1, false);
        if (wave < 4) meet();
    } else {
        if (n > 0) issue(sa0, sb0);
        if (n > 1) issue(sa1, sb1);
        __syncthreads();
        read(sa0, sb0, 0);
        int s = 0;
        for (; s + 1 < n; s += 2) {
            step(sa0, sb0, sa1, sb1, s + 2 < n);
            step(sa1, sb1, sa0, sb0, s + 3 < n);
        }
        if (s < n) step(sa0, sb0, sa1, sb1, false);
    }

    // acc[i][j][e] is row m = .. + lane % 16, column n = .. + 4 (lane / 16) + e.  Each wave turns 32 rows at a time in
    // LDS of its own, so that memory is read and written along the rows.
    __syncthreads();
    constexpr int kRow = CW + 4, kTurn = 32 * kRow * 4;    // floats a row (four more than it holds: no bank twice)
    constexpr int kFit = (BM < BN ? BM : BN) * 128 / kTurn;
    static_assert(kFit >= 1 && 4 * kFit >= NW, "a turn buffer for every wave");
    float* turn = (float*)((wave / kFit == 0 ? sa0 : wave / kFit == 1 ? sb0 : wave / kFit == 2 ? sa1 : sb1) + wave % kFit * kTurn);
    constexpr int kLanes = EPI == kGate ? CW / 8 : CW / 4, kTake = 64 / kLanes;      // lanes a row, rows a turn
    const int tc = (lane % kLanes) * 4;
#pragma unroll
    for (int i = 0; i < MT; i += 2) {
        const int64_t mb = m0 + wm + i * 16, n = n0 + (EPI == kGate ? wn / 2 : wn) + tc;
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int j = 0; j < NT; ++j)
                *(f32x4*)(turn + (x * 16 + (lane & 15)) * kRow + j * 16 + (lane >> 4) * 4) = acc[i + x][j];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        // (kGateGrad: G and U of kAhead turns are asked for together; with the planes of 32-bit arrays so much code would
        // not be unrolled, and the sums would leave the registers)
        constexpr int kTurns = 32 / kTake, kAhead = EPI == kGateGrad && sizeof(Out) == 2 ? 4 : 1;
#pragma unroll 1
        for (int k0 = 0; k0 < kTurns; k0 += kAhead) {
        f32x4 gs[kAhead], us[kAhead];
        if constexpr (EPI == kGateGrad) {
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                const int64_t m = mb + lane / kLanes + (k0 + k) * kTake;
                gs[k] = us[k] = f32x4{};
                if (m < p.M) {
                    gs[k] = load4(p.saved + m * 2 * p.N, n, p.N);
                    us[k] = load4(p.saved + m * 2 * p.N + p.N, n, p.N);
                }
            }
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int r = lane / kLanes + (k0 + k) * kTake;
            const int64_t m = mb + r;
            if (m >= p.M) continue;
            const f32x4 v = *(const f32x4*)(turn + r * kRow + tc);
            if constexpr (EPI == kGate) {
                const f32x4 u = *(const f32x4*)(turn + r * kRow + CW / 2 + tc);
                f32x4 h;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float a, da;
                    activate(p.act, v[e], a, da);
                    h[e] = a * u[e];
                }
                store_mid<T, Out>(p.c, m, p.ldc, p.plane_c, n, p.N, p.ldc, h);
                if (p.saved) {
                    store4<float>(p.saved + m * 2 * p.N, n, p.N, 0, v);
                    store4<float>(p.saved + m * 2 * p.N + p.N, n, p.N, 0, u);
                }
            } else if constexpr (EPI == kStore) {
                store4<Out>((Out*)p.c + m * p.ldc, n, p.N, 0, v);
            } else if constexpr (EPI == kPartial) {
                store4<float>((float*)p.c + ((int64_t)split * p.M + m) * p.ldc, n, p.N, 0, v);
            } else {
                const f32x4 g = gs[k], u = us[k];
                f32x4 dg, du, h;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float a, da;
                    activate(p.act, g[e], a, da);
                    dg[e] = v[e] * u[e] * da;
                    du[e] = v[e] * a;
                    h[e] = a * u[e];
                }
                store_gate_grad<T, Out>(p, m, n, dg, du, h);
            }
        }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
#endif
}

template <typename T, typename Out, int BM, bool AC, bool BC, int EPI> int run_tile(const TileArgs& p, hipStream_t s) {
    constexpr int WM = 2, WN = BM == 256 ? 4 : 2;
    tile_kernel<T, Out, BM, BM, WM, WN, AC, BC, EPI><<<dim3((unsigned)(p.tiles_m * p.tiles_n * p.splits)), 64 * WM * WN, 0, s>>>(p);
    return (int)hipGetLastError();
}

// tile: 256 or 128 (outputs a side of a work-group)
template <typename T, typename Out> int run_product(const TileArgs& p, int32_t epilogue, bool ac, bool bc, int32_t tile, hipStream_t s) {
#define FFN_RUN(AC, BC, EPI) (tile == 256 ? run_tile<T, Out, 256, AC, BC, EPI>(p, s) : run_tile<T, Out, 128, AC, BC, EPI>(p, s))
    if (epilogue == kGate && !ac && !bc) return FFN_RUN(false, false, kGate);
    if (epilogue == kGateGrad && !ac && bc) return FFN_RUN(false, true, kGateGrad);
    if (epilogue == kStore) {
        if (!ac && !bc) return FFN_RUN(false, false, kStore);
        if (!ac && bc) return FFN_RUN(false, true, kStore);
        if (ac && bc) return FFN_RUN(true, true, kStore);
    }
    if (epilogue == kPartial) {
        if (!ac && !bc) return FFN_RUN(false, false, kPartial);
        if (!ac && bc) return FFN_RUN(false, true, kPartial);
        if (ac && bc) return FFN_RUN(true, true, kPartial);
    }
#undef FFN_RUN
    return (int)hipErrorInvalidValue;
}

}  // namespace dev
}  // namespace ffn
