// Tiled matrix product on the 16-bit matrix instructions, with the feed-forward
// block's epilogues.  Internal; instantiated once per array type (ffn_tile_*.hip).
//
// C(m, n) = sum_k A(m, k) B(n, k), A and B each stored with k adjacent ("rows")
// or with m / n adjacent ("columns").  A work-group of BM x BN outputs walks k in
// steps of 128 bytes (64 values of 16 bits, 32 of 32): operands go from memory to
// LDS directly (16 bytes a lane, no registers), a step ahead of the one that is
// multiplied, in two buffers.  Each of the WM x WN waves holds the 16 x 16
// accumulators of a (BM / WM) x (BN / WN) block.
//
// LDS layouts, chosen so that the direct loads write whole 1 KB runs and the
// reads meet no bank twice:
//   rows:    [row][128 bytes of k], 16-byte chunk c of row r kept at chunk
//            c ^ (r & 7), with 32 bits the even chunks before the odd ones
//            (c / 2 + 4 (c % 2) in place of c); fragments by 16-byte reads, in
//            both types of q ^ (r & 7) and that ^ 4 by lanes 16 q .. + 15
//   columns, 16 bits: [k][BM or BN], 32-byte unit u of row k kept at u ^ s(k),
//            s(k) = (k & 3) | ((k >> 3) & 1) << 2; fragments by the transposing
//            8-byte read (16 lanes give four k-rows of 16 values and get back one
//            column of four k each)
//   columns, 32 bits: [k][BM or BN], 64-byte unit u of row k kept at u ^ (k >> 3);
//            fragments by 4-byte reads
//
// 32-bit arrays run as three bf16 planes, x = x0 + x1 + x2 exactly (8 bits of the
// significand each; x0 is cut off, so that no plane overflows, x1 rounded to
// nearest, so that |x1| <= 2^-7 |x| and |x2| <= 2^-16 |x|, of either sign), by the
// six products x_i y_j with i + j <= 2.  What is left out, x1 y2 + x2 y1 + x2 y2, is
// at most 2^-22 of |x| |y|, 2^-25.5 of it in the root mean square over random
// significands, and has no preferred sign.  (The 32-bit matrix instruction has a
// sixteenth of the rate.)  The planes are formed in registers, behind the matrix
// instructions of the fragment before.
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

// Eight 32-bit values as three planes of bf16: the upper 16 bits, the nearest to the rest, and what is then left (at most
// eight bits of it: its upper half).  A nearest value in the first plane too would leave out a quarter of what is left out
// so, but pass the largest of the type; kept below it by two more instructions a pair, a training step takes 4 % more.
struct Planes { s16x8 p[3]; };
__device__ __forceinline__ Planes planes_of(const f32x4 (&x)[2]) {
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    typedef bf16 bf16x2 __attribute__((ext_vector_type(2)));
    u32x4 out[3];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        float v[2] = {x[k >> 1][(k & 1) * 2], x[k >> 1][(k & 1) * 2 + 1]};
#pragma unroll
        for (int i = 0; i < 3; ++i) {
            uint32_t w;
            if (i == 1) w = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{v[0], v[1]}), bf16x2));
            else w = __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, v[1]), __builtin_bit_cast(uint32_t, v[0]), 0x07060302);   // upper halves
            out[i][k] = w;
            v[0] -= __builtin_bit_cast(float, w << 16);
            v[1] -= __builtin_bit_cast(float, w & 0xFFFF0000u);
        }
    }
    return Planes{{__builtin_bit_cast(s16x8, out[0]), __builtin_bit_cast(s16x8, out[1]), __builtin_bit_cast(s16x8, out[2])}};
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

// dG and dU side by side (zeros behind dU), and H
template <typename T> __device__ __forceinline__ void store_gate_grad(const TileArgs& p, int64_t m, int64_t n, f32x4 dg, f32x4 du, f32x4 h) {
    T* d = (T*)p.c + m * p.ldc;
    store4<T>(d, n, p.N, 0, dg);
    store4<T>(d + p.N, n, p.N, p.ldc - p.N, du);
    store4<T>((T*)p.h + m * p.ldh, n, p.N, p.ldh, h);
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

// An operand that is read as it lies in memory: `end` is behind its last byte that may be read, and rows of a (COLS not)
// are rows index[..] / per of it, slots of `slots`, where index is given.
struct Exact {
    const char* end;
    const int32_t* index;
    uint32_t per, slots;
};

// The direct loads of one operand: `R` rows of C's index a tile, a step of k, by NW waves, values of ES bytes.  GATE: in
// blocks of GATE tile rows, half of the gate's rows, then the same half of the up projection's.  EXACT: rows start on any
// element and hold no zeros behind them (a direct load takes 16 bytes from any address that its values have, and zeros for
// each four bytes that are not wholly inside the buffer's range).
template <int ES, int R, int NW, bool COLS, int GATE, bool EXACT = false> struct Loader {
    static constexpr int kLoads = R * 128 / 1024 / NW, kPer = 16 / ES, kStep = 128 / ES;   // values a chunk, k a step
    static constexpr int kRows = R * ES <= 1024 ? 1024 / (R * ES) : 1, kChunks = 64 / kRows;   // columns: k rows a load, chunks of one
    __amdgpu_buffer_rsrc_t rsrc[GATE ? 2 : 1];
    const char* base[GATE ? 2 : 1];
    uint32_t voff[kLoads];
    uint32_t kpos;       // first k of this lane's chunk (rows) or k row of its first load (columns)
    int64_t step;
    const char* end;     // EXACT

    static __device__ __forceinline__ int swizzle(int k) {
        if constexpr (ES == 4) return k >> 3;
        return (k & 3) | ((k >> 3) & 1) << 2;
    }

    __device__ __forceinline__ void init(const void* p, int64_t ld, int64_t r0, int64_t rows, int64_t half, int wave, int lane, const Exact& x = {}) {
        end = x.end;
        if constexpr (!COLS) {
            const int sub = lane >> 3, at = (lane & 7) ^ sub, c = ES == 4 ? (at & 3) * 2 + (at >> 2) : at;
            kpos = c * kPer;
            step = 128;
            base[0] = (const char*)p + r0 * ld * ES;
            if constexpr (GATE != 0) base[1] = base[0] + half * ld * ES;
            const bool indexed = EXACT && x.index;
            if (indexed) base[0] = (const char*)p;
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int t = (i * NW + wave) * 8 + sub;
                int64_t r = t;
                if constexpr (GATE != 0) r = t / GATE * (GATE / 2) + t % (GATE / 2);
                if (r0 + r >= rows) r = rows - 1 - r0;
                if (indexed) {
                    const uint32_t slot = (uint32_t)x.index[r0 + r];
                    r = slot < x.slots ? slot / x.per : 0;
                }
                voff[i] = (uint32_t)(r * ld * ES + c * 16);
            }
        } else {
            constexpr int kUnit = ES == 4 ? 4 : 2;                  // chunks a swizzled unit
            base[0] = (const char*)p + r0 * ES;
            step = kStep * ld * ES;
            kpos = wave * kRows + lane / kChunks;
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int k = i * NW * kRows + (int)kpos, pos = lane % kChunks;
                int c = ((pos / kUnit) ^ swizzle(k)) * kUnit + pos % kUnit;
                if (r0 + c * kPer >= rows) c = 0;
                voff[i] = (uint32_t)(k * ld * ES + c * 16);
            }
        }
    }

    __device__ __forceinline__ int range(const char* from) const {
        if constexpr (!EXACT) return 0x7FFFFFFF;
        const int64_t left = end - from;
        return left < 0 ? 0 : left < 0x7FFFFFFF ? (int)left : 0x7FFFFFFF;
    }
    __device__ __forceinline__ void seek(int64_t bytes) {
#pragma unroll
        for (int g = 0; g < (GATE ? 2 : 1); ++g)
            rsrc[g] = __builtin_amdgcn_make_buffer_rsrc((void*)(base[g] + bytes), 0, range(base[g] + bytes), 0x00020000);
    }

    // left: k from this step's first on, or more
    __device__ __forceinline__ void issue(char* lds, int wave, int left) const {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int k = COLS ? (int)kpos + i * NW * kRows : (int)kpos;
            const uint32_t v = k < left ? voff[i] : kOut;
            FFN_LDS void* to = (FFN_LDS void*)(lds + (i * NW + wave) * 1024);
            if constexpr (GATE != 0) {
                if ((i * NW + wave) * 8 % GATE < GATE / 2) __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc[0], to, 16, v, 0, 0, 0);
                else __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc[1], to, 16, v, 0, 0, 0);
            } else {
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc[0], to, 16, v, 0, 0, 0);
            }
        }
    }
};

// Fragments: 16 rows and 32 k of an operand (16 bits: half kk of the step); lane l gets row l % 16, k = 8 (l / 16) .. + 7.
// The swizzles are exclusive ors of fields that hold nothing else, so that one lane offset serves all fragments: base()
// for the wave's first row r0 (a multiple of its tiles' rows), then an exclusive or and a constant for tile i.
template <int ES, int R, bool COLS> struct Fragments {
    static __device__ __forceinline__ int base(int r0, int lane) {
        const int q = lane >> 4, i = lane & 15;
        if constexpr (!COLS) return (r0 + i) * 128 + ((q ^ (i & 7)) << 4);
        if constexpr (ES == 4) return 8 * q * R * 4 + (((r0 >> 4) ^ q) << 6) + i * 4;
        const int k = q * 8 + (i >> 2);
        return k * R * 2 + (((r0 >> 4) ^ Loader<2, R, 1, true, 0>::swizzle(k)) << 5) + (i & 3) * 8;
    }
    static __device__ __forceinline__ s16x8 get(const char* lds, int base, int i, int kk) {
        if constexpr (!COLS) return *(const s16x8*)(lds + (base ^ (kk << 6)) + i * 2048);
        const char* at = lds + (base ^ (i << 5)) + kk * 64 * R;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((FFN_LDS s16x4*)at);
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((FFN_LDS s16x4*)(at + 8 * R));
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    }
    static __device__ __forceinline__ void get32(const char* lds, int base, int i, f32x4 (&v)[2]) {
        if constexpr (!COLS) {
            v[0] = *(const f32x4*)(lds + base + i * 2048);
            v[1] = *(const f32x4*)(lds + (base ^ 64) + i * 2048);
        } else {
            const char* at = lds + (base ^ (i << 6));
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e >> 2][e & 3] = *(const float*)(at + e * R * 4);
        }
    }
};

// Consecutive work-groups go to the eight dies in turn; each die gets a run of consecutive numbers of `total`.
__device__ __forceinline__ int by_die(int id, int total) {
    const int die = id & 7, per = total >> 3, more = total & 7;
    return die * per + (die < more ? die : more) + (id >> 3);
}
// Tile t of tm x tn: down `group` rows of tiles before one column on, so that what consecutive tiles read is little.
__device__ __forceinline__ void walk(int t, int tm, int tn, int group, int& m, int& n) {
    const int band = t / (group * tn), r = t - band * group * tn;
    const int rows = tm - band * group < group ? tm - band * group : group;
    m = band * group + r % rows;
    n = r / rows;
}
// Which part of k and which tile a work-group takes: each die a run of consecutive tiles of one part, down eight rows of
// them at a time, so that a die's L2 holds what its tiles share (down projection, 8192 x 4096 x 16384: 1.28 against 0.99
// PFLOP/s without).
__device__ __forceinline__ void place(int id, int tm, int tn, int splits, int& m, int& n, int& split) {
    const int tiles = tm * tn, t = by_die(id, tiles * splits);
    if (tm == 1) {   // nothing shared but x: a tile's parts side by side read its rows of B through (24 rows, 4096 x 16384: 29 us against 32)
        split = t % splits;
        m = 0;
        n = t / splits;
        return;
    }
    split = t / tiles;
    walk(t - split * tiles, tm, tn, 8, m, n);
}

template <bool V> struct Flag { static constexpr bool value = V; };

// The work-group meets with every wave's direct loads in LDS.  (A barrier alone orders the waves' own LDS accesses; the
// direct loads of the others are in flight as far as it goes, and whether the compiler waits for them before it depends on
// what it can tell of the buffers.)
__device__ __forceinline__ void landed() {
    __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0)
    __syncthreads();
}

// What one work-group multiplies: rows m0 .. m_end - 1 of A, of which it takes BM, by B's rows from tile tn on, over K, of
// which it takes part `split`; row m of the result is row out_row + m of out_rows in memory.
struct Work {
    const void *a, *b;
    int64_t m0, m_end, K, out_row, out_rows;
    int tn, split;
    Exact xa, xb;                         // EXACT
    float* part;                          // kEither: where the sums go, in rows of N up to a multiple of four; NULL: C
};

// A work-group's LDS: NB buffers of both operands, BM and BN rows of 128 bytes each, the kernel's own arrays (apart, so that
// the compiler can tell them apart).
template <int NB> struct TileLds { char *a[NB], *b[NB]; };
#define FFN_TILE_LDS(BM, BN)                                       \
    __shared__ __align__(1024) char sa0[BM * 128], sb0[BN * 128];  \
    __shared__ __align__(1024) char sa1[BM * 128], sb1[BN * 128];  \
    const TileLds<2> lds = {{sa0, sa1}, {sb0, sb1}}
#define FFN_TILE_LDS4(BM, BN)                                      \
    __shared__ __align__(1024) char sa0[BM * 128], sb0[BN * 128];  \
    __shared__ __align__(1024) char sa1[BM * 128], sb1[BN * 128];  \
    __shared__ __align__(1024) char sa2[BM * 128], sb2[BN * 128];  \
    __shared__ __align__(1024) char sa3[BM * 128], sb3[BN * 128];  \
    const TileLds<4> lds = {{sa0, sa1, sa2, sa3}, {sb0, sb1, sb2, sb3}}

// EXACT: operands as they lie in memory (see Loader).  Where rows end inside a chunk of 16 bytes, what follows them is set to
// zero in the registers, on both sides, in the last step.
// NB == 4 (128-wide tiles of 16-bit arrays): three steps are in flight where a work-group has a compute unit for itself, and
// each block of outputs has two waves, one for each half of a step, whose sums are added at the end.
template <typename T, int BM, int BN, int WM, int WN, bool AC, bool BC, int EPI, bool EXACT = false, int NB = 2>
__device__ __forceinline__ void tile_body(const TileArgs& p, const Work& w, const TileLds<NB>& lds) {
#ifdef __HIP_DEVICE_COMPILE__   // (the host's pass needs the launch stub alone)
    constexpr int KS = NB == 4 ? 2 : 1, NW = WM * WN * KS, MT = BM / WM / 16, CW = BN / WN, NT = CW / 16, ES = (int)sizeof(T), kStep = 128 / ES;
    char *const sa0 = lds.a[0], *const sb0 = lds.b[0], *const sa1 = lds.a[1], *const sb1 = lds.b[1];
    auto buffer = [&](int i) {
        if constexpr (NB == 4) if (i >= 4) return i == 4 ? lds.a[2] : i == 5 ? lds.b[2] : i == 6 ? lds.a[3] : lds.b[3];
        return i == 0 ? sa0 : i == 1 ? sb0 : i == 2 ? sa1 : sb1;
    };
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int half = wave / (WM * WN), at_block = wave % (WM * WN);   // (NB == 4: half of a step; 0)
    const int wm = (at_block / WN) * (BM / WM), wn = (at_block % WN) * CW;
    constexpr int kCols = EPI == kGate ? BN / 2 : BN;      // columns of C a tile covers
    const int64_t m0 = w.m0, n0 = (int64_t)w.tn * kCols;

    Loader<ES, BM, NW, AC, 0, EXACT> la;
    Loader<ES, BN, NW, BC, EPI == kGate ? CW : 0, EXACT> lb;
    la.init(w.a, p.lda, m0, w.m_end, 0, wave, lane, w.xa);
    lb.init(w.b, p.ldb, n0, p.N, p.N, wave, lane, w.xb);

    // this part's steps
    const int steps = (int)((w.K + kStep - 1) / kStep);
    const int s0 = (int)((int64_t)steps * w.split / p.splits), s1 = (int)((int64_t)steps * (w.split + 1) / p.splits), n = s1 - s0;
    const int last = steps - 1 - s0;                       // of the product, counted from this part's first
    const int rest = (int)(w.K - (int64_t)(steps - 1) * kStep);   // k in it
    const int clean = EXACT && (!AC || !BC) && rest % (16 / ES) != 0 ? last : -1;
    int ks = s0;
    auto issue = [&](char* a, char* b) {
        la.seek(ks * la.step);
        lb.seek(ks * lb.step);
        const int64_t left = w.K - (int64_t)ks * kStep;
        la.issue(a, wave, left < kStep ? (int)left : kStep);
        lb.issue(b, wave, left < kStep ? (int)left : kStep);
        ++ks;
    };

    f32x4 acc[MT][NT] = {};
    const int base_a = Fragments<ES, BM, AC>::base(wm, lane), base_b = Fragments<ES, BN, BC>::base(wn, lane);
    if constexpr (ES == 4) {
        // One step out of (a, b) while the next goes to (an, bn).  The planes of A's fragment i + 1 are cut, and fragment
        // i + 2 is read, behind the 6 NT matrix instructions of fragment i.
        auto step = [&](const char* a, const char* b, char* an, char* bn, bool more, auto cleaned) {
            if (more) issue(an, bn);
            auto cut = [&](f32x4 (&v)[2]) {
                if constexpr (decltype(cleaned)::value) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e >> 2][e & 3] = 8 * (lane >> 4) + e < rest ? v[e >> 2][e & 3] : 0.0f;
                }
            };
            int oa = base_a, ob = base_b;   // (made anew at every step: kept over the loop their sums would not fit the registers)
            asm volatile("" : "+v"(oa), "+v"(ob));
            Planes fb[NT], fa[2];
            f32x4 raw[2][2];
            Fragments<4, BM, AC>::get32(a, oa, 0, raw[0]);
            if constexpr (!AC) cut(raw[0]);
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                f32x4 v[2];
                Fragments<4, BN, BC>::get32(b, ob, j, v);
                if constexpr (!BC) cut(v);
                fb[j] = planes_of(v);
            }
            fa[0] = planes_of(raw[0]);
            Fragments<4, BM, AC>::get32(a, oa, 1, raw[1]);
            if constexpr (!AC) cut(raw[1]);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                if (i + 2 < MT) {
                    Fragments<4, BM, AC>::get32(a, oa, i + 2, raw[i & 1]);
                    if constexpr (!AC) cut(raw[i & 1]);
                }
                if (i + 1 < MT) fa[(i + 1) & 1] = planes_of(raw[(i + 1) & 1]);
                // planes (0, 2), (2, 0), (1, 1), (0, 1), (1, 0), (0, 0): the smallest first
#pragma unroll
                for (int x = 0; x < 6; ++x)
#pragma unroll
                    for (int j = 0; j < NT; ++j)
                        acc[i][j] = mfma16(fb[j].p[0x001102 >> (4 * x) & 3], fa[i & 1].p[0x010120 >> (4 * x) & 3], acc[i][j], bf16());
#pragma unroll
                for (int x = 0; x < 6 * NT; ++x) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x002, 2, 0);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            landed();
        };
        if (n > 0) issue(sa0, sb0);
        landed();
        // (the step that is cut is code of its own: a branch in the others would part the matrix instructions from what runs
        // behind them; 8192 x 512 to 3281 columns 199 us with it)
        const int plain = EXACT && clean == n - 1 ? n - 1 : n;
        int s = 0;
        for (; s + 1 < plain; s += 2) {
            step(sa0, sb0, sa1, sb1, true, Flag<false>());
            step(sa1, sb1, sa0, sb0, s + 2 < n, Flag<false>());
        }
        if (s < plain) step(sa0, sb0, sa1, sb1, s + 1 < n, Flag<false>());
        if constexpr (EXACT && (!AC || !BC))
            if (plain < n) step(plain & 1 ? sa1 : sa0, plain & 1 ? sb1 : sb0, sa0, sb0, false, Flag<true>());
    } else {
        s16x8 fa[2][MT], fb[2][NT];
        // half kk of step s into the registers' half `to`
        auto read = [&](const char* a, const char* b, int kk, int s, int to) {
            int oa = base_a, ob = base_b;   // (as above)
            asm volatile("" : "+v"(oa), "+v"(ob));
#pragma unroll
            for (int j = 0; j < NT; ++j) fb[to][j] = Fragments<2, BN, BC>::get(b, ob, j, kk);
#pragma unroll
            for (int i = 0; i < MT; ++i) fa[to][i] = Fragments<2, BM, AC>::get(a, oa, i, kk);
            if constexpr (EXACT && (!AC || !BC))
                if (s == clean) {
                    s16x8 keep;
#pragma unroll
                    for (int e = 0; e < 8; ++e) keep[e] = 32 * kk + 8 * (lane >> 4) + e < rest ? -1 : 0;
                    if constexpr (!BC)
#pragma unroll
                        for (int j = 0; j < NT; ++j) fb[to][j] &= keep;
                    if constexpr (!AC)
#pragma unroll
                        for (int i = 0; i < MT; ++i) fa[to][i] &= keep;
                }
        };
        auto multiply = [&](int kk) {
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j) acc[i][j] = mfma16(fb[kk][j], fa[kk][i], acc[i][j], T());
        };
        if constexpr (NB == 4) {
            // While a wave multiplies its half of a step, it reads that of the next.  Between steps all waves meet: by then
            // each has read its part of this step's buffer, which takes the step NB further on, and the next step's data,
            // asked for NB - 1 steps earlier, is there.
            constexpr int kIssued = (BM + BN) * 128 / 1024 / NW;   // a wave's direct loads a step
            static_assert(KS == 2 && kIssued == 4 && MT % 4 == 0, "the waits below; what the waves exchange");
            // Own LDS reads are done, and of the direct loads those of steps later than s, of which `ahead` at the most
            // have been asked for, may be in flight.
            auto arrived = [&](int s, int ahead) {
                const int later = n - 1 - s < ahead ? n - 1 - s : ahead;
                if (later >= 3) __builtin_amdgcn_s_waitcnt(0x007C);        // 12 loads
                else if (later == 2) __builtin_amdgcn_s_waitcnt(0x0078);   // 8
                else if (later == 1) __builtin_amdgcn_s_waitcnt(0x0074);   // 4
                else __builtin_amdgcn_s_waitcnt(0x0070);
                __builtin_amdgcn_sched_barrier(0);
                __builtin_amdgcn_s_barrier();
                asm volatile("" ::: "memory");   // (no read moves up)
                __builtin_amdgcn_sched_barrier(0);
            };
            auto step = [&](int at, int s) {
                const int next = (at + 1) % NB;
                arrived(s + 1, NB - 2);
                read(lds.a[next], lds.b[next], half, s + 1, next & 1);
                if (s + NB < n) issue(lds.a[at], lds.b[at]);
                multiply(at & 1);
            };
#pragma unroll
            for (int k = 0; k < NB; ++k)
                if (n > k) issue(lds.a[k], lds.b[k]);
            arrived(0, NB - 1);
            read(sa0, sb0, half, 0, 0);
            int s = 0;
            for (; s + NB <= n; s += NB)
#pragma unroll
                for (int k = 0; k < NB; ++k) step(k, s + k);
#pragma unroll
            for (int k = 0; k < NB - 1; ++k)
                if (s + k < n) step(k, s + k);
            // both halves' sums: each wave finishes one half of the rows
            __syncthreads();
            constexpr int kSwap = MT / 2 * NT;
            f32x4* const box = (f32x4*)buffer(wave);
            static_assert(kSwap * 1024 <= BM * 128, "the box");
#pragma unroll
            for (int i = 0; i < MT / 2; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j) box[(i * NT + j) * 64 + lane] = half ? acc[i][j] : acc[i + MT / 2][j];
            __syncthreads();
            const f32x4* const theirs = (const f32x4*)buffer(wave ^ 4);
#pragma unroll
            for (int i = 0; i < MT / 2; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j) acc[i][j] = (half ? acc[i + MT / 2][j] : acc[i][j]) + theirs[(i * NT + j) * 64 + lane];
        } else if constexpr (NW == 8) {
            // Two waves a SIMD, of which one reads fragments while the other multiplies: waves 4 - 7 run one phase behind.
            // (8192 x 4096 x 16384, bf16, down projection: 1.31 PFLOP/s; with all waves in step 1.20.)
            auto meet = [] {
                __builtin_amdgcn_sched_barrier(0);
                __builtin_amdgcn_s_barrier();
                __builtin_amdgcn_sched_barrier(0);
            };
            auto phases = [&](char* a, char* b, char* an, char* bn, int s, bool more) {
                if (more) issue(an, bn);
                read(a, b, 0, s, 0);
                __builtin_amdgcn_s_waitcnt(0xC07F);     // own LDS reads done
                meet();
                __builtin_amdgcn_s_setprio(1);
                multiply(0);
                __builtin_amdgcn_s_setprio(0);
                meet();
                read(a, b, 1, s, 1);
                __builtin_amdgcn_s_waitcnt(0x0070);     // own LDS reads done, own direct loads landed
                meet();
                __builtin_amdgcn_s_setprio(1);
                multiply(1);
                __builtin_amdgcn_s_setprio(0);
                meet();
            };
            if (n > 0) issue(sa0, sb0);
            landed();
            if (wave >= 4) meet();
            int s = 0;
            for (; s + 1 < n; s += 2) {
                phases(sa0, sb0, sa1, sb1, s, true);
                phases(sa1, sb1, sa0, sb0, s + 1, s + 2 < n);
            }
            if (s < n) phases(sa0, sb0, sa1, sb1, s, false);
            if (wave < 4) meet();
        } else {
            // While the matrix instructions of one half of a step run, the fragments of the next half are read.  Between
            // the halves all waves meet: by then each has read the last of this step's buffer, which takes the step after
            // the next from memory, and the next step's data is there.
            auto step = [&](int at, int s) {
                read(lds.a[at], lds.b[at], 1, s, 1);
                multiply(0);
                landed();
                read(lds.a[at ^ 1], lds.b[at ^ 1], 0, s + 1, 0);
                if (s + 2 < n) issue(lds.a[at], lds.b[at]);
                multiply(1);
            };
            if (n > 0) issue(sa0, sb0);
            if (n > 1) issue(sa1, sb1);
            landed();
            read(sa0, sb0, 0, 0, 0);
            int s = 0;
            for (; s + 2 <= n; s += 2) {
                step(0, s);
                step(1, s + 1);
            }
            if (s < n) step(0, s);
        }
    }

    // acc[i][j][e] is row m = .. + lane % 16, column n = .. + 4 (lane / 16) + e.  Each wave turns 32 rows at a time in
    // LDS of its own, so that memory is read and written along the rows.
    __syncthreads();
    constexpr int kRow = CW + 4, kTurn = 32 * kRow * 4;    // floats a row (four more than it holds: no bank twice)
    constexpr int kFit = (BM < BN ? BM : BN) * 128 / kTurn;
    static_assert(kFit >= 1 && 2 * NB * kFit >= NW, "a turn buffer for every wave");
    float* turn = (float*)(buffer(wave / kFit) + wave % kFit * kTurn);
    constexpr int kLanes = EPI == kGate ? CW / 8 : CW / 4, kTake = 64 / kLanes;      // lanes a row, rows a turn
    const int tr = lane / kLanes, tc = (lane % kLanes) * 4;
    // this wave's first column, and whether it and the ones behind it are all inside, with nothing to be written behind the
    // last (EXACT: whoever reads the rows cuts them)
    const int64_t nb = n0 + (EPI == kGate ? wn / 2 : wn), past = nb + kLanes * 4;
    const int64_t pad = EXACT ? 0 : EPI == kGate ? p.ldc : EPI == kGateGrad ? (p.ldc > 2 * p.N || p.ldh > p.N ? p.N + 1 : 0) : 0;
    const bool whole = past < p.N || (past == p.N && pad <= p.N);
#pragma unroll
    for (int i = 0; i < MT / KS; i += 2) {
        const int64_t mb = m0 + wm + half * (MT / 2 * 16) + i * 16, n = nb + tc;
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int j = 0; j < NT; ++j)
                *(f32x4*)(turn + (x * 16 + (lane & 15)) * kRow + j * 16 + (lane >> 4) * 4) = acc[i + x][j];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        // (kGateGrad: G and U of kAhead turns are asked for together)
        constexpr int kTurns = 32 / kTake, kAhead = EPI == kGateGrad ? 4 : 2;
        const float* from = turn + tr * kRow + tc;
        if (whole && mb + 32 <= w.m_end) {
            // All 32 rows inside: a wave's addresses are one scalar and 32-bit offsets of its lanes.  (Beside a short k the
            // epilogue is what counts: 11712 rows of 408 values to 2 x 1339 gated columns in bf16: 67 us, 79 with the bounds
            // and the activation's branch at every value.)
            const int64_t row = w.out_row + mb;
            const uint32_t ld = (uint32_t)p.ldc;
            char *c = nullptr, *h = nullptr, *sv = nullptr;
            if constexpr (EPI == kPartial) c = (char*)((float*)p.c + ((int64_t)w.split * w.out_rows + row) * p.ldc + nb);
            else c = (char*)((T*)p.c + row * p.ldc + nb);
            if constexpr (EPI == kGate || EPI == kGateGrad) sv = (char*)(p.saved + mb * 2 * p.N + nb);
            if constexpr (EPI == kGateGrad) h = (char*)((T*)p.h + mb * p.ldh + nb);
            auto put = [](char* base, uint32_t at, f32x4 v, auto zero) {
                typedef decltype(zero) Out;
                typedef Out Out4 __attribute__((ext_vector_type(4)));
                Out4 o;
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] = (Out)v[e];
                __builtin_memcpy(base + at, &o, sizeof(o));
            };
            auto get = [](const char* base, uint32_t at) {
                f32x4 v;
                __builtin_memcpy(&v, base + at, sizeof(v));
                return v;
            };
            const uint32_t two = (uint32_t)(8 * p.N), up = (uint32_t)(4 * p.N);   // bytes of a row of `saved`, of half of one
#pragma unroll 1
            for (int k0 = 0; k0 < kTurns; k0 += kAhead) {
                f32x4 gs[kAhead], us[kAhead];
                if constexpr (EPI == kGateGrad) {
#pragma unroll
                    for (int k = 0; k < kAhead; ++k) {
                        const uint32_t at = (tr + (k0 + k) * kTake) * two + tc * 4;
                        gs[k] = get(sv, at);
                        us[k] = get(sv + up, at);
                    }
                }
#pragma unroll
                for (int k = 0; k < kAhead; ++k) {
                    const int dr = (k0 + k) * kTake;
                    const uint32_t at = (tr + dr) * ld + tc;
                    const f32x4 v = *(const f32x4*)(from + dr * kRow);
                    if constexpr (EPI == kGate) {
                        const f32x4 u = *(const f32x4*)(from + dr * kRow + CW / 2);
                        f32x4 a, da;
                        activate_all<T, 4>(p.act, v, a, da);
                        put(c, at * ES, a * u, T());
                        if (p.saved) {
                            const uint32_t as = (tr + dr) * two + tc * 4;
                            put(sv, as, v, 0.0f);
                            put(sv + up, as, u, 0.0f);
                        }
                    } else if constexpr (EPI == kStore) {
                        put(c, at * ES, v, T());
                    } else if constexpr (EPI == kPartial) {
                        put(c, at * 4, v, 0.0f);
                    } else if constexpr (EPI == kEither) {
                        if (w.part) put((char*)(w.part + mb * ((p.N + 3) & ~3LL) + nb), ((tr + dr) * (uint32_t)((p.N + 3) & ~3LL) + tc) * 4, v, 0.0f);
                        else put(c, at * ES, v, T());
                    } else {
                        f32x4 a, da;
                        activate_all<T, 4>(p.act, gs[k], a, da);
                        put(c, at * ES, v * us[k] * da, T());
                        put(c + p.N * ES, at * ES, v * a, T());
                        put(h, ((tr + dr) * (uint32_t)p.ldh + tc) * ES, a * us[k], T());
                    }
                }
            }
        } else {
#pragma unroll 1
            for (int k0 = 0; k0 < kTurns; ++k0) {
                const int r = tr + k0 * kTake;
                const int64_t m = mb + r;
                if (m >= w.m_end) continue;
                const f32x4 v = *(const f32x4*)(turn + r * kRow + tc);
                if constexpr (EPI == kGate) {
                    const f32x4 u = *(const f32x4*)(turn + r * kRow + CW / 2 + tc);
                    f32x4 a, da;
                    activate_all<T, 4>(p.act, v, a, da);
                    store4<T>((T*)p.c + m * p.ldc, n, p.N, EXACT ? 0 : p.ldc, a * u);
                    if (p.saved) {
                        store4<float>(p.saved + m * 2 * p.N, n, p.N, 0, v);
                        store4<float>(p.saved + m * 2 * p.N + p.N, n, p.N, 0, u);
                    }
                } else if constexpr (EPI == kStore) {
                    store4<T>((T*)p.c + (w.out_row + m) * p.ldc, n, p.N, 0, v);
                } else if constexpr (EPI == kEither) {
                    if (w.part) store4<float>(w.part + m * ((p.N + 3) & ~3LL), n, p.N, 0, v);
                    else store4<T>((T*)p.c + (w.out_row + m) * p.ldc, n, p.N, 0, v);
                } else if constexpr (EPI == kPartial) {
                    store4<float>((float*)p.c + ((int64_t)w.split * w.out_rows + w.out_row + m) * p.ldc, n, p.N, 0, v);
                } else {
                    const f32x4 g = load4(p.saved + m * 2 * p.N, n, p.N), u = load4(p.saved + m * 2 * p.N + p.N, n, p.N);
                    f32x4 a, da;
                    activate_all<T, 4>(p.act, g, a, da);
                    store_gate_grad<T>(p, m, n, v * u * da, v * a, a * u);
                }
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
#endif
}

template <typename T, int BM, int BN, int WM, int WN, bool AC, bool BC, int EPI>
__global__ __launch_bounds__(64 * WM * WN) void tile_kernel(TileArgs p) {
    FFN_TILE_LDS(BM, BN);
    int tm, tn, split;
    place(blockIdx.x, p.tiles_m, p.tiles_n, p.splits, tm, tn, split);
    tile_body<T, BM, BN, WM, WN, AC, BC, EPI>(p, Work{p.a, p.b, (int64_t)tm * BM, p.M, p.K, 0, p.M, tn, split}, lds);
}

template <typename T, int BM, bool AC, bool BC, int EPI> int run_tile(const TileArgs& p, hipStream_t s) {
    constexpr int WM = 2, WN = BM == 256 ? 4 : 2;
    tile_kernel<T, BM, BM, WM, WN, AC, BC, EPI><<<dim3((unsigned)(p.tiles_m * p.tiles_n * p.splits)), 64 * WM * WN, 0, s>>>(p);
    return (int)hipGetLastError();
}

// tile: 256 or 128 (outputs a side of a work-group)
template <typename T> int run_product(const TileArgs& p, int32_t epilogue, bool ac, bool bc, int32_t tile, hipStream_t s) {
#define FFN_RUN(AC, BC, EPI) (tile == 256 ? run_tile<T, 256, AC, BC, EPI>(p, s) : run_tile<T, 128, AC, BC, EPI>(p, s))
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
