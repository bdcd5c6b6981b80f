// Tiles, operands and masks shared by the attention kernels (attention.hip,
// attention_grad.hip).
//
// Matrix products run as 32 x 32 tiles.  An operand fragment holds eight values a
// lane: lane l has row (A) or column (B) l % 32 and, of a step of 16 along the
// summed dimension, the eight from 8 (l / 32).  bfloat16 takes one 32x32x16
// instruction a step, float32 eight 32x32x2 ones.  The result's lane has column
// l % 32 and in register r row tile_row(l, r).
//
// So the scores are formed transposed (keys are rows, queries columns): a lane
// then holds scores of one query, and, read as a fragment, its registers 8c..8c+7
// are the eight values of step c of the next product's B operand, with the keys in
// the order tile_row gives.  Sums do not care for the order, so the other operand
// is read in the same one and probabilities never leave their registers.
#pragma once

#include "ops.h"

namespace pd {
namespace attn {

constexpr float kLog2e = 1.44269504f, kLn2 = 0.693147181f;

// The hardware's base-2 exponential (1 ulp; results under 2^-126 are 0, which
// beside the row's largest term, 1, is below float32's rounding).
__device__ inline float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// A row's log of its sum, from the largest unscaled score, the scale and the sum of
// 2^(scores over the largest): the product is rounded as the backward pass rounds
// a score, so that a row with one large score finds p = 1 there.
__device__ inline float log_sum(float top, float scale, float total) {
    return total == 0.f ? -INFINITY : top * scale + log2f(total) * kLn2;
}

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4_u __attribute__((ext_vector_type(4), aligned(4)));
typedef bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef bf16x4 bf16x4_u __attribute__((aligned(2)));

template <typename T>
using Frag = typename Vec8<T>::type;

__device__ inline f32x16 mma(bf16x8 a, bf16x8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ inline f32x16 mma(f32x8 a, f32x8 b, f32x16 c) {
#pragma unroll
    for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b[e], c, 0, 0, 0);
    return c;
}
__device__ inline int tile_row(int lane, int r) { return 8 * (r >> 2) + 4 * (lane >> 5) + (r & 3); }

// registers 8c..8c+7 of a result as the next product's operand
__device__ inline f32x8 eight(const f32x16& v, int c) {
    f32x8 f;
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = v[8 * c + e];
    return f;
}
template <typename T>
__device__ inline Frag<T> as_frag(const f32x16& v, int c) {
    return narrow<T>(eight(v, c));
}

// A tile of rows in LDS: 16-byte units, those of row r exchanged by swz(r), so that the
// 16 units that a cycle reads lie in the 16 places of a 256-byte line: 16 rows at one
// unit (rows), and four rows at four neighbouring units or, in float32, two rows four
// apart at eight (cols).  Two rows of 128 bytes share a line.
template <typename T, int DP>
struct Tile {
    static constexpr int kPitch = (DP * (int)sizeof(T) + 127) / 128 * 128;   // bytes a row
    static constexpr int kUnits = DP * (int)sizeof(T) / 16;                  // units a row that hold values
    static __device__ inline int swz(int row) {
        if constexpr (kPitch % 256 != 0) return ((row & 2) << 1) | ((row >> 2) & 3);
        else if constexpr (sizeof(T) == 2) return ((row & 3) << 2) | ((row >> 2) & 3);
        else return ((row & 4) << 1) | ((row & 3) << 1) | ((row >> 3) & 1);
    }
    static __device__ inline int at(int row, int unit) { return row * kPitch + ((unit ^ swz(row)) << 4); }
    // rows row0 .. row0 + 31 of the tile as a fragment, step c of its 16-wide steps
    static __device__ inline Frag<T> rows(const char* lds, int row0, int c, int lane) {
        const int row = row0 + (lane & 31), h = lane >> 5;
        if constexpr (sizeof(T) == 2) {
            return *reinterpret_cast<const Frag<T>*>(lds + at(row, 2 * c + h));
        } else {
            const f32x4 a = *reinterpret_cast<const f32x4*>(lds + at(row, 4 * c + 2 * h));
            const f32x4 b = *reinterpret_cast<const f32x4*>(lds + at(row, 4 * c + 2 * h + 1));
            return Frag<T>{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
        }
    }
    // columns 32 dt .. 32 dt + 31 as the rows of a fragment, the tile's rows row0 .. row0
    // + 15 as its step, in the order of as_frag
    static __device__ inline Frag<T> cols(const char* lds, int row0, int dt, int lane) {
        const int h = lane >> 5;
        if constexpr (sizeof(T) == 2) {
            // the transposing read: of 16 lanes, 4j .. 4j + 3 point at 16 values of row j, and
            // lane i receives column i of the four rows
            const int i = lane & 15, row = row0 + 4 * h + (i >> 2);
            const int unit = 4 * dt + 2 * ((lane >> 4) & 1) + ((i & 3) >> 1);
            typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
            const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(lds + at(row, unit) + 8 * (i & 1)));
            const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(lds + at(row + 8, unit) + 8 * (i & 1)));
            typedef short s16x8 __attribute__((ext_vector_type(8)));
            return __builtin_bit_cast(Frag<T>, s16x8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]});
        } else {
            Frag<T> f;
            const int d = 32 * dt + (lane & 31);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int row = row0 + 8 * (e >> 2) + 4 * h + (e & 3);
                f[e] = *reinterpret_cast<const float*>(lds + at(row, d >> 2) + 4 * (d & 3));
            }
            return f;
        }
    }
    // eight values (chunk c of the row) into the tile
    static __device__ inline void put(char* lds, int row, int c, Frag<T> v) {
        if constexpr (sizeof(T) == 2) {
            *reinterpret_cast<Frag<T>*>(lds + at(row, c)) = v;
        } else {
            *reinterpret_cast<f32x4*>(lds + at(row, 2 * c)) = f32x4{v[0], v[1], v[2], v[3]};
            *reinterpret_cast<f32x4*>(lds + at(row, 2 * c + 1)) = f32x4{v[4], v[5], v[6], v[7]};
        }
    }
};

// ---------------------------------------------------------------- float32 in three parts
// A float32 value is the sum of three bfloat16 ones (8 bits each; exact but where the
// last falls under the smallest, for values under 2^-110), and a product of two such
// values that of six products, what is left out being under 2^-24: 6 x 32 cycles for
// 16 steps in place of 8 x 64, as accurate as float32's own instructions.  (An
// infinity splits into infinity and NaN: its rows are formed again from memory.)
struct Split {
    bf16x8 h, m, l;
};
__device__ __forceinline__ Split split(f32x8 x) {
    Split s;
    s.h = narrow<bf16>(x);
    const f32x8 r = x - widen(s.h);
    s.m = narrow<bf16>(r);
    s.l = narrow<bf16>(r - widen(s.m));
    return s;
}
__device__ __forceinline__ f32x16 mma(const Split& a, const Split& b, f32x16 c) {
    c = mma(a.l, b.h, c);
    c = mma(a.h, b.l, c);
    c = mma(a.m, b.m, c);
    c = mma(a.m, b.h, c);
    c = mma(a.h, b.m, c);
    return mma(a.h, b.h, c);
}

// The same with the operands exchanged: the bits that mma(b, a, .) gives at the turned
// place.
__device__ __forceinline__ f32x16 mma_turned(const Split& a, const Split& b, f32x16 c) {
    c = mma(a.h, b.l, c);
    c = mma(a.l, b.h, c);
    c = mma(a.m, b.m, c);
    c = mma(a.h, b.m, c);
    c = mma(a.m, b.h, c);
    return mma(a.h, b.h, c);
}
__device__ __forceinline__ f32x16 mma_turned(bf16x8 a, bf16x8 b, f32x16 c) { return mma(a, b, c); }

// How a kernel holds its operands: as they are, in tiles that copies fill, or in three
// parts, in three tiles that are filled through the registers.
template <typename T, int DP>
struct AsIs {
    using Type = T;
    using Operand = Frag<T>;
    static __device__ __forceinline__ Operand make(f32x8 v) { return narrow<T>(v); }
    static __device__ __forceinline__ Operand rows(const char* lds, int row0, int c, int lane) {
        return Tile<T, DP>::rows(lds, row0, c, lane);
    }
    static __device__ __forceinline__ Operand cols(const char* lds, int row0, int dt, int lane) {
        return Tile<T, DP>::cols(lds, row0, dt, lane);
    }
};
template <int DP, int ROWS>
struct InParts {
    using Type = float;
    using Operand = Split;
    using Ti = Tile<bf16, DP>;
    static constexpr int kPart = ROWS * Ti::kPitch, kBytes = 3 * kPart;
    static __device__ __forceinline__ Operand make(f32x8 v) { return split(v); }
    static __device__ __forceinline__ Operand rows(const char* lds, int row0, int c, int lane) {
        return Split{Ti::rows(lds, row0, c, lane), Ti::rows(lds + kPart, row0, c, lane), Ti::rows(lds + 2 * kPart, row0, c, lane)};
    }
    static __device__ __forceinline__ Operand cols(const char* lds, int row0, int dt, int lane) {
        return Split{Ti::cols(lds, row0, dt, lane), Ti::cols(lds + kPart, row0, dt, lane), Ti::cols(lds + 2 * kPart, row0, dt, lane)};
    }
    static __device__ __forceinline__ void put(char* lds, int row, int c, f32x8 v) {
        const Split s = split(v);
        Ti::put(lds, row, c, s.h);
        Ti::put(lds + kPart, row, c, s.m);
        Ti::put(lds + 2 * kPart, row, c, s.l);
    }
};

// Fills a tile in parts: 256 threads read its rows into registers (0 where `keep` is
// false and past the head's end) and, when the tile's place is free, split them there.
template <int DP, int ROWS>
struct FillParts {
    static constexpr int kUnits = ROWS * (DP / 8), kEach = (kUnits + 255) / 256;
    f32x8 v[kEach];
    template <class Keep>
    __device__ __forceinline__ void fetch(const float* base, int64_t stride, int head_dim, Keep keep) {
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int u = i * 256 + threadIdx.x, row = u / (DP / 8), e = u % (DP / 8) * 8;
            v[i] = f32x8{};
            if (u < kUnits && keep(row)) v[i] = load8(base + row * stride + e, head_dim - e);
        }
    }
    __device__ __forceinline__ void put(char* lds) const {
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int u = i * 256 + threadIdx.x;
            if (u < kUnits) InParts<DP, ROWS>::put(lds, u / (DP / 8), u % (DP / 8), v[i]);
        }
    }
};

// Runs COUNT products in order, each with a fragment from LDS: reads go G fragments at a
// time, a group ahead of the products, so that a group's latency passes behind the
// products of the one before.  (Left to itself the compiler reads a fragment just
// before its product and waits about 100 cycles for it, three times the product.)
template <class Operand, int COUNT>
struct Stream {
    // (four bfloat16 fragments; of three parts, whose product takes six, one)
    static constexpr int G = sizeof(Operand) > 16 ? 1 : COUNT < 4 ? COUNT : 4, kGroups = (COUNT + G - 1) / G;
    Operand f[2][G];
    template <class Read>
    __device__ __forceinline__ void read(int g, Read& r) {
#pragma unroll
        for (int i = 0; i < G; ++i)
            if (g * G + i < COUNT) f[g & 1][i] = r(g * G + i);
    }
    // the first group alone, ahead of other work
    template <class Read>
    __device__ __forceinline__ void begin(Read r) {
        read(0, r);
        __builtin_amdgcn_sched_barrier(0);
    }
    template <class Read, class Use>
    __device__ __forceinline__ void run(Read r, Use use) {
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            if (g + 1 < kGroups) read(g + 1, r);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < G; ++i)
                if (g * G + i < COUNT) use(g * G + i, f[g & 1][i]);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
};

// Four consecutive values of a result's column to memory, the first n of them.
__device__ inline void store4(float* p, int n, f32x4 v) {
    if (n >= 4) {
        *reinterpret_cast<f32x4_u*>(p) = v;
        return;
    }
#pragma unroll
    for (int e = 0; e < 3; ++e)
        if (e < n) p[e] = v[e];
}
__device__ inline void store4(bf16* p, int n, f32x4 v) {
    const bf16x4 w = __builtin_convertvector(v, bf16x4);
    if (n >= 4) {
        *reinterpret_cast<bf16x4_u*>(p) = w;
        return;
    }
#pragma unroll
    for (int e = 0; e < 3; ++e)
        if (e < n) p[e] = w[e];
}

// Consecutive blocks go to the 8 dies of the chip in turn; this numbers them so that
// each die, with its own L2, has a run of neighbours (blocks that read the same keys).
__device__ inline int near_blocks(int id, int count) {
    const int die = id & 7, at = id >> 3, each = count >> 3, more = count & 7;
    return die * each + min(die, more) + at;
}

// ---------------------------------------------------------------- memory to LDS
// One copy of 16 bytes a lane from base + off to LDS at lds + 16 lane, past the
// registers (M0 = lds).  Inline assembly, so that the compiler's wait counts do not
// see it (it would wait for the copies before every LDS read): who reads the data
// waits with wait_copies() and a barrier first.  The hardware does not wait by itself for
// what a copy reads: M0 must be a wait state old, an address that a vector instruction
// (readfirstlane) wrote to scalar registers five.  The compiler sees to that between
// instructions of its own, but not where one of them is in a string: hence the s_nop.
__device__ __forceinline__ uint64_t uniform_address(const void* p) {
    const uint64_t v = (uint64_t)(uintptr_t)p;
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v);
    const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
    uint64_t u = ((uint64_t)hi << 32) | lo;
    asm("s_nop 4" : "+s"(u));
    return u;
}
__device__ __forceinline__ void copy16(uint64_t base, uint32_t off, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %2\n\t"
                 "s_nop 0\n\t"
                 "global_load_lds_dwordx4 %0, %1"
                 :
                 : "v"(off), "s"(base), "s"(lds)
                 : "memory", "m0");
}
__device__ __forceinline__ void wait_copies() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
__device__ __forceinline__ uint32_t lds_address(const char* p) {
    return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char*)p;
}
// Barrier for LDS traffic alone: copies and stores to memory may be in flight.
__device__ __forceinline__ void lds_barrier() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// Fills a tile of ROWS rows with THREADS threads.  Copies need rows and their stride aligned
// to 16 bytes, a head of whole 16-byte units, and ROWS rows within 2^31 bytes;
// the host says whether that holds (copies_fit).  Units past the head's end repeat
// its first one: what they meet is zero (queries) or not stored (output columns).
// (Copies, and the same through registers, which takes any alignment: 8192 tokens with a
// window 283 and 523 us, backward on latents 385 and 624 us, the next token of 16 sequences
// 178 and 580 us.)
template <typename T, int DP, int ROWS, int THREADS, bool ONE = false>
struct Fill {
    using Ti = Tile<T, DP>;
    static constexpr int kRowUnits = Ti::kPitch / 16;
    static constexpr int kCopies = ROWS * kRowUnits / THREADS;
    static constexpr int kStep = THREADS / kRowUnits;         // rows from a thread's copy to its next
    // ONE: one offset a thread instead of one a copy, for a kernel without registers to
    // spare.  swz repeats every 16 rows: copies that are so far apart differ by rows alone,
    // which the scalar base can say (two instructions a copy more).
    static constexpr bool kOne = ONE;
    static_assert(!ONE || kStep % 16 == 0, "copies at whole periods of swz");
    static_assert(ROWS * kRowUnits % THREADS == 0 && THREADS % 64 == 0, "whole copies");
    uint32_t off[kOne ? 1 : kCopies];      // of this thread's copies from the tile's first row
    uint32_t step;                         // bytes from row to row
    uint32_t to;                           // this wave's part of a tile, from its start
    __device__ __forceinline__ void plan(int64_t stride, int units, int thread) {
        step = (uint32_t)stride * (uint32_t)sizeof(T);
#pragma unroll
        for (int i = 0; i < (kOne ? 1 : kCopies); ++i) {
            const int at = i * THREADS + thread, row = at / kRowUnits;
            const int unit = (at % kRowUnits) ^ Ti::swz(row);
            off[i] = (uint32_t)row * step + (unit < units ? unit : 0) * 16;
        }
        to = __builtin_amdgcn_readfirstlane((thread & ~63) * 16);
    }
    // the tile whose first row is at `base`
    __device__ __forceinline__ void copy(const T* base, const char* lds) const {
        const uint64_t from = uniform_address(base);
        const uint32_t at = __builtin_amdgcn_readfirstlane(lds_address(lds) + to);
#pragma unroll
        for (int i = 0; i < kCopies; ++i)
            copy16(kOne ? from + (uint32_t)(i * kStep) * step : from, off[kOne ? 0 : i], at + i * THREADS * 16);
    }
    // the same, but its row r from the row that source(r) names
    template <class Source>
    __device__ __forceinline__ void copy_some(const T* base, const char* lds, int thread, Source source) const {
        const uint64_t from = uniform_address(base);
        const uint32_t at = __builtin_amdgcn_readfirstlane(lds_address(lds) + to);
#pragma unroll
        for (int i = 0; i < kCopies; ++i) {
            const int row = (i * THREADS + thread) / kRowUnits, mine = kOne ? thread / kRowUnits : row;
            copy16(from, off[kOne ? 0 : i] + (uint32_t)(source(row) - mine) * step, at + i * THREADS * 16);
        }
    }
    // the same through registers, any stride and alignment; rows for which `keep` is
    // false and values past the head's end are 0
    template <class Keep>
    static __device__ __forceinline__ void load(const T* base, int64_t stride, int head_dim, char* lds, int thread, Keep keep) {
        for (int u = thread; u < ROWS * (DP / 8); u += THREADS) {
            const int row = u / (DP / 8), c = u % (DP / 8);
            Frag<T> v = {};
            if (keep(row)) v = load8(base + row * stride + 8 * c, head_dim - 8 * c);
            Ti::put(lds, row, c, v);
        }
    }
};
inline bool copies_fit(const void* p, const int64_t* stride, int64_t batch, int64_t tokens, int64_t heads, int head_dim, int elem) {
    const int64_t count[3] = {batch, tokens, heads};       // (a stride over one element is never taken)
    for (int i = 0; i < 3; ++i)
        if (count[i] > 1 && stride[i] * elem % 16) return false;
    return (uintptr_t)p % 16 == 0 && head_dim * elem % 16 == 0 && (tokens <= 1 || stride[1] * elem < (1 << 24));
}

// ---------------------------------------------------------------- who sees what
// One sequence: n queries at t = m - n + i, m keys.
struct Seq {
    int n, m;
};
__device__ inline Seq sequence(const AttentionArgs& a, int b) {
    Seq s{a.d.q_len, a.d.kv_len};
    if (a.q_lens) s.n = min(max(a.q_lens[b], 0), a.d.q_len);
    if (a.kv_lens) s.m = min(max(a.kv_lens[b], 0), a.d.kv_len);
    return s;
}
// The keys that a query sees: lo <= j < hi, or j < sk.  (The host has made a window
// that limits nothing 0, so no sum here passes 2^31.)
struct See {
    int lo, hi, sk;
    __device__ inline bool operator()(int j) const { return (j >= lo && j < hi) || j < sk; }
    __device__ inline bool none() const { return hi <= lo && sk <= 0; }
    // for a lane that asks about tile_row(lane, r) = tile_row(0, r) + 4 (lane / 32): the same with
    // keys counted from 4 (lane / 32), so that the question is one of a uniform number
    __device__ inline See from(int lane) const {
        const int h4 = 4 * (lane >> 5);
        return See{lo - h4, hi - h4, sk - h4};
    }
};
__device__ inline See sees(const pd_attention_desc& d, const Seq& s, int i) {
    if (i >= s.n) return See{0, 0, 0};
    const int t = s.m - s.n + i;
    const int end = d.causal ? min(s.m, max(t + 1, 0)) : s.m;     // the last key that order allows
    if (!d.window) return See{0, end, 0};
    return See{max(t - d.window + 1, 0), min(end, max(t + d.window, 0)), min(d.sinks, end)};
}
// Union over the queries i0 .. i1 (both < s.n).
__device__ inline See sees_any(const pd_attention_desc& d, const Seq& s, int i0, int i1) {
    const See a = sees(d, s, i0), b = sees(d, s, i1);
    return See{a.lo, b.hi, b.sk};
}

// The tiles of BN keys that hold the union `any` of a set of rows: first those of the
// sinks, then those of the window, each once.
template <int BN>
struct KeyTiles {
    See any;
    int sinks, first, count;
    __device__ inline explicit KeyTiles(const See& see) : any(see) {
        sinks = (any.sk + BN - 1) / BN;
        first = max(any.lo / BN, sinks);
        count = sinks + max((any.hi + BN - 1) / BN, first) - first;
    }
    __device__ inline int start(int it) const { return (it < sinks ? it : first + it - sinks) * BN; }
    // every key of the tile at j0 is in the union
    __device__ inline bool whole(int j0) const { return (j0 >= any.lo && j0 + BN <= any.hi) || j0 + BN <= any.sk; }
    // a key of the tile at j0 that is in the union: j itself where it is
    __device__ inline int inside(int j0, int j) const {
        if (any(j)) return j;
        const int lo = max(any.lo, j0), hi = min(any.hi, j0 + BN);
        return lo < hi ? min(max(j, lo), hi - 1) : min(any.sk, j0 + BN) - 1;
    }
};
// What a wave's rows see between them: the smallest and the largest bounds, so that a
// tile of keys can be told to be in sight of all rows or of none.
struct Sight {
    int lo_min, lo_max, hi_min, hi_max, sk_min, sk_max;
    __device__ inline bool all(int j0, int n) const { return (j0 >= lo_max && j0 + n <= hi_min) || j0 + n <= sk_min; }
    __device__ inline bool none(int j0, int n) const { return (j0 >= hi_max || j0 + n <= lo_min) && j0 >= sk_max; }
};
// Of the queries i0 .. i1, whose bounds grow with i; a query past s.n sees nothing.
__device__ inline Sight sight_of(const pd_attention_desc& d, const Seq& s, int i0, int i1) {
    if (i0 >= s.n) return Sight{0, 0, 0, 0, 0, 0};
    const See a = sees(d, s, i0), b = sees(d, s, min(i1, s.n - 1));
    const bool whole = i1 < s.n;
    return Sight{a.lo, b.lo, whole ? a.hi : 0, b.hi, whole ? a.sk : 0, b.sk};
}

// rows of a shared tile: two buffers of two tiles stay within half a compute unit's LDS
template <typename T, int DP>
constexpr int tile_rows() {
    return Tile<T, DP>::kPitch <= 256 ? 64 : 32;
}

}  // namespace attn
}  // namespace pd
