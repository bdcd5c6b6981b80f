// The gated product of a feed-forward block, forward and backward.
//
//   g = x Wg, u = x Wu, h = act(g) u
//   dg = dh u act'(g), du = dh act(g);  dx = dg Wg^T + du Wu^T,  dWg = x^T dg, dWu = x^T du
//
// All products run in one kernel (k_product) over bfloat16 operands: blocks of BM rows
// and twice HN columns, the two halves being gate and up, or neighbours of one matrix.
// Operands are read as they lie, along the sum (units of a row are fragments) or across
// it (transposing LDS reads).  float32 operands are split into three bfloat16 parts first,
// and the six products of parts that count are six segments of the sum, small ones first;
// dg and du of bfloat16 are two parts, and their products two segments.
// Operands that copies of 16 bytes cannot read (alignment, odd sizes) are laid out first.
// Few rows forward (up to 64 or 128) go to a kernel of their own (k_gated_few).
//
// What bounds it: the matrix units (a 32 x 32 x 16 product takes 32 cycles, and a wave of
// 128 x 128 results issues 64 of them a step), with one wave a SIMD that has to find everything
// else in their shadow.  So the next step's fragments are read, and the copies of the step
// after it sent, between products; a block goes from tile to tile, whose first steps come while
// the last one's results go; products are formed transposed, so that results leave from the
// registers in rows of 16 bytes.  What has no shadow is a tile's results: activation,
// rounding, stores.
//
// Measured (bfloat16, silu): 8192 x 4096 x 4096 435 to 440 us (1250 to 1265 TFLOP/s; a large
// library product reaches 1228), where a tile has 64 steps; 36864 x 1024 x 4096 580 us (1065;
// the library's product of x with both weights side by side, without the rest, 552), where it
// has 16 and results take a quarter of a tile; with gelu 630.  Matrix units busy 44% of the
// cycles there, vector units 29, no bank conflicts.  Gradients of 9216 x 1024 x 2736 534 to 556 us
// (372 to 387, and twice that executed, as dgate and dup have two parts), of which dgate and dup 55 (6.4 TB/s); float32 4096 x 1024 x 2736 272 us (169; the library's
// float32 products 154).
#include "attention_tile.h"

namespace pd {
namespace {

using namespace attn;

constexpr int kSegs = 12;                // the sum's segments: 6 in float32, twice as many for dx

struct Product {
    // segment s: a[s] times b0[s] (first half of the columns) and b1[s] (second)
    const bf16* a[kSegs];
    const bf16* b0[kSegs];
    const bf16* b1[kSegs];
    int64_t lda, ldb;
    int64_t a_group;                     // elements between the a of one group and the next
    int segs, k, steps;                  // steps of the form's BK a segment
    int m, n;                            // rows, and columns of a half's matrix
    int apart;                           // the halves are two matrices (else neighbours in one)
    int tiles_m, tiles_n, groups, splits;
    int act;
    void* c[2];                          // by half if apart, else by group; gated: c[0] is h
    int64_t ldc[2];
    void* gate;                          // gated only
    void* up;
    int64_t ld_gate, ld_up;
    float* partial;                      // [splits][c's matrices][m][n]
};

// ------------------------------------------------------------------ activations
// From the hardware's 2^x and 1/x (1 ulp each); with the math library's functions and
// divisions a tile's results took about as long as its products over 1024 values.
// FINE (float32 results): e^x with what the product x log2 e leaves out, 2^-24 |x| of it.
template <bool FINE>
__device__ __forceinline__ float e_to(float x) {
    const float t = x * kLog2e, e = exp2_fast(t);
    if constexpr (!FINE) return e;
    const float rest = fmaf(x, 1.92596299e-8f, fmaf(x, kLog2e, -t));       // log2 e = kLog2e + 1.926e-8
    return fabsf(t) < 127.f ? fmaf(e, rest * kLn2, e) : e;                 // (else near 0, or infinity)
}
template <bool FINE>
__device__ __forceinline__ float sigmoid(float x) {
    return __builtin_amdgcn_rcpf(1.f + e_to<FINE>(-x));
}
// e^(-g^2 / 2).  FINE: with what g^2 leaves out, 2^-25 g^2 of it (4e-6 at 12).
template <bool FINE>
__device__ __forceinline__ float bell(float g) {
    const float s = g * g, e = e_to<FINE>(-0.5f * s);
    if constexpr (!FINE) return e;
    return e == 0.f ? 0.f : fmaf(e, -0.5f * fmaf(g, g, -s), e);            // (past 0 g^2 may be infinite)
}
// The normal distribution's part past |g|: for x = |g| / sqrt 2, erfc(x) / 2 = e^(-x^2) t Q(t) with
// t = 1 / (1 + c x); Q is fitted to e^(x^2) erfc(x) / 2t over 0 <= x <= 10 (past it the exponential is
// 0): with relative errors up to 2e-8 for float32 results, 9e-6 for bfloat16.  The tail itself is
// off by 5e-7 of it at most in float32, and by 9e-6 + 2^-23 g^2 / 2 for bfloat16 results.
template <bool FINE>
__device__ __forceinline__ float normal_past(float g) {
    if constexpr (FINE) {
        const float t = __builtin_amdgcn_rcpf(fmaf(fabsf(g), 0.212132034f, 1.f));        // (c = 0.3)
        float q = -0.06476157f;
        q = fmaf(q, t, 0.242782207f);
        q = fmaf(q, t, -0.256140369f);
        q = fmaf(q, t, 0.273861635f);
        q = fmaf(q, t, -0.0473265675f);
        q = fmaf(q, t, 0.107463585f);
        q = fmaf(q, t, 0.0741694301f);
        q = fmaf(q, t, 0.0853576373f);
        q = fmaf(q, t, 0.0845940011f);
        return bell<true>(g) * (q * t);
    } else {
        const float t = __builtin_amdgcn_rcpf(fmaf(fabsf(g), 0.318198052f, 1.f));        // (c = 0.45)
        float q = -0.0674448580f;
        q = fmaf(q, t, 0.144600437f);
        q = fmaf(q, t, 0.0465514324f);
        q = fmaf(q, t, 0.123206058f);
        q = fmaf(q, t, 0.126125300f);
        q = fmaf(q, t, 0.126957110f);
        return exp2_fast(g * g * -0.721347520f) * (q * t);
    }
}
// 2 sqrt(2/pi) (g + 0.044715 g^3), of which gelu's tanh form takes the sigmoid
__device__ __forceinline__ float twice_inner(float g) { return 1.59576912f * fmaf(0.044715f * g * g, g, g); }
// largest of g and 0, or NaN
__device__ __forceinline__ float positive(float g) { return g > 0.f ? g : (g != g ? g : 0.f); }

template <class V, class F>
__device__ __forceinline__ V each(V g, F f) {
#pragma unroll
    for (int e = 0; e < (int)(sizeof(V) / 4); ++e) g[e] = f(g[e]);
    return g;
}
template <bool FINE, class V>
__device__ __forceinline__ V activate(int act, V g) {
    switch (act) {
        case PD_ACT_SILU: return each(g, [](float v) { return v * sigmoid<FINE>(v); });
        case PD_ACT_GELU:
            return each(g, [](float v) {
                const float tail = normal_past<FINE>(v);
                return v * (v < 0.f ? tail : 1.f - tail);
            });
        case PD_ACT_GELU_TANH: return each(g, [](float v) { return v * sigmoid<FINE>(twice_inner(v)); });
        case PD_ACT_SIGMOID: return each(g, [](float v) { return sigmoid<FINE>(v); });
        default: return each(g, [](float v) { return positive(v); });
    }
}
// act and its slope
template <bool FINE>
__device__ __forceinline__ void activate_grad(int act, f32x8 g, f32x8& a, f32x8& slope) {
    switch (act) {
        case PD_ACT_SILU:
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float s = sigmoid<FINE>(g[e]);
                a[e] = g[e] * s;
                slope[e] = s * fmaf(g[e], 1.f - s, 1.f);
            }
            return;
        case PD_ACT_GELU:
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float tail = normal_past<FINE>(g[e]), p = g[e] < 0.f ? tail : 1.f - tail, d = bell<FINE>(g[e]);
                a[e] = g[e] * p;
                slope[e] = d == 0.f ? p : fmaf(g[e], d * 0.398942280f, p);
            }
            return;
        case PD_ACT_GELU_TANH:
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float s = sigmoid<FINE>(twice_inner(g[e])), d = s * (1.f - s);
                a[e] = g[e] * s;
                slope[e] = d == 0.f ? s : fmaf(g[e] * d, 1.59576912f * fmaf(0.134145f * g[e], g[e], 1.f), s);
            }
            return;
        case PD_ACT_SIGMOID:
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                a[e] = sigmoid<FINE>(g[e]);
                slope[e] = a[e] * (1.f - a[e]);
            }
            return;
        default:
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                a[e] = positive(g[e]);
                slope[e] = g[e] > 0.f ? 1.f : (g[e] != g[e] ? g[e] : 0.f);
            }
    }
}

// ------------------------------------------------------------------ copies
// What lanes past the sum's end copy.
__device__ const __attribute__((aligned(16))) float kZeros[4] = {0.f, 0.f, 0.f, 0.f};

// One copy of 16 bytes a lane from an address of its own.
__device__ __forceinline__ void copy16_from(const void* p, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %1\n\t"
                 "s_nop 0\n\t"
                 "global_load_lds_dwordx4 %0, off"
                 :
                 : "v"(p), "s"(lds)
                 : "memory", "m0");
}

// A tile of ROWS rows of UNITS units of 16 bytes, copied by 256 threads.  ACROSS: its rows
// run along the sum, else its units do.  Units of row r are exchanged by swz(r), so that
// what a cycle reads (16 rows at one unit; ACROSS: four rows at four neighbouring units)
// lies in the 16 places of a 256-byte line, which 4, 2 or 1 rows share.
template <int ROWS, int UNITS, bool ACROSS>
struct Operand {
    static constexpr int kPitch = UNITS * 16;
    static __device__ __forceinline__ int swz(int row) {
        if constexpr (UNITS == 4) return (row >> 2) & 3;
        else if constexpr (UNITS % 16 == 8) return ((row & 2) << 1) | ((row >> 2) & 3);    // (neighbours half a line apart)
        else return ((row & 3) << 2) | ((row >> 2) & 3);
    }
    static __device__ __forceinline__ int place(int row, int unit) { return row * kPitch + ((unit ^ swz(row)) << 4); }
    static constexpr int kCopies = ROWS * UNITS / 256, kBytes = ROWS * UNITS * 16;
    static_assert(ROWS * UNITS % 256 == 0, "whole copies");
    uint32_t off[kCopies];                 // from the tile's first element
    uint32_t to;
    static __device__ __forceinline__ int row_of(int i, int thread) { return (i * 256 + thread) / UNITS; }
    static __device__ __forceinline__ int unit_of(int i, int thread) {
        return ((i * 256 + thread) % UNITS) ^ swz(row_of(i, thread));
    }
    // `left` rows (ACROSS: columns) of the matrix from the tile's first on; copies past
    // them repeat the last: what they meet is not stored
    __device__ __forceinline__ void plan(int64_t stride, int left, int thread) {
#pragma unroll
        for (int i = 0; i < kCopies; ++i) {
            int row = row_of(i, thread), unit = unit_of(i, thread);
            if (ACROSS) unit = min(unit, (left + 7) / 8 - 1);
            else row = min(row, left - 1);
            off[i] = (uint32_t)row * (uint32_t)stride * 2 + unit * 16;
        }
        to = __builtin_amdgcn_readfirstlane((thread & ~63) * 16);
    }
    // copy i of the tile at `base` (from uniform_address) to `lds` (from lds_address)
    __device__ __forceinline__ void copy(int i, uint64_t base, uint32_t lds) const { copy16(base, off[i], lds + to + i * 4096); }
    // the whole tile, of whose values along the sum only `k` are left: zeros past them
    __device__ __forceinline__ void copy_end(const bf16* base, uint32_t lds, int k, int thread) const {
#pragma unroll
        for (int i = 0; i < kCopies; ++i) {
            const bool real = ACROSS ? row_of(i, thread) < k : unit_of(i, thread) * 8 < k;
            copy16_from(real ? reinterpret_cast<const char*>(base) + off[i] : reinterpret_cast<const char*>(kZeros), lds + to + i * 4096);
        }
    }
    // rows (ACROSS: columns) 32 t .. 32 t + 31 as a fragment, step c of 16: lane l has
    // row l % 32 and of the step the eight values from 8 (l / 32)
    static __device__ __forceinline__ bf16x8 read(const char* lds, int t, int c, int lane) {
        if constexpr (!ACROSS) {
            return *reinterpret_cast<const bf16x8*>(lds + place(32 * t + (lane & 31), 2 * c + (lane >> 5)));
        } else {
            const int i = lane & 15, row = 16 * c + 8 * (lane >> 5) + (i >> 2);
            const int unit = 4 * t + 2 * ((lane >> 4) & 1) + ((i & 3) >> 1);
            typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
            const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(lds + place(row, unit) + 8 * (i & 1)));
            const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(lds + place(row + 4, unit) + 8 * (i & 1)));
            typedef short s16x8 __attribute__((ext_vector_type(8)));
            return __builtin_bit_cast(bf16x8, s16x8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]});
        }
    }
};

// ------------------------------------------------------------------ the product
enum Out { kGated, kStore, kPartial };

// Waits for all copies but the last n; then the barrier: LDS may be read where older copies
// went, and written where it was read.
template <int N>
__device__ __forceinline__ void wait_copies_but() {
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// Of a transposed product's registers 8 p .. 8 p + 7, in bfloat16: lanes 0 .. 31 get the
// eight neighbouring columns from 16 p on, lanes 32 .. 63 those from 16 p + 8 on.
__device__ __forceinline__ bf16x8 eight_neighbours(const f32x16& v, int p) {
    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    const f32x4 lo = {v[8 * p], v[8 * p + 1], v[8 * p + 2], v[8 * p + 3]}, hi = {v[8 * p + 4], v[8 * p + 5], v[8 * p + 6], v[8 * p + 7]};
    const u32x2 a = __builtin_bit_cast(u32x2, __builtin_convertvector(lo, bf16x4));
    const u32x2 b = __builtin_bit_cast(u32x2, __builtin_convertvector(hi, bf16x4));
    const auto s = __builtin_amdgcn_permlane32_swap(a[0], b[0], false, false), t = __builtin_amdgcn_permlane32_swap(a[1], b[1], false, false);
    return __builtin_bit_cast(bf16x8, u32x4{s[0], t[0], s[1], t[1]});
}

// WM x 4/WM waves of 32 MT rows and in each half 16 NT columns; BK values along the sum a
// step, of which BUFS steps are in LDS or on the way.
template <int MT, int NT, int WM, int BK, int BUFS>
struct Form {
    static constexpr int kMT = MT, kNT = NT, kWM = WM, kBK = BK, kBufs = BUFS;
    static constexpr int BM = 32 * MT * WM, HN = 16 * NT * (4 / WM);
    static constexpr int kBlocks = MT * NT > 8 ? 1 : 2;        // a compute unit
};
template <class F, bool AC, bool BC, Out OUT, typename TO>
__global__ __launch_bounds__(256, F::kBlocks) void k_product(const Product p) {
    constexpr int MT = F::kMT, NT = F::kNT, WM = F::kWM, BK = F::kBK, BUFS = F::kBufs;
    constexpr int WN = 4 / WM, BM = F::BM, HT = NT / 2, HN = F::HN, KS = BK / 16;
    using A = std::conditional_t<AC, Operand<BK, BM / 8, true>, Operand<BM, BK / 8, false>>;
    using B = std::conditional_t<BC, Operand<BK, HN / 8, true>, Operand<HN, BK / 8, false>>;
    constexpr int kBuffer = A::kBytes + 2 * B::kBytes, kCopies = A::kCopies + 2 * B::kCopies;
    constexpr int kCols = 32 * HT;                               // of a wave, in each half
    __shared__ __attribute__((aligned(256))) char lds[BUFS * kBuffer];
    const int thread = threadIdx.x, lane = thread & 63, wave = __builtin_amdgcn_readfirstlane(thread >> 6);
    const int wm = wave / WN, wn = wave % WN;
    const uint32_t lds0 = lds_address(lds);
    const int per = p.tiles_m * p.tiles_n, tiles = per * p.groups * p.splits;
    // a tile of the block's: which split and group, its first row and columns, its steps
    int z, group, m0, n0, n1, first, last;
    // the next step to copy: its segment, where in it, its operands, where to
    int fill_t, fill_s, fill_k, fill_at;
    uint64_t ua, ub0, ub1;
    const uint64_t step_a = (AC ? p.lda : 1) * (BK * 2), step_b = (BC ? p.ldb : 1) * (BK * 2);
    bool two;
    A a;
    B b0, b1;
    // neighbours on a die share rows of a and columns of b
    const auto take = [&](int tile) {
        int id = near_blocks(tile, tiles);
        z = id / (per * p.groups);
        id -= z * per * p.groups;
        group = id / per;
        id -= group * per;
        constexpr int kStrip = 8;
        const int strip = id / (kStrip * p.tiles_n), in = id - strip * kStrip * p.tiles_n;
        const int high = min(kStrip, p.tiles_m - strip * kStrip);
        m0 = (strip * kStrip + in % high) * BM;
        n0 = in / high * (p.apart ? HN : 2 * HN);
        n1 = p.apart ? n0 : n0 + HN;
        const int all = p.segs * p.steps;
        first = (int)((int64_t)all * z / p.splits);
        last = (int)((int64_t)all * (z + 1) / p.splits);
        a.plan(p.lda, p.m - m0, thread);
        b0.plan(p.ldb, p.n - n0, thread);
        two = n1 < p.n;                                          // (else the second half repeats the first)
        b1.plan(p.ldb, two ? p.n - n1 : p.n - n0, thread);
        fill_t = first;
        fill_s = first / p.steps;
        fill_k = (first - fill_s * p.steps) * BK;
        fill_at = 0;
    };
    // The operands' addresses stay in scalar registers from step to step: reading the segment's
    // from memory for each took a tenth of a step.
    const auto aim = [&] {
        const int n = two ? n1 : n0;
        ua = uniform_address(p.a[fill_s] + group * p.a_group + (AC ? (int64_t)fill_k * p.lda + m0 : (int64_t)m0 * p.lda + fill_k));
        ub0 = uniform_address(p.b0[fill_s] + (BC ? (int64_t)fill_k * p.ldb + n0 : (int64_t)n0 * p.ldb + fill_k));
        ub1 = uniform_address(p.b1[fill_s] + (BC ? (int64_t)fill_k * p.ldb + n : (int64_t)n * p.ldb + fill_k));
    };
    uint32_t to = 0;
    // the next step's copies are done with
    const auto advance = [&] {
        ++fill_t;
        fill_at = fill_at + 1 == BUFS ? 0 : fill_at + 1;
        fill_k += BK;
        ua += step_a, ub0 += step_b, ub1 += step_b;
        if (fill_k >= p.steps * BK) {
            fill_k = 0;
            ++fill_s;
            if (fill_t < last) aim();
        }
    };
    // begins a step's copies; true: copy(i) does them one by one, then advance() (else they are
    // done here)
    const auto begin = [&]() -> bool {
        to = __builtin_amdgcn_readfirstlane(lds0 + fill_at * kBuffer);
        const int k = p.k - fill_k;
        if (k >= BK) return true;
        a.copy_end(reinterpret_cast<const bf16*>(ua), to, k, thread);
        b0.copy_end(reinterpret_cast<const bf16*>(ub0), to + A::kBytes, k, thread);
        b1.copy_end(reinterpret_cast<const bf16*>(ub1), to + A::kBytes + B::kBytes, k, thread);
        advance();
        return false;
    };
    const auto copy = [&](int i) {
        if (i < A::kCopies) a.copy(i, ua, to);
        else if (i < A::kCopies + B::kCopies) b0.copy(i - A::kCopies, ub0, to + A::kBytes);
        else b1.copy(i - A::kCopies - B::kCopies, ub1, to + A::kBytes + B::kBytes);
    };
    const auto fill_all = [&] {
        aim();
#pragma unroll 1
        for (int i = 0; i < BUFS; ++i)
            if (fill_t < last && begin()) {
#pragma unroll
                for (int j = 0; j < kCopies; ++j) copy(j);
                advance();
            }
    };
    take(blockIdx.x);
    fill_all();
    wait_copies();
    for (int tile = blockIdx.x;;) {
        // here the tile's first steps have come
        lds_barrier();
        f32x16 acc[MT][NT];
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j) acc[i][j] = f32x16{};
        bf16x8 fa[2][MT], fb[2][NT];
        const auto read = [&](const char* from, int c, int to, int i) {      // fragment i of step c
            if (i < MT) fa[to][i] = A::read(from, wm * MT + i, c, lane);
            else fb[to][i - MT] = B::read(from + A::kBytes + ((i - MT) / HT) * B::kBytes, wn * HT + (i - MT) % HT, c, lane);
        };
#pragma unroll
        for (int i = 0; i < MT + NT; ++i) read(lds, 0, 0, i);
        int now = 0;
#pragma unroll 1
        for (int t = first; t < last; ++t) {
            const char* here = lds + now * kBuffer;
            now = now + 1 == BUFS ? 0 : now + 1;
            const char* next = lds + now * kBuffer;
#pragma unroll
            for (int c = 0; c < KS; ++c) {
                bool more = false;
                if (c == KS - 1) {
                    // this step's fragments are all in registers, its place is free; the next one's must be there
                    if (t + BUFS <= last) wait_copies_but<(BUFS - 2) * kCopies>();
                    else wait_copies();
                    lds_barrier();
                    if (fill_t < last) more = begin();
                }
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = 0; i < MT * NT; ++i) {
                    acc[i / NT][i % NT] = mma(fb[c & 1][i % NT], fa[c & 1][i / NT], acc[i / NT][i % NT]);
                    // under the products: the next fragments, and the next copies
                    if (i < MT + NT) read(c == KS - 1 ? next : here, c == KS - 1 ? 0 : c + 1, (c + 1) & 1, i);
                    if (c == KS - 1 && i < kCopies && more) copy(i);
                    __builtin_amdgcn_sched_barrier(0);
                }
                if (c == KS - 1 && more) {
#pragma unroll
                    for (int i = MT * NT; i < kCopies; ++i) copy(i);
                    advance();
                }
#pragma unroll
                for (int i = MT * NT; i < MT + NT; ++i) read(c == KS - 1 ? next : here, c == KS - 1 ? 0 : c + 1, (c + 1) & 1, i);
            }
        }
        lds_barrier();
        // the next tile's first steps come while this one's results go
        const int row0 = m0 + wm * MT * 32, at_z = z, at_group = group, at_n0 = n0 + wn * kCols, at_n1 = n1 + wn * kCols;
        tile += gridDim.x;
        const bool go_on = tile < tiles;
        if (go_on) {
            take(tile);
            fill_all();
        }
        // results: the products are formed transposed, so lane l has row l % 32 and in registers
        // 4 q .. 4 q + 3 columns 8 q + 4 (l / 32) ..; for bfloat16 halves of the wave exchange
        // two such fours
        constexpr int kSpan = sizeof(TO) == 2 ? 8 : 4;           // values a store: 16 bytes
        const int lane_row = row0 + (lane & 31), lane_col = kSpan * (lane >> 5);
        const auto emit = [&](const f32x16& v, int i, int j, TO* to, int64_t ld, int at) {
            TO* mine = to + lane_row * ld + (at + lane_col) + 32 * i * ld + 32 * j;
#pragma unroll
            for (int s = 0; s < 16 / kSpan; ++s) {
                const int left = p.n - at - lane_col - 32 * j - 2 * kSpan * s;
                const bool real = lane_row + 32 * i < p.m && left > 0;
                if constexpr (sizeof(TO) == 2) {
                    const bf16x8 w = eight_neighbours(v, s);     // (all lanes)
                    if (real) store8(mine + 2 * kSpan * s, left, w);
                } else if (real) {
                    store4(mine + 2 * kSpan * s, left, f32x4{v[4 * s], v[4 * s + 1], v[4 * s + 2], v[4 * s + 3]});
                }
            }
        };
#pragma unroll
        for (int i = 0; i < MT; ++i) {
#pragma unroll
            for (int j = 0; j < HT; ++j) {
                const f32x16 v0 = acc[i][j], v1 = acc[i][j + HT];
                if constexpr (OUT == kGated) {
                    if (p.gate) emit(v0, i, j, static_cast<TO*>(p.gate), p.ld_gate, at_n0);
                    if (p.up) emit(v1, i, j, static_cast<TO*>(p.up), p.ld_up, at_n0);
                    emit(activate<sizeof(TO) == 4>(p.act, v0) * v1, i, j, static_cast<TO*>(p.c[0]), p.ldc[0], at_n0);
                } else {
                    const int h0 = p.apart ? 0 : at_group, h1 = p.apart ? 1 : at_group;
                    if constexpr (OUT == kStore) {
                        emit(v0, i, j, static_cast<TO*>(p.c[h0]), p.ldc[h0], at_n0);
                        emit(v1, i, j, static_cast<TO*>(p.c[h1]), p.ldc[h1], at_n1);
                    } else {
                        const int64_t size = (int64_t)p.m * p.n, count = p.apart ? 2 : p.groups;
                        emit(v0, i, j, p.partial + (at_z * count + h0) * size, p.n, at_n0);
                        emit(v1, i, j, p.partial + (at_z * count + h1) * size, p.n, at_n1);
                    }
                }
                __builtin_amdgcn_sched_barrier(0);               // (one tile's results in registers at a time)
            }
            // (the copies have had time, the stores to come are not waited for)
            if (i == (MT - 1) / 2) wait_copies();
        }
        if (!go_on) return;
    }
}

// The splits' sums together, in their order, and what comes after them: eight columns a
// lane.
template <bool GATED, typename TO>
__global__ __launch_bounds__(256) void k_product_join(const Product p) {
    const int per = (p.n + 7) / 8;
    const int64_t size = (int64_t)p.m * p.n, each = (p.apart ? 2 : p.groups) * size;
    const int64_t units = (int64_t)p.m * per, count = GATED ? units : (p.apart ? 2 : p.groups) * units;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < count; i += (int64_t)gridDim.x * 256) {
        const int64_t matrix = i / units, in = i - matrix * units, row = in / per;
        const int at = (int)(in - row * per) * 8, n = p.n - at;
        const float* from = p.partial + matrix * size + row * p.n + at;
        f32x8 v0 = {}, v1 = {};
#pragma unroll 4
        for (int z = 0; z < p.splits; ++z) {
            v0 += load8(from + z * each, n);
            if (GATED) v1 += load8(from + z * each + size, n);
        }
        if constexpr (GATED) {
            const f32x8 h = activate<sizeof(TO) == 4>(p.act, v0) * v1;
            store8(static_cast<TO*>(p.c[0]) + row * p.ldc[0] + at, n, narrow<TO>(h));
            if (p.gate) store8(static_cast<TO*>(p.gate) + row * p.ld_gate + at, n, narrow<TO>(v0));
            if (p.up) store8(static_cast<TO*>(p.up) + row * p.ld_up + at, n, narrow<TO>(v1));
        } else {
            store8(static_cast<TO*>(p.c[matrix]) + row * p.ldc[matrix] + at, n, narrow<TO>(v0));
        }
    }
}

// ------------------------------------------------------------------ few rows
// Few rows (a token of each of some sequences): bound by the weights, which are read once for
// 32 rows.  A block takes 32 (or 16) columns of gate and of up; each of its four waves takes every
// fourth 128 bytes along the sum (64 values, or 32 in float32) through LDS of its own, three
// such steps on the way, and the four join in LDS: one launch and no barrier before the end.
// (1 x 1024 x 4096 bfloat16: 4.0 to 5.5 us in the kernel, of which 3.4 are the weights' 16.8 MB at a large
// copy's rate; through k_product with the sum in parts and their join 9.  Odd sizes go through registers,
// two steps on the way: 1 x 1001 x 2731 5.3 to 7.1.)
// float32 runs on float32's own matrix instructions.
// A step's tile of one operand: 4 KB, which a wave copies.  ACROSS: its rows run along the sum.
// BOTH: half of the tile (rows; ACROSS: columns) is of a second matrix.
template <typename T, bool ACROSS, bool BOTH = false>
struct FewTile {
    static constexpr int E = 16 / (int)sizeof(T), KT = 8 * E;             // values a unit; of the sum a tile
    static constexpr int UNITS = ACROSS ? 32 / E : 8;
    using Ti = Operand<256, UNITS, ACROSS>;                                // (its order in LDS)
    // `left`: rows (ACROSS: columns) from the tile's first on; k: values of the sum, zeros past
    // the last.  Here 16 bytes a lane past the registers, rows repeated past the last ..
    static __device__ __forceinline__ bool second(int& row, int& unit) {
        int& at = ACROSS ? unit : row;
        constexpr int kHalf = ACROSS ? UNITS / 2 : 16;
        if (!BOTH || at < kHalf) return false;
        at -= kHalf;
        return true;
    }
    static __device__ __forceinline__ void copy(const T* base, int64_t stride, const T* base2, int64_t stride2, int left, int k, char* lds, int lane) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int at = i * 64 + lane;
            int row = at / UNITS, unit = (at % UNITS) ^ Ti::swz(row);
            const bool other = second(row, unit);
            const bool real = ACROSS ? row < k : unit * E < k;
            if (ACROSS) unit = min(unit, (left + E - 1) / E - 1);
            else row = min(row, left - 1);
            copy16_from(real ? reinterpret_cast<const char*>((other ? base2 + row * stride2 : base + row * stride) + unit * E) : reinterpret_cast<const char*>(kZeros),
                        __builtin_amdgcn_readfirstlane(lds_address(lds) + i * 1024));
        }
    }
    // .. and here through registers, from any alignment.  A unit past the end of a row reads the
    // row's last E values (there are as many) and moves them down: a branch for each unit waited
    // for each unit's load (8 x 2688 x 687 41 us).  put() has load()'s arguments.
    typedef uint64_t Unit __attribute__((ext_vector_type(2)));
    Unit v[4];
    static __device__ __forceinline__ int start(int unit, int left, int k) { return min(unit * E, (ACROSS ? left : k) - E); }
    __device__ __forceinline__ void load(const T* base, int64_t stride, const T* base2, int64_t stride2, int left, int k, int lane) {
        typedef uint64_t Unit_u __attribute__((ext_vector_type(2), aligned(2)));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int at = i * 64 + lane;
            int row = at / UNITS, unit = (at % UNITS) ^ Ti::swz(row);
            const bool other = second(row, unit);
            row = min(row, (ACROSS ? k : left) - 1);
            v[i] = *reinterpret_cast<const Unit_u*>((other ? base2 + row * stride2 : base + row * stride) + start(unit, left, k));
        }
    }
    __device__ __forceinline__ void put(int left, int k, char* lds, int lane) const {
        const bool whole = k >= KT && (!ACROSS || left >= (BOTH ? 16 : 32));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            Unit w = v[i];
            if (!whole) {
                const int at = i * 64 + lane;
                int row = at / UNITS, unit = (at % UNITS) ^ Ti::swz(row);
                second(row, unit);
                const int off = (unit * E - start(unit, left, k)) * (int)sizeof(T) * 8;
                const uint64_t low = off ? w[0] >> (off & 63) | (w[1] << 1) << (63 - (off & 63)) : w[0];
                w = off >= 128 ? Unit{} : off >= 64 ? Unit{w[1] >> (off & 63), 0} : Unit{low, w[1] >> (off & 63)};
                if (ACROSS && row >= k) w = Unit{};
            }
            *reinterpret_cast<Unit*>(lds + i * 1024 + lane * 16) = w;
        }
    }
    // step c of 16 as a fragment
    static __device__ __forceinline__ Frag<T> read(const char* lds, int c, int lane) {
        if constexpr (sizeof(T) == 2) {
            return Ti::read(lds, 0, c, lane);
        } else if constexpr (!ACROSS) {
            const int row = lane & 31, unit = 4 * c + 2 * (lane >> 5);
            const f32x4 a = *reinterpret_cast<const f32x4*>(lds + Ti::place(row, unit));
            const f32x4 b = *reinterpret_cast<const f32x4*>(lds + Ti::place(row, unit + 1));
            return f32x8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
        } else {
            f32x8 f;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                f[e] = *reinterpret_cast<const float*>(lds + Ti::place(16 * c + 8 * (lane >> 5) + e, (lane & 31) >> 2) + 4 * (lane & 3));
            return f;
        }
    }
};
struct FewArgs {
    const void* x;
    const void* w_gate;
    const void* w_up;
    void* h;
    void* gate;
    void* up;
    int64_t ld_x, ld_gate_w, ld_up_w, ld_h, ld_gate, ld_up;
    int rows, width, hidden, act;
};
template <typename T, bool ACROSS, bool COPY, int COLS>
__global__ __launch_bounds__(256) void k_gated_few(const FewArgs p) {
    constexpr bool BOTH = COLS == 16;
    constexpr int kW = BOTH ? 1 : 2;                                       // tiles of weights
    using X = FewTile<T, false>;
    using W = FewTile<T, ACROSS, BOTH>;
    constexpr int kSlots = COPY ? 3 : 1, kTile = 4096, kSlot = (1 + kW) * kTile, kCopies = 4 * (1 + kW), KT = X::KT;
    __shared__ __attribute__((aligned(256))) char lds[4 * kSlots * kSlot];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    char* mine = lds + wave * kSlots * kSlot;
    // neighbours on a die: the same columns of other rows
    const int high = (p.rows + 31) / 32, id = near_blocks(blockIdx.x, gridDim.x), n0 = id / high * COLS, m0 = id % high * 32;
    const int rows = min(p.rows - m0, 32);
    const int steps = (p.width + KT - 1) / KT, count = steps > wave ? (steps - wave + 3) / 4 : 0;     // this wave's
    const T* x0 = static_cast<const T*>(p.x) + m0 * p.ld_x;
    const auto of_gate = [&](int k0) { return static_cast<const T*>(p.w_gate) + (ACROSS ? k0 * p.ld_gate_w + n0 : n0 * p.ld_gate_w + k0); };
    const auto of_up = [&](int k0) { return static_cast<const T*>(p.w_up) + (ACROSS ? k0 * p.ld_up_w + n0 : n0 * p.ld_up_w + k0); };
    f32x16 g = {}, u = {};
    const auto products = [&](const char* from) {
#pragma unroll
        for (int c = 0; c < KT / 16; ++c) {
            const Frag<T> x = X::read(from, c, lane);
            g = mma(W::read(from + kTile, c, lane), x, g);
            if constexpr (!BOTH) u = mma(W::read(from + 2 * kTile, c, lane), x, u);
        }
    };
    if constexpr (COPY) {
        const auto fill = [&](int t) {
            char* to = mine + t % kSlots * kSlot;
            const int k0 = (wave + 4 * t) * KT, k = p.width - k0;
            X::copy(x0 + k0, p.ld_x, nullptr, 0, rows, k, to, lane);
            W::copy(of_gate(k0), p.ld_gate_w, of_up(k0), p.ld_up_w, p.hidden - n0, k, to + kTile, lane);
            if constexpr (!BOTH) W::copy(of_up(k0), p.ld_up_w, nullptr, 0, p.hidden - n0, k, to + 2 * kTile, lane);
        };
#pragma unroll 1
        for (int t = 0; t < kSlots && t < count; ++t) fill(t);
#pragma unroll 1
        for (int t = 0; t < count; ++t) {
            if (t + 2 < count) wait_copies_but<2 * kCopies>();
            else if (t + 1 < count) wait_copies_but<kCopies>();
            else wait_copies();
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            products(mine + t % kSlots * kSlot);
            if (t + kSlots < count) {
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the slot has been read
                fill(t + kSlots);
            }
        }
    } else {
        // two steps on the way in registers; LDS serves a wave's requests in their order
        X x[2];
        W w[2][kW];
        const auto load = [&](int t, int b) {
            const int k0 = (wave + 4 * t) * KT, k = p.width - k0;
            x[b].load(x0 + k0, p.ld_x, nullptr, 0, rows, k, lane);
            w[b][0].load(of_gate(k0), p.ld_gate_w, of_up(k0), p.ld_up_w, p.hidden - n0, k, lane);
            if constexpr (!BOTH) w[b][1].load(of_up(k0), p.ld_up_w, nullptr, 0, p.hidden - n0, k, lane);
        };
        if (count > 0) load(0, 0);
        if (count > 1) load(1, 1);
#pragma unroll 1
        for (int t0 = 0; t0 < count; t0 += 2) {
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const int t = t0 + b;
                if (t >= count) break;
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                const int k = p.width - (wave + 4 * t) * KT;
                x[b].put(rows, k, mine, lane);
                w[b][0].put(p.hidden - n0, k, mine + kTile, lane);
                if constexpr (!BOTH) w[b][1].put(p.hidden - n0, k, mine + 2 * kTile, lane);
                if (t + 2 < count) load(t + 2, b);
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                products(mine);
            }
        }
    }
    // the four sums of [row][column], gate then up (BOTH: side by side), 36 values apart
    __syncthreads();
    float* sums = reinterpret_cast<float*>(lds);
    constexpr int kPitch = 36, kMatrix = 32 * kPitch, kUp = BOTH ? 16 : kMatrix;
    static_assert(sizeof(lds) >= 4 * kW * kMatrix * 4, "the sums' place");
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        float* to = sums + wave * kW * kMatrix + (lane & 31) * kPitch + 8 * q + 4 * (lane >> 5);
        *reinterpret_cast<f32x4*>(to) = f32x4{g[4 * q], g[4 * q + 1], g[4 * q + 2], g[4 * q + 3]};
        if constexpr (!BOTH) *reinterpret_cast<f32x4*>(to + kMatrix) = f32x4{u[4 * q], u[4 * q + 1], u[4 * q + 2], u[4 * q + 3]};
    }
    __syncthreads();
    const int row = threadIdx.x / (COLS / 4), col = 4 * (threadIdx.x % (COLS / 4)), left = p.hidden - n0 - col;
    if (row >= rows || left <= 0) return;
    f32x4 vg = {}, vu = {};
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const float* from = sums + w * kW * kMatrix + row * kPitch + col;
        vg += *reinterpret_cast<const f32x4*>(from);
        vu += *reinterpret_cast<const f32x4*>(from + kUp);
    }
    const f32x4 h = activate<sizeof(T) == 4>(p.act, vg) * vu;
    store4(static_cast<T*>(p.h) + (m0 + row) * p.ld_h + n0 + col, left, h);
    if (p.gate) store4(static_cast<T*>(p.gate) + (m0 + row) * p.ld_gate + n0 + col, left, vg);
    if (p.up) store4(static_cast<T*>(p.up) + (m0 + row) * p.ld_up + n0 + col, left, vu);
}

// ------------------------------------------------------------------ layouts
// A float32 in three parts, as split() makes them, but that values past the largest bfloat16
// (3.39e38) keep a finite first part, and an infinity is (1, 0, infinity) with its sign: its last part
// meets the other operand's first alone, which is 0 or has the other sign only where that operand does.
constexpr float kMostBf16 = 3.38953139e38f;
__device__ inline Split split_any(f32x8 x) {
    f32x8 y, r;
    bool infinite[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        infinite[e] = fabsf(x[e]) == INFINITY;
        y[e] = infinite[e] ? copysignf(1.f, x[e]) : fminf(fmaxf(x[e], -kMostBf16), kMostBf16);
    }
    Split s;
    s.h = narrow<bf16>(y);
    const f32x8 h = widen(s.h);
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = infinite[e] ? 0.f : x[e] - h[e];      // (NaN stays in it)
    s.m = narrow<bf16>(r);
    const f32x8 m = widen(s.m);
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = infinite[e] ? x[e] : r[e] - m[e];
    s.l = narrow<bf16>(r);
    return s;
}
// A float32 in two bfloat16 parts, to 2^-16 of it, for products with operands of one part.  The first
// is rounded towards 0 and the second is never 0 (but for 0, and values under 2^-96): where the other
// operand is infinite, both parts give infinities of one sign.
struct Halves {
    bf16x8 h, m;
};
__device__ inline Halves split_in_two(f32x8 x) {
    f32x8 h, m;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float v = x[e];
        h[e] = fabsf(v) < INFINITY ? __uint_as_float(__float_as_uint(v) & 0xffff0000u) : copysignf(1.f, v);
        const float rest = v - h[e];         // (exact; infinity and NaN stay in it)
        m[e] = rest != 0.f ? rest : v * 0x1p-30f;
    }
    return Halves{narrow<bf16>(h), narrow<bf16>(m)};
}
// [rows][cols] as bfloat16 [rows][pitch], zeros past cols; float32: three parts, each a
// matrix.
template <int PARTS>
__device__ inline void store_parts(bf16* to, int64_t plane, f32x8 v) {
    if constexpr (PARTS == 1) {
        *reinterpret_cast<bf16x8*>(to) = narrow<bf16>(v);
    } else if constexpr (PARTS == 2) {
        const Halves s = split_in_two(v);
        *reinterpret_cast<bf16x8*>(to) = s.h;
        *reinterpret_cast<bf16x8*>(to + plane) = s.m;
    } else {
        const Split s = split_any(v);
        *reinterpret_cast<bf16x8*>(to) = s.h;
        *reinterpret_cast<bf16x8*>(to + plane) = s.m;
        *reinterpret_cast<bf16x8*>(to + 2 * plane) = s.l;
    }
}
struct LayOut {
    const void* from;
    int64_t stride, rows;
    int cols, pitch;
    bf16* to;
};
struct LayOuts {
    LayOut m[3];
    int64_t end[3];          // units of the matrices up to and with each
};
template <typename T>
__global__ __launch_bounds__(256) void k_lay_out(const LayOuts a) {
    for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < a.end[2]; u += (int64_t)gridDim.x * 256) {
        const int which = u < a.end[0] ? 0 : u < a.end[1] ? 1 : 2;
        const LayOut& m = a.m[which];
        const int64_t in = u - (which ? a.end[which - 1] : 0), row = in / (m.pitch / 8);
        const int c = (int)(in - row * (m.pitch / 8)) * 8;
        f32x8 v = {};
        if (c < m.cols) v = widen(load8(static_cast<const T*>(m.from) + row * m.stride + c, m.cols - c));
        store_parts<sizeof(T) == 4 ? 3 : 1>(m.to + row * m.pitch + c, m.rows * m.pitch, v);
    }
}

// dg and du as operands, and h.
struct SlopeArgs {
    const void* gate;
    const void* up;
    const void* dh;
    void* h;
    int64_t ld_gate, ld_up, ld_dh, ld_h, rows;
    int cols, pitch, act;
    bf16* dg;                // then du, after all parts of dg
    int64_t du;              // elements from dg to du
};
template <typename T, int PARTS>
__global__ __launch_bounds__(256) void k_gated_slopes(const SlopeArgs a) {
    const int64_t units = a.rows * (a.pitch / 8);
    for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < units; u += (int64_t)gridDim.x * 256) {
        const int64_t row = u / (a.pitch / 8);
        const int c = (int)(u - row * (a.pitch / 8)) * 8, n = a.cols - c;
        f32x8 dg = {}, du = {};
        if (n > 0) {
            const f32x8 g = widen(load8(static_cast<const T*>(a.gate) + row * a.ld_gate + c, n));
            const f32x8 up = widen(load8(static_cast<const T*>(a.up) + row * a.ld_up + c, n));
            const f32x8 dh = widen(load8(static_cast<const T*>(a.dh) + row * a.ld_dh + c, n));
            f32x8 act, slope;
            activate_grad<sizeof(T) == 4>(a.act, g, act, slope);
            dg = dh * up * slope;            // (past the row's end dh and up are 0, slope is finite)
            du = dh * act;
            if (a.h) store8(static_cast<T*>(a.h) + row * a.ld_h + c, n, narrow<T>(act * up));
        }
        if (!a.dg) continue;
        bf16* to = a.dg + row * a.pitch + c;
        store_parts<PARTS>(to, a.rows * a.pitch, dg);
        store_parts<PARTS>(to + a.du, a.rows * a.pitch, du);
    }
}

template <typename T>
__global__ __launch_bounds__(256) void k_zero_rows(T* to, int64_t stride, int64_t rows, int cols) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * cols; i += (int64_t)gridDim.x * 256)
        to[i / cols * stride + i % cols] = (T)0.f;
}

// ------------------------------------------------------------------ launches
unsigned blocks_for(int64_t lanes) {
    const int64_t b = (lanes + 255) / 256;
    return (unsigned)(b < 1 ? 1 : b < 65536 ? b : 65536);
}
int64_t up_to(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

// A matrix as the products read it: where its parts begin, and its rows' distance.
struct Matrix {
    const bf16* part[3];
    int64_t ld;
};
constexpr int parts_of(int dtype) { return dtype == PD_F32 ? 3 : 1; }
// Parts of dg and du.  In bfloat16 two: one would add as much to a gradient's error as the
// rounding of the result does (1.41 times it together, with few rows up to 1.8 times), for half
// of the products (9216 x 1024 x 2736: 282 and 534 us).
constexpr int slope_parts(int dtype) { return dtype == PD_F32 ? 3 : 2; }
int64_t layout_bytes(int parts, int64_t rows, int64_t cols) { return rows * up_to(cols, 64) * 2 * parts; }
// Copies of 16 bytes read the matrix as it lies, if it begins at a multiple of them.
bool as_it_lies(int dtype, int64_t stride, int64_t rows, int64_t cols) {
    return dtype == PD_BF16 && cols % 8 == 0 && (rows == 1 || (stride % 8 == 0 && stride < (1 << 22)));
}
bool whole_units(const void* p) { return (uintptr_t)p % 16 == 0; }
bool inputs_lie(const pd_gated_desc& d) { return as_it_lies(d.dtype, d.x_stride, d.rows, d.width); }
// Both weights lie alike, as the kernel has one distance of rows for them.  `along`: the
// product reads them along the sum, 128 bytes of a row at a time; where these straddle the
// memory's lines and there are many rows, laying them out pays (20000 x 1000 x 2664: 298 and
// 266 us; 4608 rows 77 and 70; read across the sum 236 and 232).
bool weights_lie(const pd_gated_desc& d, bool along) {
    const bool in_out = d.weight_layout == PD_WEIGHTS_IN_OUT;
    const int64_t rows = in_out ? d.width : d.hidden, cols = in_out ? d.hidden : d.width;
    return as_it_lies(d.dtype, d.w_gate_stride, rows, cols) && as_it_lies(d.dtype, d.w_up_stride, rows, cols) &&
           (rows == 1 || d.w_gate_stride == d.w_up_stride) && !(along && d.rows >= 8192 && rows > 1 && d.w_gate_stride % 64);
}
// Operands as products read them; those that do not lie so are laid out by one launch.
struct Operands {
    LayOuts todo{};
    int count = 0;
    Matrix add(int dtype, const void* p, int64_t stride, int64_t rows, int64_t cols, char* to, bool lies) {
        if (lies) return Matrix{{static_cast<const bf16*>(p)}, rows == 1 ? cols : stride};
        const int64_t pitch = up_to(cols, 64), units = rows * (pitch / 8);
        bf16* q = reinterpret_cast<bf16*>(to);
        todo.m[count] = LayOut{p, stride, rows, (int)cols, (int)pitch, q};
        todo.end[count] = (count ? todo.end[count - 1] : 0) + units;
        for (int i = ++count; i < 3; ++i) todo.end[i] = todo.end[count - 1];
        return Matrix{{q, q + rows * pitch, q + 2 * rows * pitch}, pitch};
    }
    void run(int dtype, hipStream_t s) const {
        if (!count) return;
        const dim3 grid(blocks_for(todo.end[2])), block(256);
        if (dtype == PD_F32) hipLaunchKernelGGL(k_lay_out<float>, grid, block, 0, s, todo);
        else hipLaunchKernelGGL(k_lay_out<bf16>, grid, block, 0, s, todo);
        PD_HIP(hipGetLastError());
    }
};
// Appends the segments of a times (b0, b1) to p, small ones first: of the parts 0, 1, 2 of
// each the pairs whose numbers add up to 2 at most.
int segments(int parts_a, int parts_b) { return parts_a == 3 && parts_b == 3 ? 6 : parts_a * parts_b; }
void add_segments(Product& p, const Matrix& a, int parts_a, const Matrix& b0, const Matrix& b1, int parts_b) {
    static const int pa[6] = {2, 0, 1, 1, 0, 0}, pb[6] = {0, 2, 1, 0, 1, 0};
    for (int i = 0; i < 6; ++i) {
        if (pa[i] >= parts_a || pb[i] >= parts_b) continue;
        p.a[p.segs] = a.part[pa[i]];
        p.b0[p.segs] = b0.part[pb[i]];
        p.b1[p.segs] = b1.part[pb[i]];
        ++p.segs;
    }
    p.lda = a.ld;
    p.ldb = b0.ld;
}

// How a product is cut: the block's form, and into how many sums.
using Large = Form<4, 4, 2, 64, 2>;       // 256 x 256, one block a compute unit
using Wide = Form<3, 4, 2, 64, 2>;        // 192 x 256, one
using Medium = Form<2, 4, 2, 32, 3>;      // 128 x 256, two blocks
using Small = Form<2, 2, 2, 64, 2>;       // 128 x 128, two blocks
using Few = Form<1, 2, 1, 64, 2>;         // 32 x 256, two blocks
enum Shape { kLarge, kWide, kMedium, kSmall, kFew, kShapes };
// What a round of blocks takes, in us: of a step of 64 and beside its steps; measured on
// 36864 x 1024 x 4096 and 8192 x 4096 x 4096 (`alone`: of a step where a unit has one block).
struct Cost {
    int bm, hn, bk, slots;
    double step, alone, fixed;
};
constexpr Cost kCost[kShapes] = {
    {Large::BM, Large::HN, Large::kBK, kCus, 1.64, 1.64, 6.8},
    {Wide::BM, Wide::HN, Wide::kBK, kCus, 1.35, 1.35, 6.3},
    {Medium::BM, Medium::HN, Medium::kBK, 2 * kCus, 1.75, 1.0, 5.5},
    {Small::BM, Small::HN, Small::kBK, 2 * kCus, 0.95, 0.65, 3.4},
    {Few::BM, Few::HN, Few::kBK, 2 * kCus, 0.6, 0.4, 3.0},
};
struct Cut {
    Shape shape;
    int tiles_m, tiles_n, splits, steps;
};
Cut cut(int64_t m, int64_t n, bool apart, int groups, int64_t k, int segs, bool across) {
    Cut best{};
    double least = 1e30;
    for (int shape = 0; shape < kShapes; ++shape) {
        if (shape == kFew ? across || m > 64 : m <= 32 && !across) continue;      // (`across`: a runs across the sum)
        const Cost& f = kCost[shape];
        Cut c{};
        c.shape = (Shape)shape;
        c.tiles_m = (int)((m + f.bm - 1) / f.bm);
        const int wide = apart ? f.hn : 2 * f.hn;
        c.tiles_n = (int)((n + wide - 1) / wide);
        c.steps = (int)((k + f.bk - 1) / f.bk);
        const int64_t tiles = (int64_t)c.tiles_m * c.tiles_n * groups;
        const double steps = (double)c.steps * segs * f.bk / 64;
        static const int kSplits[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32};
        for (int s : kSplits) {
            if (s > 1 && (steps / s < 4 || tiles * (s - 1) >= 4 * kCus)) break;
            const int64_t blocks = tiles * s, rounds = blocks / f.slots, rest = blocks % f.slots;
            double t = (double)rounds * (steps / s * f.step + f.fixed);
            if (rest) t += steps / s * (rest <= kCus ? f.alone : f.step) + f.fixed;
            // the sums go to memory and are read again
            if (s > 1) t += 4 + 8e-6 * s * (double)m * (double)n * (apart ? 2 : groups) / 4;
            if (t < least) {
                least = t;
                best = c;
                best.splits = s;
            }
        }
    }
    return best;
}
int64_t partial_bytes(const Cut& c, int64_t m, int64_t n, bool apart, int groups) {
    return c.splits == 1 ? 0 : (int64_t)c.splits * groups * (apart ? 2 : 1) * m * n * 4;
}

template <bool AC, bool BC, Out OUT, typename TO>
void launch_shape(const Product& p, Shape shape, hipStream_t s) {
    // blocks that are on the chip together take tile after tile
    const int tiles = p.tiles_m * p.tiles_n * p.groups * p.splits, most = kCost[shape].slots;
    const dim3 grid((unsigned)(tiles < most ? tiles : most)), block(256);
    if (shape == kLarge)
        hipLaunchKernelGGL((k_product<Large, AC, BC, OUT, TO>), grid, block, 0, s, p);
    else if (shape == kWide)
        hipLaunchKernelGGL((k_product<Wide, AC, BC, OUT, TO>), grid, block, 0, s, p);
    else if (shape == kMedium)
        hipLaunchKernelGGL((k_product<Medium, AC, BC, OUT, TO>), grid, block, 0, s, p);
    else if (shape == kSmall)
        hipLaunchKernelGGL((k_product<Small, AC, BC, OUT, TO>), grid, block, 0, s, p);
    else if constexpr (!AC)
        hipLaunchKernelGGL((k_product<Few, AC, BC, OUT, TO>), grid, block, 0, s, p);
    PD_HIP(hipGetLastError());
}
template <bool AC, bool BC, bool GATED, typename TO>
void launch_product(Product& p, float* partial, hipStream_t s) {
    const Cut c = cut(p.m, p.n, p.apart, p.groups, p.k, p.segs, AC);
    p.steps = c.steps;
    p.tiles_m = c.tiles_m, p.tiles_n = c.tiles_n, p.splits = c.splits;
    p.partial = partial;
    if (c.splits == 1) return launch_shape<AC, BC, GATED ? kGated : kStore, TO>(p, c.shape, s);
    launch_shape<AC, BC, kPartial, float>(p, c.shape, s);
    hipLaunchKernelGGL((k_product_join<GATED, TO>), dim3(blocks_for((int64_t)p.m * ((p.n + 7) / 8) * (GATED || !p.apart ? 1 : 2) * p.groups)),
                       dim3(256), 0, s, p);
    PD_HIP(hipGetLastError());
}

// A call's products: f(rows, columns, apart, groups, sum, segments, across) of each.
template <class F>
void each_product(const pd_gated_desc& d, bool backward, F f) {
    const int parts = parts_of(d.dtype), segs = segments(backward ? slope_parts(d.dtype) : parts, parts);
    if (!backward) return f(d.rows, d.hidden, true, 1, d.width, segs, false);
    f(d.rows, d.width, false, 1, d.hidden, 2 * segs, false);
    if (d.weight_layout == PD_WEIGHTS_IN_OUT) f(d.width, d.hidden, true, 1, d.rows, segs, true);
    else f(d.hidden, d.width, false, 2, d.rows, segs, true);
}
// Scratch of a call: operands laid out, then the products' partial sums.
struct Layout {
    int64_t x, w, slopes, partial, total;    // bytes, each at a multiple of 256
};
Layout layout(const pd_gated_desc& d, bool backward) {
    const bool in_out = d.weight_layout == PD_WEIGHTS_IN_OUT;
    Layout l{};
    int64_t at = 0;
    const auto take = [&](int64_t bytes) {
        const int64_t here = at;
        at += up_to(bytes, 256);
        return here;
    };
    const int parts = parts_of(d.dtype);
    // (no room for operands that are read where they are)
    if (!(d.aligned && inputs_lie(d))) l.x = take(layout_bytes(parts, d.rows, d.width));
    if (!(d.aligned && weights_lie(d, backward == in_out)))
        l.w = take(2 * (in_out ? layout_bytes(parts, d.width, d.hidden) : layout_bytes(parts, d.hidden, d.width)));
    if (backward) l.slopes = take(2 * layout_bytes(slope_parts(d.dtype), d.rows, d.hidden));
    int64_t partial = 0;
    each_product(d, backward, [&](int64_t m, int64_t n, bool apart, int groups, int64_t k, int segs, bool across) {
        const int64_t b = partial_bytes(cut(m, n, apart, groups, k, segs, across), m, n, apart, groups);
        partial = b > partial ? b : partial;
    });
    l.partial = take(partial);
    l.total = at;
    return l;
}

Matrix inputs(const GatedArgs& a, const Layout& l, Operands& o) {
    const pd_gated_desc& d = a.d;
    return o.add(d.dtype, a.x, d.x_stride, d.rows, d.width, a.scratch + l.x, inputs_lie(d) && whole_units(a.x));
}
void weights(const GatedArgs& a, const Layout& l, bool along, Matrix& gate, Matrix& up, Operands& o) {
    const pd_gated_desc& d = a.d;
    const bool in_out = d.weight_layout == PD_WEIGHTS_IN_OUT;
    const int64_t rows = in_out ? d.width : d.hidden, cols = in_out ? d.hidden : d.width;
    const bool lie = weights_lie(d, along) && whole_units(a.w_gate) && whole_units(a.w_up);
    gate = o.add(d.dtype, a.w_gate, d.w_gate_stride, rows, cols, a.scratch + l.w, lie);
    up = o.add(d.dtype, a.w_up, d.w_up_stride, rows, cols, a.scratch + l.w + layout_bytes(parts_of(d.dtype), rows, cols), lie);
}

// Whether a forward pass is one of few rows.  us there and through the tiles, in bfloat16 and float32 (137 x 3200 x 6400 155 and 196):
// 64 x 1024 x 4096 6 and 12, 16 and 46; 128 rows 11 and 13, 28 and 47; 256 rows 20 and 14, 57 and 59;
// 64 x 4096 x 16384 51 to 68 and 59 to 65, 190 and 575; 128 rows 97 to 135 and 58 to 66, 400 and 573.
// 128 x 448 x 1792 4 and 9, 9 and 28.
bool few(const pd_gated_desc& d) {
    const bool small = (int64_t)d.width * d.hidden <= 1 << 22;
    return d.rows <= (d.dtype == PD_F32 ? 160 : small ? 128 : 64) && d.width >= 8 && d.hidden >= 8;
}
template <typename T, bool ACROSS, bool COPY>
void launch_few(const FewArgs& p, bool half, int64_t high, hipStream_t s) {
    const dim3 grid((unsigned)((half ? (p.hidden + 15) / 16 : (p.hidden + 31) / 32) * high)), block(256);
    if (half) hipLaunchKernelGGL((k_gated_few<T, ACROSS, COPY, 16>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((k_gated_few<T, ACROSS, COPY, 32>), grid, block, 0, s, p);
    PD_HIP(hipGetLastError());
}
template <typename T>
void gated_few(const GatedArgs& a, hipStream_t s) {
    const pd_gated_desc& d = a.d;
    const bool in_out = d.weight_layout == PD_WEIGHTS_IN_OUT;
    const int64_t wr = in_out ? d.width : d.hidden, wc = in_out ? d.hidden : d.width;
    const auto whole = [](const void* p, int64_t stride, int64_t rows, int64_t cols) {
        return (uintptr_t)p % 16 == 0 && cols * sizeof(T) % 16 == 0 && (rows == 1 || stride * sizeof(T) % 16 == 0);
    };
    const bool copy = whole(a.x, d.x_stride, d.rows, d.width) && whole(a.w_gate, d.w_gate_stride, wr, wc) &&
                      whole(a.w_up, d.w_up_stride, wr, wc);
    const FewArgs p{a.x, a.w_gate, a.w_up, a.h, a.gate, a.up, d.x_stride, d.w_gate_stride, d.w_up_stride, d.h_stride, d.gate_stride,
                    d.up_stride, (int)d.rows, d.width, d.hidden, d.activation};
    const int64_t high = (d.rows + 31) / 32;
    // 16 columns a block while these are no more than compute units (us, 32 and 16 columns: 1 x 1024 x 4096
    // bfloat16 4.8 to 5.4 and 4.0 to 5.2, with weights from memory 7.2 to 9.5 and 6.0 to 8.1, float32 12.6 to 14.5
    // and 8.3 to 10.4; 1 x 1024 x 8192 5.0 and 6.9, 15 and 17)
    const bool half = ((int64_t)d.hidden + 15) / 16 * high <= kCus;
    if (in_out && copy) launch_few<T, true, true>(p, half, high, s);
    else if (in_out) launch_few<T, true, false>(p, half, high, s);
    else if (copy) launch_few<T, false, true>(p, half, high, s);
    else launch_few<T, false, false>(p, half, high, s);
}

template <typename T>
void gated_t(const GatedArgs& a, hipStream_t s) {
    const pd_gated_desc& d = a.d;
    if (few(d)) return gated_few<T>(a, s);
    const Layout l = layout(d, false);
    Operands o;
    Matrix wg, wu;
    const Matrix x = inputs(a, l, o);
    weights(a, l, d.weight_layout == PD_WEIGHTS_OUT_IN, wg, wu, o);
    o.run(d.dtype, s);
    Product p{};
    add_segments(p, x, parts_of(d.dtype), wg, wu, parts_of(d.dtype));
    p.k = d.width, p.m = (int)d.rows, p.n = d.hidden;
    p.apart = 1, p.groups = 1;
    p.act = d.activation;
    p.c[0] = a.h, p.ldc[0] = d.h_stride;
    p.gate = a.gate, p.up = a.up, p.ld_gate = d.gate_stride, p.ld_up = d.up_stride;
    float* partial = reinterpret_cast<float*>(a.scratch + l.partial);
    if (d.weight_layout == PD_WEIGHTS_IN_OUT) launch_product<false, true, true, T>(p, partial, s);
    else launch_product<false, false, true, T>(p, partial, s);
}

template <typename T>
void gated_grad_t(const GatedArgs& a, hipStream_t s) {
    const pd_gated_desc& d = a.d;
    const bool in_out = d.weight_layout == PD_WEIGHTS_IN_OUT;
    if (d.rows == 0) {
        if (!a.dw_gate) return;
        const int64_t rows = in_out ? d.width : d.hidden;
        const int cols = in_out ? d.hidden : d.width;
        for (int i = 0; i < 2; ++i) {
            hipLaunchKernelGGL(k_zero_rows<T>, dim3(blocks_for(rows * cols)), dim3(256), 0, s,
                               static_cast<T*>(i ? a.dw_up : a.dw_gate), i ? d.dw_up_stride : d.dw_gate_stride, rows, cols);
            PD_HIP(hipGetLastError());
        }
        return;
    }
    const Layout l = layout(d, true);
    const bool products = a.dx || a.dw_gate;
    const int64_t pitch = up_to(d.hidden, 64), plane = d.rows * pitch;
    SlopeArgs g{};
    g.gate = a.gate, g.up = a.up, g.dh = a.dh, g.h = a.h;
    g.ld_gate = d.gate_stride, g.ld_up = d.up_stride, g.ld_dh = d.dh_stride, g.ld_h = d.h_stride;
    g.rows = d.rows, g.cols = d.hidden, g.pitch = (int)pitch, g.act = d.activation;
    g.dg = products ? reinterpret_cast<bf16*>(a.scratch + l.slopes) : nullptr;
    constexpr int kType = sizeof(T) == 4 ? PD_F32 : PD_BF16, parts = parts_of(kType), slopes = slope_parts(kType);
    g.du = slopes * plane;
    const dim3 grid(blocks_for(d.rows * pitch / 8)), block(256);
    hipLaunchKernelGGL((k_gated_slopes<T, slopes>), grid, block, 0, s, g);
    PD_HIP(hipGetLastError());
    const Matrix dg{{g.dg, g.dg + plane, g.dg + 2 * plane}, pitch}, du{{g.dg + g.du, g.dg + g.du + plane, g.dg + g.du + 2 * plane}, pitch};
    float* partial = reinterpret_cast<float*>(a.scratch + l.partial);
    Operands o;
    Matrix x, wg, wu;
    if (a.dx) weights(a, l, in_out, wg, wu, o);
    if (a.dw_gate) x = inputs(a, l, o);
    o.run(d.dtype, s);
    if (a.dx) {
        Product p{};
        add_segments(p, dg, slopes, wg, wg, parts);
        add_segments(p, du, slopes, wu, wu, parts);
        p.k = d.hidden, p.m = (int)d.rows, p.n = d.width;
        p.apart = 0, p.groups = 1;
        p.c[0] = a.dx, p.ldc[0] = d.dx_stride;
        if (in_out) launch_product<false, false, false, T>(p, partial, s);
        else launch_product<false, true, false, T>(p, partial, s);
    }
    if (a.dw_gate) {
        Product p{};
        if (in_out) {
            add_segments(p, x, parts, dg, du, slopes);
            p.m = d.width, p.n = d.hidden;
            p.apart = 1, p.groups = 1;
        } else {
            add_segments(p, dg, slopes, x, x, parts);
            p.m = d.hidden, p.n = d.width;
            p.apart = 0, p.groups = 2, p.a_group = g.du;
        }
        p.k = (int)d.rows;
        p.c[0] = a.dw_gate, p.c[1] = a.dw_up;
        p.ldc[0] = d.dw_gate_stride, p.ldc[1] = d.dw_up_stride;
        launch_product<true, true, false, T>(p, partial, s);
    }
}

}  // namespace

int64_t gated_scratch_bytes(const pd_gated_desc& d) { return few(d) ? 0 : layout(d, false).total; }
void launch_gated(const GatedArgs& a, hipStream_t s) { a.d.dtype == PD_F32 ? gated_t<float>(a, s) : gated_t<bf16>(a, s); }
int gated_forms(const pd_gated_desc& d, bool backward, int* out) {
    if (d.rows == 0 || (!backward && few(d))) return 0;
    int count = 0;
    each_product(d, backward, [&](int64_t m, int64_t n, bool apart, int groups, int64_t k, int segs, bool across) {
        const Cut c = cut(m, n, apart, groups, k, segs, across);
        const int values[4] = {c.shape, c.splits, c.tiles_m * c.tiles_n * groups * c.splits, kCost[c.shape].slots};
        for (int v : values) *out++ = v;
        ++count;
    });
    return count;
}
int64_t gated_grad_scratch_bytes(const pd_gated_desc& d) { return d.rows ? layout(d, true).total : 0; }
void launch_gated_grad(const GatedArgs& a, hipStream_t s) { a.d.dtype == PD_F32 ? gated_grad_t<float>(a, s) : gated_grad_t<bf16>(a, s); }

}  // namespace pd
