// Attention with a sliding window and sinks, backward.
//
//   p_ij = e^(scale q_i k_j - lse_i),  dp_ij = do_i v_j,  delta_i = do_i o_i,
//   ds_ij = p_ij (dp_ij - delta_i):
//   dq_i = scale sum_j ds_ij k_j,  dk_j = scale sum_i ds_ij q_i,  dv_j = sum_i p_ij do_i
//
// Two kernels, each summing into its own registers: dq over a block of queries
// (which also leaves delta, and what rows with large scores take them from, for the
// other), dk and dv over a block of keys and the query heads that read them.  The scores
// are formed twice (14 D operations a pair and head in place of 10), and in exchange there
// is no atomic and no order that varies from run to run.  Where there are few blocks of
// keys, their queries are split among several blocks, whose sums k_attention_dkv_join adds.
//
// Bound by the chain of LDS reads, products and vector work of a wave (two waves a SIMD):
// hence reads a group ahead (Stream) and sums that start from -lse / scale and -delta.
// Measured: 4 x 2304 tokens two-sided, 16 heads on 4 of 64 bfloat16 values 373 us (583
// TFLOP/s of the 10 D operations, 816 of the 14 D it does; profiled, at lower clocks: dq
// 158, dk and dv 217, join 21); float32, 2 x 2048 tokens causal: 64 values 407 us, 128
// values 970 to 1030.
//
// bfloat16 rounds p and ds once more, as operands: errors of 2.4e-3 where the results'
// own rounding alone makes 1.7e-3.
#include "attention_tile.h"

namespace pd {
namespace {

using namespace attn;

// p = e^(scale s - lse): one fused multiply-add in base 2 while |lse| is under 1024;
// beyond, lse log2 e and lse itself are rounded too coarsely (at 2^21 a float32 has steps
// of 1/4).  There the largest score and the sum over it are formed again, from this
// pass's own scores, and p = e^(scale s - largest) / sum, both terms rounded alike: a
// row's probabilities sum to 1 at any size, and equal scores have equal ones.
constexpr float kLarge = 1024.f;
__device__ inline bool is_large(float lse) { return !(fabsf(lse) < kLarge); }
// (float32 takes the difference first, so that neither c2's nor lse log2 e's rounding is
// multiplied by the score.)
template <typename T>
__device__ inline float probability(float s, float c2, float lse2, float scale, float lse) {
    return sizeof(T) == 2 ? exp2_fast(fmaf(s, c2, -lse2)) : exp2_fast(fmaf(s, scale, -lse) * kLog2e);
}
// What a row's scores are taken from, and what their exponentials are multiplied by:
// (lse, 1), or the largest score and 1 / sum.
struct Base {
    float from, times;
};
__device__ inline float probability(float s, float scale, const Base& b) {
    const float x = s * scale - b.from;
    return exp2_fast((x > 0.f ? 0.f : x) * kLog2e) * b.times;     // (rounding aside x <= 0)
}
__device__ inline Base base_of(float top, float total) {          // no score above -inf: p = 0
    return Base{top == -INFINITY ? 0.f : top, total == 0.f ? 0.f : 1.f / total};
}

// Scratch: delta of every row, the Base of those with a large lse, then the parts of dk
// and dv, [split][sequence, key head, key][dk, dv].
__host__ __device__ inline int64_t all_rows(const pd_attention_desc& d) { return (int64_t)d.batch * d.heads_q * d.q_len; }
__host__ __device__ inline int64_t row_floats(const pd_attention_desc& d) { return (3 * all_rows(d) + 3) & ~(int64_t)3; }
__device__ inline float* dkv_parts(const AttentionArgs& a) { return a.scratch + row_floats(a.d); }

// What the backward kernels read of one (sequence, key head).
template <typename T>
struct Views {
    const T *k, *v;              // of the key head
    const T *q, *out, *dout;     // of the group's first query head
    const float *lse, *delta;    // [group][q_len]
    const float* bases;          // [group][q_len][2]
    int group;
};
template <typename T>
__device__ inline Views<T> views(const AttentionArgs& a, int b, int hk) {
    const pd_attention_desc& d = a.d;
    const int group = d.heads_q / d.heads_kv, hq = hk * group;
    const int64_t at = ((int64_t)b * d.heads_q + hq) * d.q_len;
    return Views<T>{static_cast<const T*>(a.k) + b * d.k_stride[0] + hk * d.k_stride[2],
                    static_cast<const T*>(a.v) + b * d.v_stride[0] + hk * d.v_stride[2],
                    static_cast<const T*>(a.q) + b * d.q_stride[0] + hq * d.q_stride[2],
                    static_cast<const T*>(a.out) + b * d.out_stride[0] + hq * d.out_stride[2],
                    static_cast<const T*>(a.dout) + b * d.dout_stride[0] + hq * d.dout_stride[2],
                    a.lse + at, a.scratch + at, a.scratch + all_rows(d) + 2 * at, group};
}

// the base of a row from memory
template <typename T>
__device__ inline Base row_base(const Views<T>& w, int64_t at) {
    const float lse = w.lse[at];
    return is_large(lse) ? Base{w.bases[2 * at], w.bases[2 * at + 1]} : Base{lse, 1.f};
}

// float32 operands are held in three parts
template <typename T, int DP, int ROWS>
using Held = std::conditional_t<sizeof(T) == 2, AsIs<T, DP>, InParts<DP, ROWS>>;

// The score of each lane's own row `mine` with the wave's `one`, as the matrix cores form it for
// the kernels (TURNED: the rows are queries), so that it fits a row's base to the bit; where
// that is not finite (a value in parts: infinity less infinity), the plain sum.
template <typename T, bool TURNED>
__device__ float wave_score(const T* mine, const T* one, int D) {
    using As = Held<T, 32, 32>;
    const int lane = threadIdx.x & 63, h = lane >> 5;
    const uint64_t address = (uint64_t)(uintptr_t)mine;
    float got = 0.f;
    for (int tile = 0; tile < 2; ++tile) {
        const int from = 32 * tile + (lane & 31);
        const uint32_t lo = (uint32_t)__shfl((int)(uint32_t)address, from), hi = (uint32_t)__shfl((int)(uint32_t)(address >> 32), from);
        const T* row = reinterpret_cast<const T*>((uintptr_t)(((uint64_t)hi << 32) | lo));
        f32x16 s = {};
        for (int c = 0; 16 * c < D; ++c) {
            const int e = 16 * c + 8 * h;
            f32x8 x = {}, y = {};
            if (e < D) {
                x = widen(load8(row + e, D - e));
                y = widen(load8(one + e, D - e));
            }
            if constexpr (TURNED)
                s = mma_turned(As::make(x), As::make(y), s);
            else
                s = mma(As::make(x), As::make(y), s);
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const float a = __shfl(s[r], 0), b = __shfl(s[r], 32);
            if (lane == 32 * tile + tile_row(0, r)) got = a;
            if (lane == 32 * tile + tile_row(32, r)) got = b;
        }
    }
    if (!(fabsf(got) < INFINITY)) {
        got = 0.f;
        for (int e = 0; e < D; ++e) got = fmaf((float)mine[e], (float)one[e], got);
    }
    return got;
}

// p and ds of one pair, its score s given, from memory
template <typename T>
__device__ inline void pair_grad(const AttentionArgs& a, const Views<T>& w, int i, int g, int j, float s, float* p, float* ds) {
    const pd_attention_desc& d = a.d;
    const T* go = w.dout + i * d.dout_stride[1] + g * d.dout_stride[2];
    const T* v = w.v + j * d.v_stride[1];
    float dp = 0.f;
    for (int e = 0; e < d.head_dim; ++e) dp = fmaf((float)go[e], (float)v[e], dp);
    const int64_t at = (int64_t)g * d.q_len + i;
    *p = probability(s, d.scale, row_base(w, at));
    *ds = *p * (dp - w.delta[at]);
}

// The base of a row with a large lse from its visible keys alone, for rows whose fast sums are
// not finite; the whole wave works on the row.
template <typename T>
__device__ void base_row(const AttentionArgs& a, const Views<T>& w, int i, int g, const See see) {
    const int lane = threadIdx.x & 63;
    const T* q = w.q + i * a.d.q_stride[1] + g * a.d.q_stride[2];
    float top = -INFINITY, total = 0.f;
    for (int part = 0; part < 2; ++part) {
        const int j0 = part == 0 ? 0 : max(see.lo, see.sk), j1 = part == 0 ? see.sk : see.hi;
        for (int jb = j0; jb < j1; jb += 64) {
            const float s = wave_score<T, false>(w.k + min(jb + lane, j1 - 1) * a.d.k_stride[1], q, a.d.head_dim);
            const float x = jb + lane < j1 ? s * a.d.scale : -INFINITY;
            const float m = fmaxf(top, x), from = m == -INFINITY ? 0.f : m;
            total = total * exp2_fast((top - from) * kLog2e) + exp2_fast((x - from) * kLog2e);
            top = m;
        }
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        const float t = __shfl_xor(top, o), u = __shfl_xor(total, o), m = fmaxf(top, t), from = m == -INFINITY ? 0.f : m;
        total = total * exp2_fast((top - from) * kLog2e) + u * exp2_fast((t - from) * kLog2e);
        top = m;
    }
    const Base b = base_of(top, total);
    if (lane == 0) {
        float* to = const_cast<float*>(w.bases) + 2 * ((int64_t)g * a.d.q_len + i);
        to[0] = b.from;
        to[1] = b.times;
    }
    __threadfence();
}

// A row of dq from its visible keys alone (see attend_row in attention.hip).
template <typename T>
__device__ void dq_row(const AttentionArgs& a, const Views<T>& w, int i, int g, const See see, T* dq) {
    const int lane = threadIdx.x & 63, D = a.d.head_dim;
    const T* q = w.q + i * a.d.q_stride[1] + g * a.d.q_stride[2];
    if (is_large(w.lse[(int64_t)g * a.d.q_len + i])) base_row(a, w, i, g, see);
    float acc[2] = {0.f, 0.f};
    for (int part = 0; part < 2; ++part) {
        const int j0 = part == 0 ? 0 : max(see.lo, see.sk), j1 = part == 0 ? see.sk : see.hi;
        for (int jb = j0; jb < j1; jb += 64) {
            const int count = min(64, j1 - jb);
            float p = 0.f, ds = 0.f;
            const float s = wave_score<T, false>(w.k + (jb + min(lane, count - 1)) * a.d.k_stride[1], q, D);
            if (lane < count) pair_grad(a, w, i, g, jb + lane, s, &p, &ds);
            for (int jj = 0; jj < count; ++jj) {
                const float x = __shfl(ds, jj);
                const T* k = w.k + (int64_t)(jb + jj) * a.d.k_stride[1];
                if (lane < D) acc[0] = fmaf(x, (float)k[lane], acc[0]);
                if (lane + 64 < D) acc[1] = fmaf(x, (float)k[lane + 64], acc[1]);
            }
        }
    }
    if (lane < D) dq[lane] = (T)(acc[0] * a.d.scale);
    if (lane + 64 < D) dq[lane + 64] = (T)(acc[1] * a.d.scale);
}
// A key's dk and dv from the rows that see it alone.
template <typename T>
__device__ void dkv_row(const AttentionArgs& a, const Views<T>& w, const Seq seq, int j, T* dk, T* dv) {
    const int lane = threadIdx.x & 63, D = a.d.head_dim;
    float ak[2] = {0.f, 0.f}, av[2] = {0.f, 0.f};
    const int rows = seq.n * w.group;
    for (int r0 = 0; r0 < rows; r0 += 64) {
        const int r = r0 + lane, i = r / w.group, g = r % w.group;
        float p = 0.f, ds = 0.f;
        const bool seen = r < rows && sees(a.d, seq, i)(j);
        const int ii = r < rows ? i : 0, gg = r < rows ? g : 0;
        const float s = wave_score<T, true>(w.q + ii * a.d.q_stride[1] + gg * a.d.q_stride[2], w.k + j * a.d.k_stride[1], D);
        if (seen) pair_grad(a, w, i, g, j, s, &p, &ds);
        for (uint64_t left = __ballot(seen); left; left &= left - 1) {
            const int l = __ffsll((unsigned long long)left) - 1, rr = r0 + l;
            const float pp = __shfl(p, l), dd = __shfl(ds, l);
            const T* q = w.q + (int64_t)(rr / w.group) * a.d.q_stride[1] + (rr % w.group) * a.d.q_stride[2];
            const T* go = w.dout + (int64_t)(rr / w.group) * a.d.dout_stride[1] + (rr % w.group) * a.d.dout_stride[2];
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int e = lane + 64 * half;
                if (e >= D) continue;
                ak[half] = fmaf(dd, (float)q[e], ak[half]);
                av[half] = fmaf(pp, (float)go[e], av[half]);
            }
        }
    }
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        const int e = lane + 64 * half;
        if (e >= D) continue;
        dk[e] = (T)(ak[half] * a.d.scale);
        dv[e] = (T)av[half];
    }
}

// blocks of 256 threads a compute unit is to hold: two, where the sums and operands
// that stay in registers leave room (dq: one sum, two operands; dk, dv: two and two)
template <typename T, int DP>
constexpr int dq_blocks_per_cu() {
    return sizeof(T) == 2 || DP <= 32 ? 2 : 1;
}
template <typename T, int DP>
constexpr int dkv_blocks_per_cu() {
    return DP * (int)sizeof(T) <= 128 ? 2 : 1;
}
template <typename T, int DP, int ROWS>
constexpr int tile_bytes() {
    return ROWS * Tile<bf16, DP>::kPitch * (sizeof(T) == 2 ? 1 : 3);
}

// A wave's rows of dq: `times` o, and again from memory where that is not finite.
template <typename T, int DP>
__device__ __forceinline__ void store_dq(const AttentionArgs& a, const Views<T>& w, const Seq& seq, int b, int hk, int row0, int lane,
                                         f32x16 (&o)[DP / 32], float times) {
    constexpr int kDT = DP / 32;
    const pd_attention_desc& d = a.d;
    const int h = lane >> 5, row = row0 + (lane & 31);
    const bool real = row < d.q_len * w.group;
    const int qi = real ? row / w.group : 0, g = row % w.group;
    const See see = real ? sees(d, seq, qi) : See{0, 0, 0};
    T* dq = static_cast<T*>(a.dq) + b * d.dq_stride[0] + hk * w.group * d.dq_stride[2];
    bool odd = false;
#pragma unroll
    for (int t = 0; t < kDT; ++t) {
        o[t] = see.none() ? f32x16{} : o[t] * times;
#pragma unroll
        for (int r = 0; r < 16; ++r) odd = odd || !(fabsf(o[t][r]) < INFINITY);
    }
    const uint64_t both = __ballot(odd && real);
    uint32_t again = (uint32_t)both | (uint32_t)(both >> 32);
    if (real && !((again >> (lane & 31)) & 1)) {
        T* to = dq + qi * d.dq_stride[1] + g * d.dq_stride[2];
#pragma unroll
        for (int t = 0; t < kDT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int e = 32 * t + 8 * r + 4 * h;
                store4(to + e, d.head_dim - e, f32x4{o[t][4 * r], o[t][4 * r + 1], o[t][4 * r + 2], o[t][4 * r + 3]});
            }
    }
    if (again) __threadfence();          // this wave's delta, read back below
    while (again) {
        const int rr = row0 + __ffs(again) - 1, i = rr / w.group, gg = rr % w.group;
        again &= again - 1;
        dq_row(a, w, i, gg, sees(d, seq, i), dq + i * d.dq_stride[1] + gg * d.dq_stride[2]);
    }
}

// The kernel's arguments where they lie.
typedef const __attribute__((address_space(4))) AttentionArgs* ArgsPtr;
__device__ __forceinline__ ArgsPtr kernel_arguments() {
    return (ArgsPtr)__builtin_amdgcn_kernarg_segment_ptr();
}

// A wave's 32 rows of dq where some have a large lse, once more: from the keys and values in
// memory, with the largest score so far, the sum over it and dq going along.  (A call, so
// that it takes no registers of the kernel's loop: within it, 230 us became 290 at 128
// values.  Where every row is large 4 x 2304 tokens take 1740 us, else 373.)
template <typename T, int DP>
__device__ __attribute__((noinline)) void dq_again(ArgsPtr args, int b, int hk, int row0) {
    constexpr int kSteps = DP / 16, kDT = DP / 32, BN = tile_rows<T, DP>();
    using As = Held<T, DP, BN>;
    using Operand = typename As::Operand;
    const AttentionArgs& a = *(const AttentionArgs*)(ArgsPtr)uniform_address((const void*)args);
    b = __builtin_amdgcn_readfirstlane(b), hk = __builtin_amdgcn_readfirstlane(hk), row0 = __builtin_amdgcn_readfirstlane(row0);
    const pd_attention_desc& d = a.d;
    const int lane = threadIdx.x & 63, h = lane >> 5, row = row0 + (lane & 31);
    const Seq seq = sequence(a, b);
    const Views<T> w = views<T>(a, b, hk);
    const int rows_all = d.q_len * w.group;
    const bool real = row < rows_all;
    const int qi = real ? row / w.group : 0, g = row % w.group;
    const int64_t at = (int64_t)g * d.q_len + qi;
    const See see = real ? sees(d, seq, qi) : See{0, 0, 0}, see_from = see.from(lane);
    const int i0 = row0 / w.group, i1 = min((row0 + 31) / w.group, seq.n - 1);
    const KeyTiles<32> tiles(i0 <= i1 ? sees_any(d, seq, i0, i1) : See{0, 0, 0});
    const float lse = see.none() ? 0.f : w.lse[at];
    const bool own = is_large(lse);
    Operand qf[kSteps], gf[kSteps];
    float delta = 0.f, top = own ? -INFINITY : lse, total = own ? 0.f : 1.f;
#pragma unroll
    for (int c = 0; c < kSteps; ++c) {
        const int e = 16 * c + 8 * h;
        f32x8 u = {}, x = {}, y = {};
        if (!see.none()) {
            u = widen(load8(w.q + qi * d.q_stride[1] + g * d.q_stride[2] + e, d.head_dim - e));
            x = widen(load8(w.dout + qi * d.dout_stride[1] + g * d.dout_stride[2] + e, d.head_dim - e));
            y = widen(load8(w.out + qi * d.out_stride[1] + g * d.out_stride[2] + e, d.head_dim - e));
        }
        qf[c] = As::make(u);
        gf[c] = As::make(x);
#pragma unroll
        for (int f = 0; f < 8; ++f) delta = fmaf(x[f], y[f], delta);
    }
    delta += __shfl_xor(delta, 32);
    f32x16 o[kDT];
#pragma unroll
    for (int t = 0; t < kDT; ++t) o[t] = f32x16{};
    for (int it = 0; it < tiles.count; ++it) {
        const int j0 = tiles.start(it);
        int dim = __builtin_amdgcn_readfirstlane(d.head_dim);   // (or comparisons with it stay in registers)
        asm volatile("" : "+s"(dim));
        auto from = [&](int r) { return (int64_t)tiles.inside(j0, j0 + r); };
        const T* key = w.k + from(lane & 31) * d.k_stride[1];
        const T* value = w.v + from(lane & 31) * d.v_stride[1];
        f32x16 s = {}, dp = {};
#pragma unroll
        for (int c = 0; c < kSteps; ++c) {
            const int e = 16 * c + 8 * h;
            s = mma(As::make(widen(load8(key + e, dim - e))), qf[c], s);
            dp = mma(As::make(widen(load8(value + e, dim - e))), gf[c], dp);
            __builtin_amdgcn_sched_barrier(0);       // (a step's loads at a time)
        }
        float m = top;
        uint32_t seen = 0;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const bool yes = see_from(j0 + tile_row(0, r));
            seen |= (uint32_t)yes << r;
            s[r] = yes ? s[r] * d.scale : -INFINITY;
            m = fmaxf(m, s[r]);
        }
        m = own ? fmaxf(m, __shfl_xor(m, 32)) : top;
        const float keep = m > top ? exp2_fast((top - m) * kLog2e) : 1.f;
        top = m;
        float sum = 0.f;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const float p = probability(s[r], 1.f, base_of(top, 1.f));
            sum += p;
            s[r] = seen >> r & 1 ? p * (dp[r] - delta) : 0.f;
        }
        total = own ? total * keep + sum : 1.f;
#pragma unroll
        for (int t = 0; t < kDT; ++t) {
            o[t] *= keep;
            const int e = 32 * t + (lane & 31);
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                f32x8 x = {};
#pragma unroll
                for (int f = 0; f < 8; ++f)
                    if (e < dim) x[f] = (float)w.k[from(16 * c + 8 * (f >> 2) + 4 * h + (f & 3)) * d.k_stride[1] + e];
                o[t] = mma(As::make(x), As::make(eight(s, c)), o[t]);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    }
    Base base = {0.f, 1.f};
    if (own) {
        base = base_of(top, total + __shfl_xor(total, 32));
        if (real && h == 0) {
            float* to = const_cast<float*>(w.bases) + 2 * at;
            to[0] = base.from;
            to[1] = base.times;
        }
    }
    store_dq<T, DP>(a, w, seq, b, hk, row0, lane, o, d.scale * base.times);
}

template <typename T, int DP, bool COPY>
__global__ __launch_bounds__(256, (dq_blocks_per_cu<T, DP>())) void k_attention_dq(const AttentionArgs a, int row_tiles) {
    constexpr bool kParts = sizeof(T) == 4;
    constexpr int kSteps = DP / 16, kDT = DP / 32, BN = tile_rows<T, DP>(), kBytes = tile_bytes<T, DP, BN>();
    using As = Held<T, DP, BN>;
    using Operand = typename As::Operand;
    // (one offset: at 128 values the loop else reads offsets back from memory: 2 x 2048 tokens
    // causal 253 us for 235)
    using F = std::conditional_t<kParts, FillParts<DP, BN>, Fill<bf16, DP, BN, 256, DP == 128>>;
    __shared__ __align__(128) char lds[(kParts ? 2 : 4) * kBytes];       // keys, values; twice where copies fill them
    const pd_attention_desc& d = a.d;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
    const int id = near_blocks(blockIdx.x, gridDim.x), tile = row_tiles - 1 - id % row_tiles, head = id / row_tiles;
    const int hk = head % d.heads_kv, b = head / d.heads_kv;
    const Seq seq = sequence(a, b);
    const Views<T> w = views<T>(a, b, hk);
    const int rows_all = d.q_len * w.group;
    const int row0 = tile * 128 + wave * 32, row = row0 + (lane & 31);
    const bool real = row < rows_all;
    const int qi = real ? row / w.group : 0, g = row % w.group;
    const See see = real ? sees(d, seq, qi) : See{0, 0, 0}, see_from = see.from(lane);
    const Sight sight = sight_of(d, seq, row0 / w.group, row0 + 32 <= rows_all ? (row0 + 31) / w.group : seq.n);

    const int i0 = tile * 128 / w.group, i1 = min((tile * 128 + 127) / w.group, seq.n - 1);
    const KeyTiles<BN> tiles(i0 <= i1 ? sees_any(d, seq, i0, i1) : See{0, 0, 0});
    F fk, fv;
    if constexpr (COPY && !kParts) {
        const int units = d.head_dim * (int)sizeof(T) / 16;
        fk.plan(d.k_stride[1], units, threadIdx.x);
        fv.plan(d.v_stride[1], units, threadIdx.x);
    }
    auto fetch = [&](int it, int buf) {
        const int j0 = tiles.start(it);
        const T* kt = w.k + (int64_t)j0 * d.k_stride[1];
        const T* vt = w.v + (int64_t)j0 * d.v_stride[1];
        char* to = lds + buf * 2 * kBytes;
        if constexpr (kParts) {
            auto keep = [&](int r) { return tiles.any(j0 + r); };
            fk.fetch(kt, d.k_stride[1], d.head_dim, keep);
            fv.fetch(vt, d.v_stride[1], d.head_dim, keep);
        } else if constexpr (COPY) {
            if (tiles.whole(j0)) {
                fk.copy(kt, to);
                fv.copy(vt, to + kBytes);
            } else {
                auto from = [&](int r) { return tiles.inside(j0, j0 + r) - j0; };
                fk.copy_some(kt, to, threadIdx.x, from);
                fv.copy_some(vt, to + kBytes, threadIdx.x, from);
            }
        } else {
            auto keep = [&](int r) { return tiles.any(j0 + r); };
            F::load(kt, d.k_stride[1], d.head_dim, to, threadIdx.x, keep);
            F::load(vt, d.v_stride[1], d.head_dim, to + kBytes, threadIdx.x, keep);
        }
    };
    if (tiles.count > 0) fetch(0, 0);

    Operand qf[kSteps], gf[kSteps];
    float delta = 0.f;
#pragma unroll
    for (int c = 0; c < kSteps; ++c) {
        const int e = 16 * c + 8 * h;
        f32x8 u = {}, x = {}, y = {};
        if (!see.none()) {
            u = widen(load8(w.q + qi * d.q_stride[1] + g * d.q_stride[2] + e, d.head_dim - e));
            x = widen(load8(w.dout + qi * d.dout_stride[1] + g * d.dout_stride[2] + e, d.head_dim - e));
            y = widen(load8(w.out + qi * d.out_stride[1] + g * d.out_stride[2] + e, d.head_dim - e));
        }
        qf[c] = As::make(u);
        gf[c] = As::make(x);
#pragma unroll
        for (int f = 0; f < 8; ++f) delta = fmaf(x[f], y[f], delta);
    }
    delta += __shfl_xor(delta, 32);
    const int64_t at = (int64_t)g * d.q_len + qi;
    if (real && h == 0) const_cast<float*>(w.delta)[at] = delta;
    const float c2 = d.scale * kLog2e;
    const float lse = see.none() ? 0.f : w.lse[at];
    const bool large = __any(is_large(lse));
    const float from = sizeof(T) == 2 ? lse * kLog2e : lse;
    f32x16 o[kDT];
#pragma unroll
    for (int t = 0; t < kDT; ++t) o[t] = f32x16{};
    // where the registers allow it the products dout v start from -delta
    constexpr bool kStart = DP * sizeof(T) <= 128;
    f32x16 start = {};
    if constexpr (kStart)
#pragma unroll
        for (int r = 0; r < 16; ++r) start[r] = -delta;
    for (int it = 0; it < tiles.count; ++it) {
        const int j0 = tiles.start(it);
        const char *lk = lds + (kParts ? 0 : (it & 1) * 2 * kBytes), *lv = lk + kBytes;
        if constexpr (kParts) {
            lds_barrier();                                // the tile before has been read
            fk.put(lds);
            fv.put(lds + kBytes);
        } else if constexpr (COPY) {
            wait_copies();
        }
        lds_barrier();                                    // this tile is there, and the other buffer free
        if (it + 1 < tiles.count) fetch(it + 1, (it + 1) & 1);
        if (sight.none(j0, BN)) continue;
        const bool edge = !sight.all(j0, BN);
#pragma unroll
        for (int kt = 0; kt < BN / 32; ++kt) {
            f32x16 s = {}, dp = start;
            // the products q k and dout v, then those with the keys' columns, read ahead
            // (in turn, since a product waits for the last one with the same sum)
            auto rows = [&](int n) { return As::rows(n % 2 ? lv : lk, 32 * kt, n / 2, lane); };
            Stream<Operand, 2 * kSteps> rs;
            rs.begin(rows);
            rs.run(rows, [&](int n, const Operand& f) {
                if (n % 2 == 0)
                    s = mma(f, qf[n / 2], s);
                else
                    dp = mma(f, gf[n / 2], dp);
            });
            auto cols = [&](int n) { return As::cols(lk, 32 * kt + 16 * (n / kDT), n % kDT, lane); };
            Stream<Operand, 2 * kDT> cs;
            cs.begin(cols);
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = probability<T>(s[r], c2, from, d.scale, from);
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] *= kStart ? dp[r] : dp[r] - delta;
            if (edge) {
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (!see_from(j0 + 32 * kt + tile_row(0, r))) s[r] = 0.f;
            }
            Operand ds;
            cs.run(cols, [&](int n, const Operand& f) {
                if (n % kDT == 0) ds = As::make(eight(s, n / kDT));
                o[n % kDT] = mma(f, ds, o[n % kDT]);
            });
        }
    }

    if (large)
        dq_again<T, DP>(kernel_arguments(), b, hk, row0);
    else
        store_dq<T, DP>(a, w, seq, b, hk, row0, lane, o, d.scale);
}

// The queries that see key j: lo <= i < hi.
__device__ inline See seen_by(const pd_attention_desc& d, const Seq& s, int j) {
    if (j >= s.m) return See{0, 0, 0};
    const int off = s.m - s.n;                            // t = off + i
    int lo = 0, hi = s.n;
    if (d.causal) lo = max(lo, j - off);
    if (d.window && j >= d.sinks) {
        hi = min(hi, j + d.window - off);
        if (!d.causal) lo = max(lo, j - d.window + 1 - off);
    }
    return See{lo, max(hi, lo), 0};
}

// The same of the keys j0 .. j1 between them.  The bounds grow with j, but that a sink is
// seen to the last query: the smallest upper bound is the first key's or the first's
// after the sinks.
__device__ inline Sight sight_by(const pd_attention_desc& d, const Seq& s, int j0, int j1) {
    if (j0 >= s.m) return Sight{0, 0, 0, 0, 0, 0};
    const int j2 = min(j1, s.m - 1);
    const See a = seen_by(d, s, j0), b = seen_by(d, s, j2), c = seen_by(d, s, min(max(j0, d.sinks), j2));
    return Sight{a.lo, b.lo, j1 < s.m ? min(a.hi, c.hi) : 0, max(a.hi, b.hi), 0, 0};
}

// A block: 128 keys of one key head, 32 a wave, and the tiles of queries of the group's
// heads that see any of them, or one part of these.
template <typename T, int DP, bool COPY>
__global__ __launch_bounds__(256, (dkv_blocks_per_cu<T, DP>())) void k_attention_dkv(const AttentionArgs a, int key_tiles,
                                                                                   int splits) {
    constexpr bool kParts = sizeof(T) == 4;
    constexpr int kSteps = DP / 16, kDT = DP / 32, BR = tile_rows<T, DP>(), kBytes = tile_bytes<T, DP, BR>();
    using As = Held<T, DP, BR>;
    using Operand = typename As::Operand;
    using F = std::conditional_t<kParts, FillParts<DP, BR>, Fill<bf16, DP, BR, 256>>;
    __shared__ __align__(128) char lds[(kParts ? 2 : 4) * kBytes];       // queries, output gradients; twice where copies fill them
    __shared__ __align__(16) float stats[2][4][64];       // -lse / scale (float32: lse), -delta; where far, the bases
    __shared__ int far[2];                                // whether a row's |lse| is large
    const pd_attention_desc& d = a.d;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
    const int id = near_blocks(blockIdx.x, gridDim.x), split = id % splits, unit = id / splits;
    const int tile = unit % key_tiles, head = unit / key_tiles;
    const int hk = head % d.heads_kv, b = head / d.heads_kv;
    const Seq seq = sequence(a, b);
    const Views<T> w = views<T>(a, b, hk);
    const int key0 = tile * 128, wkey0 = key0 + wave * 32, key = wkey0 + (lane & 31);
    const bool live = key < seq.m;
    const See see = seen_by(d, seq, key).from(lane);
    const Sight sight = sight_by(d, seq, wkey0, wkey0 + 31);

    // the block's queries: from the first that sees its first key (two-sided: its earliest)
    // to the last that sees its last, or a sink among them
    const int k1 = min(key0 + 127, seq.m - 1);
    int first = 0, last = 0;
    if (key0 < seq.m) {
        first = min(seen_by(d, seq, key0).lo, seen_by(d, seq, k1).lo);
        last = max(seen_by(d, seq, key0).hi, seen_by(d, seq, k1).hi);
    }
    const int per_head = last > first ? (last - first + BR - 1) / BR : 0, all = per_head * w.group;
    const int each = (all + splits - 1) / splits, x0 = split * each, x1 = min(all, x0 + each);
    F fq, fg;
    if constexpr (COPY && !kParts) {
        const int units = d.head_dim * (int)sizeof(T) / 16;
        fq.plan(d.q_stride[1], units, threadIdx.x);
        fg.plan(d.dout_stride[1], units, threadIdx.x);
    }
    float stat = 0.f;
    const float over = -1.f / d.scale;
    auto fetch = [&](int x, int buf) {
        const int g = x / per_head, i0 = first + (x - g * per_head) * BR;
        if (threadIdx.x < 2 * BR) {
            const int i = min(i0 + (int)threadIdx.x % BR, seq.n - 1);
            stat = (threadIdx.x < BR ? w.lse : w.delta)[(int64_t)g * d.q_len + i];
        }
        const T* qt = w.q + (int64_t)i0 * d.q_stride[1] + g * d.q_stride[2];
        const T* gt = w.dout + (int64_t)i0 * d.dout_stride[1] + g * d.dout_stride[2];
        char* to = lds + buf * 2 * kBytes;
        if constexpr (kParts) {
            auto keep = [&](int r) { return i0 + r < seq.n; };
            fq.fetch(qt, d.q_stride[1], d.head_dim, keep);
            fg.fetch(gt, d.dout_stride[1], d.head_dim, keep);
        } else if constexpr (COPY) {
            if (i0 + BR <= seq.n) {
                fq.copy(qt, to);
                fg.copy(gt, to + kBytes);
            } else {
                auto from = [&](int r) { return min(i0 + r, seq.n - 1) - i0; };
                fq.copy_some(qt, to, threadIdx.x, from);
                fg.copy_some(gt, to + kBytes, threadIdx.x, from);
            }
        } else {
            auto keep = [&](int r) { return i0 + r < seq.n; };
            F::load(qt, d.q_stride[1], d.head_dim, to, threadIdx.x, keep);
            F::load(gt, d.dout_stride[1], d.head_dim, to + kBytes, threadIdx.x, keep);
        }
    };
    auto put_stat = [&](int x, int buf) {
        if (threadIdx.x < BR) {                           // (lanes of the first wave)
            stats[buf][0][threadIdx.x] = kParts ? stat : stat * over;
            const bool any = __ballot(is_large(stat)) != 0 || !(fabsf(over) < 0x1p100f);      // (a scale near 0)
            if (threadIdx.x == 0) far[buf] = any;
            if (any) {
                Base base = {stat, 1.f};
                if (is_large(stat)) {
                    const int g = x / per_head, i = min(first + (x - g * per_head) * BR + (int)threadIdx.x, seq.n - 1);
                    const float* from = w.bases + 2 * ((int64_t)g * d.q_len + i);
                    base = Base{from[0], from[1]};
                }
                stats[buf][2][threadIdx.x] = base.from;
                stats[buf][3][threadIdx.x] = base.times;
            }
        } else if (threadIdx.x < 2 * BR) {
            stats[buf][1][threadIdx.x - BR] = -stat;
        }
    };
    if (x0 < x1) {
        fetch(x0, 0);
        put_stat(x0, 0);
    }

    Operand kf[kSteps], vf[kSteps];
#pragma unroll
    for (int c = 0; c < kSteps; ++c) {
        const int e = 16 * c + 8 * h;
        f32x8 u = {}, v = {};
        if (live) {
            u = widen(load8(w.k + (int64_t)key * d.k_stride[1] + e, d.head_dim - e));
            v = widen(load8(w.v + (int64_t)key * d.v_stride[1] + e, d.head_dim - e));
        }
        kf[c] = As::make(u);
        vf[c] = As::make(v);
    }
    const float c2 = d.scale * kLog2e;
    f32x16 dk[kDT], dv[kDT];
#pragma unroll
    for (int t = 0; t < kDT; ++t) dk[t] = dv[t] = f32x16{};
    int pos = per_head ? x0 % per_head : 0;               // the tile's place among its head's
    for (int x = x0; x < x1; ++x, pos = pos + 1 == per_head ? 0 : pos + 1) {
        const int buf = (x - x0) & 1, i0 = first + pos * BR;
        if constexpr (kParts) {
            lds_barrier();                                // the tile before has been read
            fq.put(lds);
            fg.put(lds + kBytes);
        } else if constexpr (COPY) {
            wait_copies();
        }
        lds_barrier();                                    // this tile is there, and the other buffer free
        if (x + 1 < x1) fetch(x + 1, buf ^ 1);
        if (!sight.none(i0, BR)) {
            const bool edge = !sight.all(i0, BR);
            const char *lq = lds + (kParts ? 0 : buf * 2 * kBytes), *lg = lq + kBytes;
            const bool large = __builtin_amdgcn_readfirstlane(far[buf]);
#pragma unroll
            for (int rt = 0; rt < BR / 32; ++rt) {
                // the products dout v start from -delta and, in bfloat16, q k from -lse / scale,
                // so that ds = p dp and p = 2^(c2 s) (float32: see probability)
                f32x16 s, dp;
#pragma unroll
                for (int r = 0; r < 16; r += 4) {
                    const int at = 32 * rt + tile_row(lane, r);
                    const f32x4 u = *reinterpret_cast<const f32x4*>(&stats[buf][0][at]);
                    const f32x4 v = *reinterpret_cast<const f32x4*>(&stats[buf][1][at]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[r + e] = u[e], dp[r + e] = v[e];
                }
                const f32x16 from = s;
                if (large || kParts) s = f32x16{};
                auto rows = [&](int n) { return As::rows(n % 2 ? lg : lq, 32 * rt, n / 2, lane); };
                Stream<Operand, 2 * kSteps> rs;
                rs.begin(rows);
                rs.run(rows, [&](int n, const Operand& f) {
                    if (n % 2 == 0)
                        s = mma_turned(f, kf[n / 2], s);
                    else
                        dp = mma(f, vf[n / 2], dp);
                });
                // then, 16 rows at a time, dv with the output gradients' columns and dk with the queries'
                auto cols = [&](int n) {
                    const int c = n / (2 * kDT), t = n % (2 * kDT);
                    return t < kDT ? As::cols(lg, 32 * rt + 16 * c, t, lane) : As::cols(lq, 32 * rt + 16 * c, t - kDT, lane);
                };
                Stream<Operand, 4 * kDT> cs;
                cs.begin(cols);
                if (large) {
#pragma unroll
                    for (int r = 0; r < 16; r += 4) {
                        const int at = 32 * rt + tile_row(lane, r);
                        const f32x4 u = *reinterpret_cast<const f32x4*>(&stats[buf][2][at]);
                        const f32x4 v = *reinterpret_cast<const f32x4*>(&stats[buf][3][at]);
#pragma unroll
                        for (int e = 0; e < 4; ++e) s[r + e] = probability(s[r + e], d.scale, Base{u[e], v[e]});
                    }
                } else if constexpr (kParts) {
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[r] = probability<T>(s[r], 0.f, 0.f, d.scale, from[r]);
                } else {
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[r] = exp2_fast(s[r] * c2);
                }
#pragma unroll
                for (int r = 0; r < 16; ++r) dp[r] *= s[r];
                if (edge) {
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (!see(i0 + 32 * rt + tile_row(0, r))) s[r] = dp[r] = 0.f;
                }
                Operand p, ds;
                cs.run(cols, [&](int n, const Operand& f) {
                    const int c = n / (2 * kDT), t = n % (2 * kDT);
                    if (t == 0) p = As::make(eight(s, c)), ds = As::make(eight(dp, c));
                    if (t < kDT)
                        dv[t] = mma(f, p, dv[t]);
                    else
                        dk[t - kDT] = mma(f, ds, dk[t - kDT]);
                });
            }
        }
        if (x + 1 < x1) put_stat(x + 1, buf ^ 1);
    }

#pragma unroll
    for (int t = 0; t < kDT; ++t) dk[t] *= d.scale;
    if (splits > 1) {
        if (key >= d.kv_len) return;
        const int64_t keys = (int64_t)d.batch * d.heads_kv * d.kv_len, kat = ((int64_t)b * d.heads_kv + hk) * d.kv_len + key;
        float* to = dkv_parts(a) + (split * keys + kat) * 2 * d.head_dim;
#pragma unroll
        for (int t = 0; t < kDT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int e = 32 * t + 8 * r + 4 * h;
                store4(to + e, d.head_dim - e, f32x4{dk[t][4 * r], dk[t][4 * r + 1], dk[t][4 * r + 2], dk[t][4 * r + 3]});
                store4(to + d.head_dim + e, d.head_dim - e,
                       f32x4{dv[t][4 * r], dv[t][4 * r + 1], dv[t][4 * r + 2], dv[t][4 * r + 3]});
            }
        return;
    }
    bool odd = false;
#pragma unroll
    for (int t = 0; t < kDT; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) odd = odd || !(fabsf(dk[t][r]) < INFINITY) || !(fabsf(dv[t][r]) < INFINITY);
    T* dkp = static_cast<T*>(a.dk) + b * d.dk_stride[0] + hk * d.dk_stride[2];
    T* dvp = static_cast<T*>(a.dv) + b * d.dv_stride[0] + hk * d.dv_stride[2];
    const uint64_t both = __ballot(odd && live);
    uint32_t again = (uint32_t)both | (uint32_t)(both >> 32);
    if (key < d.kv_len && !((again >> (lane & 31)) & 1)) {
#pragma unroll
        for (int t = 0; t < kDT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int e = 32 * t + 8 * r + 4 * h;
                f32x4 x = {}, y = {};
                if (live) {
                    x = f32x4{dk[t][4 * r], dk[t][4 * r + 1], dk[t][4 * r + 2], dk[t][4 * r + 3]};
                    y = f32x4{dv[t][4 * r], dv[t][4 * r + 1], dv[t][4 * r + 2], dv[t][4 * r + 3]};
                }
                store4(dkp + (int64_t)key * d.dk_stride[1] + e, d.head_dim - e, x);
                store4(dvp + (int64_t)key * d.dv_stride[1] + e, d.head_dim - e, y);
            }
    }
    while (again) {
        const int j = wkey0 + __ffs(again) - 1;
        again &= again - 1;
        dkv_row(a, w, seq, j, dkp + (int64_t)j * d.dk_stride[1], dvp + (int64_t)j * d.dv_stride[1]);
    }
}

// The parts of a key's dk and dv into the result: one wave a key.  (Eight waves a SIMD, or
// the registers of the path for keys that are not finite leave room for five: 25 us for 21.)
template <typename T>
__global__ __launch_bounds__(256, 8) void k_attention_dkv_join(const AttentionArgs a, int splits) {
    const pd_attention_desc& d = a.d;
    const int lane = threadIdx.x & 63, D = d.head_dim;
    const int64_t keys = (int64_t)d.batch * d.heads_kv * d.kv_len, kat = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (kat >= keys) return;
    const int j = (int)(kat % d.kv_len), hk = (int)(kat / d.kv_len % d.heads_kv), b = (int)(kat / d.kv_len / d.heads_kv);
    const Seq seq = sequence(a, b);
    const bool live = j < seq.m;
    float v[4] = {0.f, 0.f, 0.f, 0.f};                    // dk, dv at lane; at lane + 64
    bool odd = false;
    if (live)
        for (int s = 0; s < splits; ++s) {
            const float* from = dkv_parts(a) + (s * keys + kat) * 2 * D;
#pragma unroll
            for (int half = 0; half < 2; ++half)
                if (lane + 64 * half < D) {
                    v[2 * half] += from[lane + 64 * half];
                    v[2 * half + 1] += from[D + lane + 64 * half];
                }
        }
#pragma unroll
    for (int i = 0; i < 4; ++i) odd = odd || !(fabsf(v[i]) < INFINITY);
    T* dk = static_cast<T*>(a.dk) + b * d.dk_stride[0] + hk * d.dk_stride[2] + j * d.dk_stride[1];
    T* dv = static_cast<T*>(a.dv) + b * d.dv_stride[0] + hk * d.dv_stride[2] + j * d.dv_stride[1];
    if (__any(odd)) return dkv_row(a, views<T>(a, b, hk), seq, j, dk, dv);
#pragma unroll
    for (int half = 0; half < 2; ++half)
        if (lane + 64 * half < D) {
            dk[lane + 64 * half] = (T)v[2 * half];
            dv[lane + 64 * half] = (T)v[2 * half + 1];
        }
}

// Parts of the dk, dv kernel's queries, of at least four tiles where no window leaves some
// out: the fewest that keep its blocks at work for nine tenths of the time (512 run at
// once: 288 blocks in 4 parts are 2.25 rounds of them, in 5 parts 2.8), or the best up to
// eight.  All blocks are cut alike, as suits blocks of like length.  With a window and sinks
// they are not: the block that holds a sink goes through all queries, the others through
// 128 and the window (8192 tokens, window 1024, 16 heads on 4: 176 us, with four sinks 682).
int dkv_splits(const pd_attention_desc& d) {
    const int64_t blocks = ((int64_t)d.kv_len + 127) / 128 * d.heads_kv * d.batch;
    const int64_t most = ((int64_t)d.q_len + 63) / 64 * (d.heads_q / d.heads_kv) / 4;
    int64_t best = 1;
    double used = 0.0;
    for (int64_t s = 1; s <= 8 && (s == 1 || s <= most) && used < 0.9; ++s) {
        const int64_t n = blocks * s, rounds = (n + 511) / 512;
        const double u = (double)n / (double)(rounds * 512);
        if (u > used) best = s, used = u;
    }
    return (int)best;
}

template <typename T, int DP, bool COPY>
void attention_grad_c(const AttentionArgs& a, hipStream_t s) {
    const int64_t rows = (int64_t)a.d.q_len * (a.d.heads_q / a.d.heads_kv), heads = (int64_t)a.d.heads_kv * a.d.batch;
    const int row_tiles = (int)((rows + 127) / 128), key_tiles = (int)(((int64_t)a.d.kv_len + 127) / 128);
    if (rows) {
        hipLaunchKernelGGL((k_attention_dq<T, DP, COPY>), dim3((unsigned)(row_tiles * heads)), dim3(256), 0, s, a, row_tiles);
        PD_HIP(hipGetLastError());
    }
    if (!a.d.kv_len) return;
    const int splits = dkv_splits(a.d);
    hipLaunchKernelGGL((k_attention_dkv<T, DP, COPY>), dim3((unsigned)(key_tiles * heads * splits)), dim3(256), 0, s, a, key_tiles,
                       splits);
    PD_HIP(hipGetLastError());
    if (splits == 1) return;
    hipLaunchKernelGGL((k_attention_dkv_join<T>), dim3((unsigned)((heads * a.d.kv_len + 3) / 4)), dim3(256), 0, s, a, splits);
    PD_HIP(hipGetLastError());
}
template <typename T, int DP>
void attention_grad_t(const AttentionArgs& a, hipStream_t s) {
    const pd_attention_desc& d = a.d;
    auto fits = [&](const void* p, const int64_t* stride, int64_t tokens, int64_t heads) {
        return copies_fit(p, stride, d.batch, tokens, heads, d.head_dim, sizeof(T));
    };
    if constexpr (sizeof(T) == 4)
        attention_grad_c<T, DP, false>(a, s);
    else if (fits(a.k, d.k_stride, d.kv_len, d.heads_kv) && fits(a.v, d.v_stride, d.kv_len, d.heads_kv) &&
        fits(a.q, d.q_stride, d.q_len, d.heads_q) && fits(a.dout, d.dout_stride, d.q_len, d.heads_q))
        attention_grad_c<T, DP, true>(a, s);
    else
        attention_grad_c<T, DP, false>(a, s);
}
template <typename T>
void attention_grad_dim(const AttentionArgs& a, hipStream_t s) {
    if (a.d.head_dim <= 32) return attention_grad_t<T, 32>(a, s);
    if (a.d.head_dim <= 64) return attention_grad_t<T, 64>(a, s);
    if (a.d.head_dim <= 96) return attention_grad_t<T, 96>(a, s);
    attention_grad_t<T, 128>(a, s);
}

}  // namespace

int64_t attention_grad_scratch_bytes(const pd_attention_desc& d) {
    const int splits = dkv_splits(d);
    const int64_t parts = splits == 1 ? 0 : (int64_t)splits * d.batch * d.heads_kv * d.kv_len * 2 * d.head_dim;
    return (row_floats(d) + parts) * (int64_t)sizeof(float);
}

void launch_attention_grad(const AttentionArgs& a, hipStream_t s) {
    a.d.dtype == PD_F32 ? attention_grad_dim<float>(a, s) : attention_grad_dim<bf16>(a, s);
}

}  // namespace pd
