// Attention with a sliding window and sinks, forward.
//
//   x_ij = scale q_i k_j over the keys that query i sees,  o_i = sum_j e^(x_ij - m_i) v_j / l_i
//
// One pass over the keys with a running reference m and sum l, in base 2: p = 2^(s c
// - m c), c = scale log2 e, one fused multiply-add and one exponential a score.  m
// is the row's largest score of some earlier tile: it is raised, and o and l
// rescaled, only when a score passes it by 2^8 (the terms are float32, and a
// bfloat16 probability is rounded relative to itself, so nothing is lost below that).
// The product m c is rounded: a shift of all of a row's terms, without effect while
// it is small.  Where |m c| passes 1024 the difference (s - m) c is formed instead,
// exact for the row's largest scores of any size.
//
// A row is a query of one of the query heads that share a key head: keys and values
// are read once for all of them.  Blocks of 128 rows share the key tiles in LDS
// (k_attention; float32: k_attention_parts); at most 32 rows (a token's heads, a short
// sequence) go to waves that stream key tiles of their own (k_attention_few).  Where
// there are few blocks the keys are split among several of them, whose results
// k_attention_join puts together.
//
// What bounds it: a 32 x 32 x 16 product takes 32 cycles and 16 of the vector units' issue, a
// score 12 cycles of vector operations and 8 for its exponential, and within a wave
// nothing overlaps a product, so two waves a SIMD from different blocks fill it
// between them.  Measured (bfloat16): 8192 tokens two-sided, 32 heads on 8 of 128 values,
// 1063 us (1034 TFLOP/s; a large library product reaches 1247), of 64 values 567 us
// (970); with a window of 2048 and sinks, where tiles end outside the window and a block
// has 34 of them, 277 us (868); 64 sequences of 576 tokens of 64 values, nine tiles a block,
// 132 us (661): there a third of the time is reading queries and writing results.
//
// bfloat16 rounds a probability once more, as the matrix instruction's operand (the sum
// takes it unrounded): relative to itself, so the result's error is 2.3e-3 where the
// result's own rounding alone makes 1.7e-3.  Two parts would take half as many products
// again.
#include "attention_tile.h"

namespace pd {
namespace {

using namespace attn;

constexpr float kLarge = 1024.f;
constexpr float kSlack = 8.f;        // log2 of what a score may pass its reference by

// The row's result from its visible keys alone, one after the other: for rows
// whose fast sum is not finite.  There a probability of 0 for a key out of
// sight met an infinity or NaN among its values; here such keys are not read.
// The whole wave works on the row.
template <typename T>
__device__ void attend_row(const AttentionArgs& a, const T* q, const T* k, const T* v, const See see, T* out, float* lse) {
    const int lane = threadIdx.x & 63, D = a.d.head_dim;
    float top = -INFINITY, total = 0.f, acc[2] = {0.f, 0.f};
    for (int part = 0; part < 2; ++part) {
        const int j0 = part == 0 ? 0 : max(see.lo, see.sk), j1 = part == 0 ? see.sk : see.hi;
        for (int jb = j0; jb < j1; jb += 64) {
            const int j = jb + lane, count = min(64, j1 - jb);
            float x = -INFINITY;
            if (lane < count) {
                float s = 0.f;
                for (int e = 0; e < D; ++e) s = fmaf((float)q[e], (float)k[(int64_t)j * a.d.k_stride[1] + e], s);
                x = s * a.d.scale;
            }
            float m = x;
#pragma unroll
            for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
            m = fmaxf(m, top);
            const float base = m == -INFINITY ? 0.f : m;
            const float p = lane < count ? exp2_fast((x - base) * kLog2e) : 0.f, keep = exp2_fast((top - base) * kLog2e);
            float sum = p;
#pragma unroll
            for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
            total = total * keep + sum;
            top = m;
            acc[0] *= keep;
            acc[1] *= keep;
            for (int jj = 0; jj < count; ++jj) {
                const float pj = __shfl(p, jj);
                const T* vj = v + (int64_t)(jb + jj) * a.d.v_stride[1];
                if (lane < D) acc[0] = fmaf(pj, (float)vj[lane], acc[0]);
                if (lane + 64 < D) acc[1] = fmaf(pj, (float)vj[lane + 64], acc[1]);
            }
        }
    }
    const float inv = total == 0.f ? 0.f : 1.f / total;     // (no score above -inf: 0, as for a row that sees nothing)
    if (lane < D) out[lane] = (T)(acc[0] * inv);
    if (lane + 64 < D) out[lane + 64] = (T)(acc[1] * inv);
    if (lse && lane == 0) *lse = log_sum(top, 1.f, total);
}

// The 32 QT rows of a wave (lane: rows 32 t + lane % 32) and what they have summed.
template <class As, int DP, int QT>
struct Rows {
    static constexpr int kSteps = DP / 16, kDT = DP / 32;
    using T = typename As::Type;
    using Operand = typename As::Operand;
    Operand q[QT][kSteps];
    f32x16 o[QT][kDT];           // transposed: the lane's row, columns 32 t + tile_row
    float top[QT], limit[QT];    // the reference and the score that raises it (unscaled)
    float mc[QT];                // top c2
    float total[QT];             // over the keys of this half of the wave
    float c2;
    bool large;

    __device__ __forceinline__ void start(const pd_attention_desc& d) {
        // the reference is one of unscaled scores: c2 > 0 (a scale of 0: zero queries)
        c2 = d.scale == 0.f ? 1.f : fabsf(d.scale) * kLog2e;
        large = false;
#pragma unroll
        for (int i = 0; i < QT; ++i) {
#pragma unroll
            for (int t = 0; t < kDT; ++t) o[i][t] = f32x16{};
            top[i] = limit[i] = -INFINITY;
            mc[i] = total[i] = 0.f;
        }
    }
    __device__ __forceinline__ void load(int i, const pd_attention_desc& d, const T* qp, bool real, int lane) {
        const int h = lane >> 5;
#pragma unroll
        for (int c = 0; c < kSteps; ++c) {
            const int e = 16 * c + 8 * h;
            f32x8 v = {};
            if (real && d.scale != 0.f) v = widen(load8(qp + e, d.head_dim - e));
            q[i][c] = As::make(d.scale < 0.f ? -v : v);
        }
    }

    // 32 NK keys from j0 on, in LDS; `edge`: some row does not see all of them; `half`:
    // none sees one past the first 16.  `see` is from(lane).
    template <int NK>
    __device__ __forceinline__ void attend(const char* k, const char* v, int j0, const See (&see)[QT], bool edge, int lane,
                                           bool half = false) {
        f32x16 s[QT][NK];
        __builtin_amdgcn_s_setprio(1);       // matrix instructions go first: the other wave's vector ones fill in
#pragma unroll
        for (int kt = 0; kt < NK; ++kt) {
#pragma unroll
            for (int i = 0; i < QT; ++i) s[i][kt] = f32x16{};
#pragma unroll
            for (int c = 0; c < kSteps; ++c) {
                const Operand f = As::rows(k, 32 * kt, c, lane);
#pragma unroll
                for (int i = 0; i < QT; ++i) s[i][kt] = mma(f, q[i][c], s[i][kt]);
            }
        }
        __builtin_amdgcn_s_setprio(0);
        if (edge) {
#pragma unroll
            for (int i = 0; i < QT; ++i)
#pragma unroll
                for (int kt = 0; kt < NK; ++kt)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (!see[i](j0 + 32 * kt + tile_row(0, r))) s[i][kt][r] = -INFINITY;
        }
        float m[QT];
        bool raise = false;
#pragma unroll
        for (int i = 0; i < QT; ++i) {
            m[i] = s[i][0][0];
#pragma unroll
            for (int kt = 0; kt < NK; ++kt)
#pragma unroll
                for (int r = 0; r < 16; ++r) m[i] = fmaxf(m[i], s[i][kt][r]);
            const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(m[i]), __float_as_uint(m[i]), false, false);
            m[i] = fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1]));
            raise = raise || m[i] > limit[i];
        }
        if (__any(raise)) {
            bool far = false;
#pragma unroll
            for (int i = 0; i < QT; ++i) {
                const float up = fmaxf(m[i], top[i]);
                const float keep = up == top[i] ? 1.f : exp2_fast((top[i] - up) * c2);
                top[i] = up;
                limit[i] = up + kSlack / c2;
                mc[i] = up == -INFINITY ? 0.f : up * c2;
                far = far || !(fabsf(mc[i]) < kLarge);
                total[i] *= keep;
#pragma unroll
                for (int t = 0; t < kDT; ++t) o[i][t] *= keep;
            }
            large = __any(far);
        }
#pragma unroll
        for (int i = 0; i < QT; ++i) {
            float sum = 0.f;
            if (large) {
#pragma unroll
                for (int kt = 0; kt < NK; ++kt)
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const float x = s[i][kt][r];
                        s[i][kt][r] = x == -INFINITY ? 0.f : exp2_fast((x - top[i]) * c2);
                        sum += s[i][kt][r];
                    }
            } else {
#pragma unroll
                for (int kt = 0; kt < NK; ++kt)
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        s[i][kt][r] = exp2_fast(fmaf(s[i][kt][r], c2, -mc[i]));
                        sum += s[i][kt][r];
                    }
            }
            total[i] += sum;
        }
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int kt = 0; kt < NK; ++kt)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                if (c == 1 && half) continue;
                Operand p[QT];
#pragma unroll
                for (int i = 0; i < QT; ++i) p[i] = As::make(eight(s[i][kt], c));
#pragma unroll
                for (int t = 0; t < kDT; ++t) {
                    const Operand f = As::cols(v, 32 * kt + 16 * c, t, lane);
#pragma unroll
                    for (int i = 0; i < QT; ++i) o[i][t] = mma(f, p[i], o[i][t]);
                }
            }
        __builtin_amdgcn_s_setprio(0);
    }

    __device__ __forceinline__ void finish(int i) { total[i] += __shfl_xor(total[i], 32); }
    // whether a value of the lane's row is not finite
    __device__ __forceinline__ bool odd(int i) const {
        float x = 0.f;                   // 0 times what is not finite is NaN
#pragma unroll
        for (int t = 0; t < kDT; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) x = fmaf(o[i][t][r], 0.f, x);
        return x != 0.f;
    }
};

// Where the parts of split rows go: [split][row over batch, query head, query] of
// (head_dim sums, reference, total).
struct Parts {
    float* sums;
    float* stats;      // [..][2]
};
__host__ __device__ inline Parts parts(const pd_attention_desc& d, float* scratch, int splits) {
    const int64_t rows = (int64_t)d.batch * d.heads_q * d.q_len;
    return Parts{scratch + (((int64_t)splits * rows * 2 + 3) & ~(int64_t)3), scratch};
}

// Which wave does what.
struct Plan {
    int group, rows;           // rows of a key head: group * q_len
    int shift;                 // group = 2^shift, or -1
    int row_tiles;             // of 128 wave_tiles rows, or of 32
    int splits, split_tiles;   // parts of the key tiles, and the tiles of each
    int64_t units;             // row tiles over all key heads and sequences
    int waves;                 // few rows: waves that share a part's tiles
    int wave_tiles;            // else: tiles of 32 rows a wave
};

__device__ inline int rows_to_query(const Plan& p, int row) { return p.shift >= 0 ? row >> p.shift : row / p.group; }

// The rows row0 .. row0 + 31, tile x of the wave's.
template <class As, int DP, int QT>
__device__ __forceinline__ void store_rows(const AttentionArgs& a, const Plan& p, Rows<As, DP, QT>& w, int x, const Seq& seq, int b,
                                           int hk, int row0, int split, const typename As::Type* kb, const typename As::Type* vb) {
    using T = typename As::Type;
    const pd_attention_desc& d = a.d;
    const int lane = threadIdx.x & 63, h = lane >> 5, row = row0 + (lane & 31);
    const bool real = row < p.rows;
    const int qi = real ? rows_to_query(p, row) : 0, hq = hk * p.group + (real ? row - qi * p.group : 0);
    w.finish(x);
    if (p.splits > 1) {
        const Parts to = parts(d, a.scratch, p.splits);
        const int64_t at = ((int64_t)split * d.batch + b) * d.heads_q * d.q_len + (int64_t)hq * d.q_len + qi;
        if (!real) return;
        if (h == 0) {
            to.stats[2 * at] = w.top[x];
            to.stats[2 * at + 1] = w.total[x];
        }
        if (w.total[x] == 0.f) return;            // the join leaves such parts out
        float* sums = to.sums + at * d.head_dim;
#pragma unroll
        for (int t = 0; t < w.kDT; ++t)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int e = 32 * t + 8 * g + 4 * h;
                store4(sums + e, d.head_dim - e, f32x4{w.o[x][t][4 * g], w.o[x][t][4 * g + 1], w.o[x][t][4 * g + 2], w.o[x][t][4 * g + 3]});
            }
        return;
    }
    // a row that sees nothing: 0, also where 0 met a NaN
    const float inv = w.total[x] == 0.f ? 0.f : 1.f / w.total[x];
#pragma unroll
    for (int t = 0; t < w.kDT; ++t) w.o[x][t] *= inv;
    const bool odd = w.odd(x);
    if (__any(odd && w.total[x] == 0.f))
#pragma unroll
        for (int t = 0; t < w.kDT; ++t) w.o[x][t] = w.total[x] == 0.f ? f32x16{} : w.o[x][t];
    const uint64_t both = __ballot(odd && w.total[x] != 0.f && real);
    uint32_t again = (uint32_t)both | (uint32_t)(both >> 32);
    if (real && !((again >> (lane & 31)) & 1)) {
        T* out = static_cast<T*>(a.out) + b * d.out_stride[0] + qi * d.out_stride[1] + hq * d.out_stride[2];
#pragma unroll
        for (int t = 0; t < w.kDT; ++t)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int e = 32 * t + 8 * g + 4 * h;
                store4(out + e, d.head_dim - e, f32x4{w.o[x][t][4 * g], w.o[x][t][4 * g + 1], w.o[x][t][4 * g + 2], w.o[x][t][4 * g + 3]});
            }
        if (a.lse && h == 0)
            a.lse[((int64_t)b * d.heads_q + hq) * d.q_len + qi] = log_sum(w.top[x], fabsf(d.scale), w.total[x]);
    }
    while (again) {
        const int rr = row0 + __ffs(again) - 1;
        again &= again - 1;
        const int i = rr / p.group, hh = hk * p.group + rr % p.group;
        attend_row<T>(a, static_cast<const T*>(a.q) + b * d.q_stride[0] + i * d.q_stride[1] + hh * d.q_stride[2], kb, vb,
                      sees(d, seq, i), static_cast<T*>(a.out) + b * d.out_stride[0] + i * d.out_stride[1] + hh * d.out_stride[2],
                      a.lse ? a.lse + ((int64_t)b * d.heads_q + hh) * d.q_len + i : nullptr);
    }
}

// 32-row tiles of a wave: two where their sums and operands leave room for two waves a
// SIMD, since both then read each key and value once from LDS.
template <typename T, int DP>
constexpr int wave_tiles() {
    return sizeof(T) == 2 && DP <= 64 ? 2 : 1;
}

// A block: 128 QT rows of one key head, or one part of their keys.  The next tile of keys
// and values is copied to LDS while the waves work on the present one.
template <typename T, int DP, bool COPY, int QT>
__global__ __launch_bounds__(256, 2) void k_attention(const AttentionArgs a, const Plan p) {
    using Ti = Tile<T, DP>;
    constexpr int BN = tile_rows<T, DP>(), kBytes = BN * Ti::kPitch, BM = 128 * QT;
    using F = Fill<T, DP, BN, 256>;
    __shared__ __align__(128) char lds[4 * kBytes];       // keys, values; twice
    const pd_attention_desc& d = a.d;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int id = near_blocks(blockIdx.x, gridDim.x);
    const int split = id % p.splits, unit = id / p.splits;
    const int tile = p.row_tiles - 1 - unit % p.row_tiles, head = unit / p.row_tiles;     // the longest rows first
    const int hk = head % d.heads_kv, b = head / d.heads_kv;
    const Seq seq = sequence(a, b);
    const int row0 = tile * BM + wave * 32 * QT;
    const T* kb = static_cast<const T*>(a.k) + b * d.k_stride[0] + hk * d.k_stride[2];
    const T* vb = static_cast<const T*>(a.v) + b * d.v_stride[0] + hk * d.v_stride[2];

    const int i0 = rows_to_query(p, tile * BM), i1 = min(rows_to_query(p, tile * BM + BM - 1), seq.n - 1);
    const KeyTiles<BN> tiles(i0 <= i1 ? sees_any(d, seq, i0, i1) : See{0, 0, 0});
    const int it0 = split * p.split_tiles, it1 = min(tiles.count, it0 + p.split_tiles);
    F fk, fv;
    if constexpr (COPY) {
        const int units = d.head_dim * (int)sizeof(T) / 16;
        fk.plan(d.k_stride[1], units, threadIdx.x);
        fv.plan(d.v_stride[1], units, threadIdx.x);
    }
    auto fetch = [&](int it, int buf) {
        const int j0 = tiles.start(it);
        const T* kt = kb + (int64_t)j0 * d.k_stride[1];
        const T* vt = vb + (int64_t)j0 * d.v_stride[1];
        char* to = lds + buf * 2 * kBytes;
        if constexpr (COPY) {
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
    if (it0 < it1) fetch(it0, 0);

    Rows<AsIs<T, DP>, DP, QT> w;
    w.start(d);
    See see[QT];
    const Sight sight = sight_of(d, seq, rows_to_query(p, row0), row0 + 32 * QT <= p.rows ? rows_to_query(p, row0 + 32 * QT - 1) : seq.n);
#pragma unroll
    for (int x = 0; x < QT; ++x) {
        const int row = row0 + 32 * x + (lane & 31);
        const bool real = row < p.rows;
        const int qi = real ? rows_to_query(p, row) : 0, hq = hk * p.group + (real ? row - qi * p.group : 0);
        see[x] = real ? sees(d, seq, qi) : See{0, 0, 0};
        w.load(x, d, static_cast<const T*>(a.q) + b * d.q_stride[0] + qi * d.q_stride[1] + hq * d.q_stride[2],
               real && !see[x].none(), lane);
        see[x] = see[x].from(lane);
    }
    for (int it = it0; it < it1; ++it) {
        const int buf = (it - it0) & 1, j0 = tiles.start(it);
        if constexpr (COPY) wait_copies();
        lds_barrier();                                    // this tile is there, the other buffer is free
        if (it + 1 < it1) fetch(it + 1, buf ^ 1);
        if (sight.none(j0, BN)) continue;
        const char* at = lds + buf * 2 * kBytes;
        w.template attend<BN / 32>(at, at + kBytes, j0, see, !sight.all(j0, BN), lane);
    }
#pragma unroll
    for (int x = 0; x < QT; ++x) store_rows(a, p, w, x, seq, b, hk, row0 + 32 * x, split, kb, vb);
}

// The same for float32, in three parts: a tile is read into registers while the one
// before is worked on, and split on its way to LDS, once for the block's four waves.
// (Heads of over 96 values: one block a compute unit, since for two 33 registers spill:
// 278 us, 357.)  Measured: 2 x 2048 tokens causal, 16 heads on 4: 64 values 138 us, 96 values
// 210 us, 128 values 278 us, where float32 products took 213, 313 and 570.
template <int DP>
__global__ __launch_bounds__(256, (DP <= 96 ? 2 : 1)) void k_attention_parts(const AttentionArgs a, const Plan p) {
    constexpr int BN = tile_rows<float, DP>(), BM = 128;
    using As = InParts<DP, BN>;
    __shared__ __align__(128) char lds[2 * As::kBytes];   // keys, values
    char *lk = lds, *lv = lds + As::kBytes;
    const pd_attention_desc& d = a.d;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int id = near_blocks(blockIdx.x, gridDim.x);
    const int part = id % p.splits, unit = id / p.splits;
    const int tile = p.row_tiles - 1 - unit % p.row_tiles, head = unit / p.row_tiles;     // the longest rows first
    const int hk = head % d.heads_kv, b = head / d.heads_kv;
    const Seq seq = sequence(a, b);
    const int row0 = tile * BM + wave * 32, row = row0 + (lane & 31);
    const float* kb = static_cast<const float*>(a.k) + b * d.k_stride[0] + hk * d.k_stride[2];
    const float* vb = static_cast<const float*>(a.v) + b * d.v_stride[0] + hk * d.v_stride[2];

    const int i0 = rows_to_query(p, tile * BM), i1 = min(rows_to_query(p, tile * BM + BM - 1), seq.n - 1);
    const KeyTiles<BN> tiles(i0 <= i1 ? sees_any(d, seq, i0, i1) : See{0, 0, 0});
    const int it0 = part * p.split_tiles, it1 = min(tiles.count, it0 + p.split_tiles);
    FillParts<DP, BN> fk, fv;
    auto fetch = [&](int it) {
        const int j0 = tiles.start(it);
        auto keep = [&](int r) { return tiles.any(j0 + r); };
        fk.fetch(kb + (int64_t)j0 * d.k_stride[1], d.k_stride[1], d.head_dim, keep);
        fv.fetch(vb + (int64_t)j0 * d.v_stride[1], d.v_stride[1], d.head_dim, keep);
    };
    if (it0 < it1) fetch(it0);

    Rows<As, DP, 1> w;
    w.start(d);
    const Sight sight = sight_of(d, seq, rows_to_query(p, row0), row0 + 32 <= p.rows ? rows_to_query(p, row0 + 31) : seq.n);
    const bool real = row < p.rows;
    const int qi = real ? rows_to_query(p, row) : 0, hq = hk * p.group + (real ? row - qi * p.group : 0);
    See see[1] = {real ? sees(d, seq, qi) : See{0, 0, 0}};
    w.load(0, d, static_cast<const float*>(a.q) + b * d.q_stride[0] + qi * d.q_stride[1] + hq * d.q_stride[2],
           real && !see[0].none(), lane);
    see[0] = see[0].from(lane);
    for (int it = it0; it < it1; ++it) {
        const int j0 = tiles.start(it);
        lds_barrier();                                    // the tile before has been read
        fk.put(lk);
        fv.put(lv);
        lds_barrier();                                    // this one is there
        if (it + 1 < it1) fetch(it + 1);
        if (sight.none(j0, BN)) continue;
        w.template attend<BN / 32>(lk, lv, j0, see, !sight.all(j0, BN), lane);
    }
    store_rows(a, p, w, 0, seq, b, hk, row0, part, kb, vb);
}

// Waves that share the keys of at most 32 rows, each with two buffers of its own.
template <typename T, int DP>
constexpr int few_waves() {
    return 131072 / (4 * 32 * Tile<T, DP>::kPitch) < 8 ? 131072 / (4 * 32 * Tile<T, DP>::kPitch) : 8;
}

// A block: 32 rows of one key head, or one part of their keys.  Each of its W waves
// streams every W-th tile of keys through buffers of its own, with no barrier, and the
// waves' sums are joined in LDS.  Bound by memory on long caches: the next token of 16
// sequences over up to 32768 keys, window 16384, 150 us (5.5 TB/s); on short ones by its
// chain of loads and products: one sequence, 1024 keys, 11 us.
template <typename T, int DP, bool COPY, int W>
__global__ __launch_bounds__(64 * W) void k_attention_few(const AttentionArgs a, const Plan p) {
    using Ti = Tile<T, DP>;
    constexpr int BN = 32, kBytes = BN * Ti::kPitch, kPart = DP + 4;      // floats of a row's part
    using F = Fill<T, DP, BN, 64>;
    static_assert(BN * kPart * 4 <= 4 * kBytes, "a wave's sums fit its buffers");
    constexpr int kBufs = W == 1 ? 1 : 2;                 // a lone wave has a tile or two: no second buffer
    __shared__ __align__(128) char lds_all[W][kBufs * 2 * kBytes];
    __shared__ float stats[W][2][32], totals[32];
    __shared__ int redo[32];
    const pd_attention_desc& d = a.d;
    const int lane = threadIdx.x & 63, wave = W == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    char* lds = lds_all[wave];
    const int split = blockIdx.x % p.splits, head = blockIdx.x / p.splits;   // one row tile a key head
    const int hk = head % d.heads_kv, b = head / d.heads_kv;
    const Seq seq = sequence(a, b);
    const int row = lane & 31;
    const bool real = row < p.rows;
    const int qi = real ? rows_to_query(p, row) : 0, hq = hk * p.group + (real ? row - qi * p.group : 0);
    const See see = real ? sees(d, seq, qi) : See{0, 0, 0};
    const Sight sight = sight_of(d, seq, 0, p.rows == 32 ? d.q_len - 1 : seq.n);
    const T* kb = static_cast<const T*>(a.k) + b * d.k_stride[0] + hk * d.k_stride[2];
    const T* vb = static_cast<const T*>(a.v) + b * d.v_stride[0] + hk * d.v_stride[2];

    const KeyTiles<BN> tiles(seq.n > 0 ? sees_any(d, seq, 0, seq.n - 1) : See{0, 0, 0});
    const int it0 = split * p.split_tiles + wave, it1 = min(tiles.count, split * p.split_tiles + p.split_tiles);
    F fk, fv;
    if constexpr (COPY) {
        const int units = d.head_dim * (int)sizeof(T) / 16;
        fk.plan(d.k_stride[1], units, lane);
        fv.plan(d.v_stride[1], units, lane);
    }
    auto fetch = [&](int it, char* to) {
        const int j0 = tiles.start(it);
        const T* kt = kb + (int64_t)j0 * d.k_stride[1];
        const T* vt = vb + (int64_t)j0 * d.v_stride[1];
        if constexpr (COPY) {
            if (tiles.whole(j0)) {
                fk.copy(kt, to);
                fv.copy(vt, to + kBytes);
            } else {
                auto from = [&](int r) { return tiles.inside(j0, j0 + r) - j0; };
                fk.copy_some(kt, to, lane, from);
                fv.copy_some(vt, to + kBytes, lane, from);
            }
        } else {
            auto keep = [&](int r) { return tiles.any(j0 + r); };
            F::load(kt, d.k_stride[1], d.head_dim, to, lane, keep);
            F::load(vt, d.v_stride[1], d.head_dim, to + kBytes, lane, keep);
        }
    };
    if (COPY && it0 < it1) fetch(it0, lds);
    Rows<AsIs<T, DP>, DP, 1> w;
    w.start(d);
    w.load(0, d, static_cast<const T*>(a.q) + b * d.q_stride[0] + qi * d.q_stride[1] + hq * d.q_stride[2], real && !see.none(), lane);
    const See sees_from[1] = {see.from(lane)};
    if constexpr (COPY && W == 1) {
        for (int it = it0; it < it1; ++it) {
            const int j0 = tiles.start(it);
            if (it > it0) {
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                fetch(it, lds);
            }
            wait_copies();
            __builtin_amdgcn_wave_barrier();
            w.template attend<1>(lds, lds + kBytes, j0, sees_from, !sight.all(j0, BN), lane, tiles.any.hi <= j0 + 16 && tiles.any.sk <= j0 + 16);
            __builtin_amdgcn_wave_barrier();
        }
    } else if constexpr (COPY) {
        int buf = 0;
        for (int it = it0; it < it1; it += W, buf ^= 1) {
            const int j0 = tiles.start(it);
            // the wave's reads of the other buffer are done (their values were used), so
            // the next tile may go there; then all copies but the next tile's have landed
            if (it + W < it1) {
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                fetch(it + W, lds + (buf ^ 1) * 2 * kBytes);
                asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * F::kCopies) : "memory");
            } else {
                wait_copies();
            }
            __builtin_amdgcn_wave_barrier();
            const char* at = lds + buf * 2 * kBytes;
            w.template attend<1>(at, at + kBytes, j0, sees_from, !sight.all(j0, BN), lane);
            __builtin_amdgcn_wave_barrier();
        }
    } else {
        for (int it = it0; it < it1; it += W) {
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            fetch(it, lds);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            const int j0 = tiles.start(it);
            w.template attend<1>(lds, lds + kBytes, j0, sees_from, !sight.all(j0, BN), lane);
        }
    }
    if constexpr (W == 1) {
        store_rows(a, p, w, 0, seq, b, hk, 0, split, kb, vb);
    } else {
        w.finish(0);
        if (lane < 32) {
            stats[wave][0][row] = w.top[0];
            stats[wave][1][row] = w.total[0];
            redo[row] = 0;
        }
        __syncthreads();
        // each wave's sums go to the largest reference of one that has terms
        float top = -INFINITY, total = 0.f;
#pragma unroll
        for (int i = 0; i < W; ++i)
            if (stats[i][1][row] != 0.f) top = fmaxf(top, stats[i][0][row]);
#pragma unroll
        for (int i = 0; i < W; ++i) {
            const float t = stats[i][1][row], m = stats[i][0][row];
            if (t != 0.f) total = fmaf(m == top ? 1.f : exp2_fast((m - top) * w.c2), t, total);
        }
        const float f = w.total[0] == 0.f ? 0.f : w.top[0] == top ? 1.f : exp2_fast((w.top[0] - top) * w.c2);
        float* mine = reinterpret_cast<float*>(lds) + row * kPart;
#pragma unroll
        for (int t = 0; t < w.kDT; ++t)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                f32x4 v = {w.o[0][t][4 * g], w.o[0][t][4 * g + 1], w.o[0][t][4 * g + 2], w.o[0][t][4 * g + 3]};
                v = w.total[0] == 0.f ? f32x4{} : v * f;
                *reinterpret_cast<f32x4*>(mine + 32 * t + 8 * g + 4 * (lane >> 5)) = v;
            }
        const int64_t rows_all = (int64_t)d.batch * d.heads_q * d.q_len, at = ((int64_t)b * d.heads_q + hq) * d.q_len + qi;
        const Parts to = parts(d, a.scratch, p.splits);
        if (wave == 0 && lane < 32 && real) {
            if (p.splits > 1) {
                to.stats[2 * (split * rows_all + at)] = top;
                to.stats[2 * (split * rows_all + at) + 1] = total;
            } else if (a.lse) {
                a.lse[at] = log_sum(top, fabsf(d.scale), total);
            }
        }
        if (wave == 0 && lane < 32) totals[row] = total;
        __syncthreads();
        for (int u = threadIdx.x; u < p.rows * (DP / 4); u += 64 * W) {
            const int r = u / (DP / 4), e = u % (DP / 4) * 4;
            if (e >= d.head_dim) continue;
            f32x4 v = {};
#pragma unroll
            for (int i = 0; i < W; ++i) v += *reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(lds_all[i]) + r * kPart + e);
            const int i = r / p.group, hh = hk * p.group + r % p.group;
            if (p.splits > 1) {
                const int64_t ra = ((int64_t)b * d.heads_q + hh) * d.q_len + i;
                store4(to.sums + (split * rows_all + ra) * d.head_dim + e, d.head_dim - e, v);
                continue;
            }
            const float t = totals[r];
            v = t == 0.f ? f32x4{} : v * (1.f / t);
            store4(static_cast<T*>(a.out) + b * d.out_stride[0] + i * d.out_stride[1] + hh * d.out_stride[2] + e, d.head_dim - e, v);
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (!(fabsf(v[k]) < INFINITY)) redo[r] = 1;
        }
        if (p.splits > 1) return;
        __syncthreads();
        for (int r = wave; r < p.rows; r += W) {
            if (!redo[r]) continue;
            const int i = r / p.group, hh = hk * p.group + r % p.group;
            attend_row<T>(a, static_cast<const T*>(a.q) + b * d.q_stride[0] + i * d.q_stride[1] + hh * d.q_stride[2], kb, vb,
                          sees(d, seq, i), static_cast<T*>(a.out) + b * d.out_stride[0] + i * d.out_stride[1] + hh * d.out_stride[2],
                          a.lse ? a.lse + ((int64_t)b * d.heads_q + hh) * d.q_len + i : nullptr);
        }
    }
}

// A row's parts into its result: one wave a row, lane e has values e and e + 64.
template <typename T>
__global__ __launch_bounds__(256) void k_attention_join(const AttentionArgs a, const Plan p) {
    const pd_attention_desc& d = a.d;
    const int lane = threadIdx.x & 63;
    const int64_t rows = (int64_t)d.batch * d.heads_q * d.q_len, row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= rows) return;
    const int i = (int)(row % d.q_len), hq = (int)(row / d.q_len % d.heads_q), b = (int)(row / d.q_len / d.heads_q);
    const Parts from = parts(d, a.scratch, p.splits);
    const float c2 = d.scale == 0.f ? 1.f : fabsf(d.scale) * kLog2e;
    // the largest reference of a part that has terms (a NaN total counts as one)
    float top = -INFINITY;
    for (int s = lane; s < p.splits; s += 64) {
        const float* st = from.stats + 2 * (s * rows + row);
        if (st[1] != 0.f) top = fmaxf(top, st[0]);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
    float total = 0.f, acc[2] = {0.f, 0.f};
    for (int s0 = 0; s0 < p.splits; s0 += 64) {
        // lane s: the factor of part s0 + s; then the parts' sums, eight loads at a time
        float f = 0.f;
        if (s0 + lane < p.splits) {
            const float* st = from.stats + 2 * ((s0 + lane) * rows + row);
            const float t = st[1];
            if (t != 0.f) {
                f = st[0] == top ? 1.f : exp2_fast((st[0] - top) * c2);
                total = fmaf(f, t, total);
            }
        }
        const int count = min(64, p.splits - s0);
        const uint64_t some = __ballot(f != 0.f);          // (also a NaN)
        for (int s = 0; s < count; s += 8) {
            if (!((some >> s) & 255)) continue;
            float v[8][2];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float* sums = from.sums + (min(s0 + s + k, p.splits - 1) * rows + row) * d.head_dim;
                v[k][0] = lane < d.head_dim ? sums[lane] : 0.f;
                v[k][1] = lane + 64 < d.head_dim ? sums[lane + 64] : 0.f;
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float g = __shfl(f, (s + k) & 63);
                if (!((some >> s >> k) & 1)) continue;      // a part without terms has no sums
                acc[0] = fmaf(g, v[k][0], acc[0]);
                acc[1] = fmaf(g, v[k][1], acc[1]);
            }
        }
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) total += __shfl_xor(total, o);
    T* out = static_cast<T*>(a.out) + b * d.out_stride[0] + i * d.out_stride[1] + hq * d.out_stride[2];
    float* lse = a.lse ? a.lse + row : nullptr;
    const float inv = total == 0.f ? 0.f : 1.f / total;
    acc[0] *= inv;
    acc[1] *= inv;
    if (__any(!(fabsf(acc[0]) < INFINITY) || !(fabsf(acc[1]) < INFINITY))) {
        const int hk = hq / p.group;
        attend_row<T>(a, static_cast<const T*>(a.q) + b * d.q_stride[0] + i * d.q_stride[1] + hq * d.q_stride[2],
                      static_cast<const T*>(a.k) + b * d.k_stride[0] + hk * d.k_stride[2],
                      static_cast<const T*>(a.v) + b * d.v_stride[0] + hk * d.v_stride[2], sees(d, sequence(a, b), i), out, lse);
        return;
    }
    if (lane < d.head_dim) out[lane] = (T)acc[0];
    if (lane + 64 < d.head_dim) out[lane + 64] = (T)acc[1];
    if (lse && lane == 0) *lse = log_sum(top, fabsf(d.scale), total);
}

// The most tiles of bn keys that a tile of rows can have to read.
int64_t most_tiles(const pd_attention_desc& d, int rows_per_tile, int group, int bn) {
    const int64_t all = ((int64_t)d.kv_len + bn - 1) / bn;
    if (!d.window) return all;
    const int64_t queries = (int64_t)(rows_per_tile - 1) / group + 2;
    const int64_t span = (d.causal ? 1 : 2) * (int64_t)d.window + (queries < d.q_len ? queries : d.q_len);
    const int64_t some = span / bn + 2 + ((int64_t)d.sinks + bn - 1) / bn;
    return some < all ? some : all;
}

bool few_rows(const pd_attention_desc& d) { return (int64_t)d.q_len * (d.heads_q / d.heads_kv) <= 32; }

int bn_of(const pd_attention_desc& d) { return d.dtype == PD_BF16 || d.head_dim <= 64 ? 64 : 32; }
// 32-row tiles a wave takes: two where they leave two blocks for each compute unit (a
// window of 64 latents of 576 tokens: 144 us, with one 148)
int wave_tiles_of(const pd_attention_desc& d) {
    if (d.dtype != PD_BF16 || d.head_dim > 64) return 1;
    const int64_t rows = (int64_t)d.q_len * (d.heads_q / d.heads_kv);
    return (rows + 255) / 256 * d.heads_kv * d.batch >= 512 ? 2 : 1;
}

int few_waves_of(const pd_attention_desc& d) {
    const int bytes = d.head_dim <= 32 ? 32 : d.head_dim <= 64 ? 64 : d.head_dim <= 96 ? 96 : 128;
    const int pitch = (bytes * (d.dtype == PD_BF16 ? 2 : 4) + 127) / 128 * 128, n = 131072 / (4 * 32 * pitch);
    return n < 8 ? n : 8;
}

// The fewest parts, from as many as give each of 256 compute units a block, that keep
// them busy for nine tenths of the rounds it takes, or the best of the next few.
int64_t fill_units(int64_t blocks) {
    const int64_t first = blocks < 256 ? 256 / blocks : 1;
    int64_t best = first;
    double used = 0.0;
    for (int64_t s = first; s < first + 5 && used < 0.9; ++s) {
        const int64_t n = blocks * s, rounds = (n + 255) / 256;
        const double u = (double)n / (double)(rounds * 256);
        if (u > used) best = s, used = u;
    }
    return best;
}

// How the work is cut (figures in us).
// At most 32 rows go to k_attention_few: 16 tokens over long caches 151, one over 1024
// keys 12, 100 sequences of 16 tokens in float32 13 (in blocks of 128 rows 162, 20, 32).  One
// wave up to two tiles of keys (the sequences; with four waves 54), else few_waves
// (the tokens), in parts that give each compute unit a block, of at least eight tiles a
// wave (16 tokens: 256 blocks 151, 512 163, 1024 175, 2048 178).
// More rows go in blocks of 128 (two waves' tiles: wave_tiles_of).  Where they would not
// fill the chip (two a compute unit), parts of at least four tiles (the float32 chunk
// over ragged caches: 3 parts 62, 4 56, 6 and 7 48, 11 55).
Plan plan(const pd_attention_desc& d) {
    Plan p{};
    p.group = d.heads_q / d.heads_kv;
    p.rows = d.q_len * p.group;
    p.shift = p.group & (p.group - 1) ? -1 : __builtin_ctz(p.group);
    const bool few = few_rows(d);
    p.wave_tiles = few ? 1 : wave_tiles_of(d);
    const int bm = 128 * p.wave_tiles;
    p.row_tiles = few ? 1 : (p.rows + bm - 1) / bm;
    p.units = (int64_t)p.row_tiles * d.heads_kv * d.batch;
    const int64_t tiles = most_tiles(d, few ? 32 : bm, p.group, few ? 32 : bn_of(d));
    int64_t splits;
    if (few) {
        p.waves = tiles <= 2 ? 1 : few_waves_of(d);
        const int64_t most = (tiles + 8 * p.waves - 1) / (8 * p.waves);
        splits = p.units > 0 ? fill_units(p.units) : 1;
        if (splits > most) splits = most;
    } else {
        splits = p.units >= 256 ? 1 : 512 / p.units;
        if (splits > tiles / 4) splits = tiles / 4;
    }
    if (splits < 1) splits = 1;
    p.split_tiles = (int)((tiles + splits - 1) / splits);
    p.splits = tiles ? (int)((tiles + p.split_tiles - 1) / p.split_tiles) : 1;
    return p;
}

template <typename T, int DP, bool COPY>
void attention_c(const AttentionArgs& a, hipStream_t s) {
    const Plan p = plan(a.d);
    constexpr int W = few_waves<T, DP>();
    const dim3 few((unsigned)(p.units * p.splits));
    if (few_rows(a.d) && p.waves == 1)
        hipLaunchKernelGGL((k_attention_few<T, DP, COPY, 1>), few, dim3(64), 0, s, a, p);
    else if (few_rows(a.d))
        hipLaunchKernelGGL((k_attention_few<T, DP, COPY, W>), few, dim3(64 * W), 0, s, a, p);
    else if constexpr (sizeof(T) == 4)
        hipLaunchKernelGGL((k_attention_parts<DP>), dim3((unsigned)(p.units * p.splits)), dim3(256), 0, s, a, p);
    else if (p.wave_tiles == 1)
        hipLaunchKernelGGL((k_attention<T, DP, COPY, 1>), dim3((unsigned)(p.units * p.splits)), dim3(256), 0, s, a, p);
    else if constexpr (wave_tiles<T, DP>() == 2)
        hipLaunchKernelGGL((k_attention<T, DP, COPY, 2>), dim3((unsigned)(p.units * p.splits)), dim3(256), 0, s, a, p);
    PD_HIP(hipGetLastError());
    if (p.splits == 1) return;
    const int64_t rows = (int64_t)a.d.batch * a.d.heads_q * a.d.q_len;
    hipLaunchKernelGGL((k_attention_join<T>), dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, s, a, p);
    PD_HIP(hipGetLastError());
}
template <typename T, int DP>
void attention_t(const AttentionArgs& a, hipStream_t s) {
    const pd_attention_desc& d = a.d;
    if (copies_fit(a.k, d.k_stride, d.batch, d.kv_len, d.heads_kv, d.head_dim, sizeof(T)) &&
        copies_fit(a.v, d.v_stride, d.batch, d.kv_len, d.heads_kv, d.head_dim, sizeof(T)))
        attention_c<T, DP, true>(a, s);
    else
        attention_c<T, DP, false>(a, s);
}
template <typename T>
void attention_dim(const AttentionArgs& a, hipStream_t s) {
    if (a.d.head_dim <= 32) return attention_t<T, 32>(a, s);
    if (a.d.head_dim <= 64) return attention_t<T, 64>(a, s);
    if (a.d.head_dim <= 96) return attention_t<T, 96>(a, s);
    attention_t<T, 128>(a, s);
}

}  // namespace

int64_t attention_scratch_bytes(const pd_attention_desc& d) {
    if (d.batch == 0 || d.q_len == 0) return 0;
    const Plan p = plan(d);
    if (p.splits == 1) return 0;
    const int64_t rows = (int64_t)d.batch * d.heads_q * d.q_len * p.splits;
    return (((rows * 2 + 3) & ~(int64_t)3) + rows * d.head_dim) * (int64_t)sizeof(float);
}

void launch_attention(const AttentionArgs& a, hipStream_t s) {
    a.d.dtype == PD_F32 ? attention_dim<float>(a, s) : attention_dim<bf16>(a, s);
}

}  // namespace pd
