// Attention with a sliding window and sinks, forward.
//
//   x_ij = scale q_i k_j over the keys that query i sees,  o_i = sum_j e^(x_ij - m_i) v_j / l_i
//
// One pass over the keys with a running maximum m and sum l (in base 2: p = 2^(s c
// - m c), c = scale log2 e, one fused multiply-add and one exponential a score).
// (The product m c is rounded: a shift of all of a row's terms, without effect
// while it is small.  Where |m c| passes 1024 the difference (s - m) c is formed
// instead, exact for the row's largest scores of any size.)
// A block holds 128 rows, 32 a wave; a row is a query of one of the heads that
// share a key head, so keys and values are read once for all of them.
#include "attention_tile.h"

namespace pd {
namespace {

using namespace attn;

constexpr int kBN = 64;          // keys a tile
constexpr float kLarge = 1024.f;


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
    const float inv = 1.f / total;
    if (lane < D) out[lane] = (T)(acc[0] * inv);
    if (lane + 64 < D) out[lane + 64] = (T)(acc[1] * inv);
    if (lse && lane == 0) *lse = log_sum(top, 1.f, total);
}

template <typename T, int DP>
__global__ __launch_bounds__(256) void k_attention(const AttentionArgs a) {
    using Ti = Tile<T, DP>;
    constexpr int kSteps = DP / 16, kDT = DP / 32;
    __shared__ __align__(16) char lds_k[kBN * Ti::kPitch];
    __shared__ __align__(16) char lds_v[kBN * Ti::kPitch];
    const pd_attention_desc& d = a.d;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = lane >> 5;
    const int group = d.heads_q / d.heads_kv;
    const int b = blockIdx.z, hk = blockIdx.y;
    const Seq seq = sequence(a, b);
    const int rows_all = d.q_len * group;
    const int row0 = blockIdx.x * 128 + wave * 32, row = row0 + (lane & 31);
    const bool real = row < rows_all;
    const int qi = real ? row / group : 0, hq = hk * group + row % group;
    const See see = real ? sees(d, seq, qi) : See{0, 0, 0};

    const T* kb = static_cast<const T*>(a.k) + b * d.k_stride[0] + hk * d.k_stride[2];
    const T* vb = static_cast<const T*>(a.v) + b * d.v_stride[0] + hk * d.v_stride[2];
    const T* qp = static_cast<const T*>(a.q) + b * d.q_stride[0] + qi * d.q_stride[1] + hq * d.q_stride[2];

    Frag<T> qf[kSteps];
#pragma unroll
    for (int c = 0; c < kSteps; ++c) {
        const int e = 16 * c + 8 * h;
        qf[c] = Frag<T>{};
        if (real && !see.none() && d.scale != 0.f) qf[c] = load8(qp + e, d.head_dim - e);
        if (d.scale < 0.f) qf[c] = -qf[c];
    }
    // the running maximum is one of unscaled scores: c2 > 0 (a scale of 0: zero queries)
    const float c2 = d.scale == 0.f ? 1.f : fabsf(d.scale) * kLog2e;

    // the block's queries, its keys, and the tiles that hold them
    const int i0 = blockIdx.x * 128 / group, i1 = min((blockIdx.x * 128 + 127) / group, seq.n - 1);
    See any{0, 0, 0};
    if (i0 <= i1) any = sees_any(d, seq, i0, i1);
    const int sink_tiles = (any.sk + kBN - 1) / kBN;
    const int first = max(any.lo / kBN, sink_tiles), end = max((any.hi + kBN - 1) / kBN, first);
    const int tiles = sink_tiles + end - first;

    f32x16 o[kDT];
#pragma unroll
    for (int t = 0; t < kDT; ++t) o[t] = f32x16{};
    float top = -INFINITY, total = 0.f;

    for (int it = 0; it < tiles; ++it) {
        const int j0 = (it < sink_tiles ? it : first + it - sink_tiles) * kBN;
        __syncthreads();
        for (int u = threadIdx.x; u < kBN * (DP / 8); u += 256) {
            const int r = u / (DP / 8), c = u % (DP / 8), j = j0 + r;
            Frag<T> kv = {}, vv = {};
            if (any(j)) {
                kv = load8(kb + (int64_t)j * d.k_stride[1] + 8 * c, d.head_dim - 8 * c);
                vv = load8(vb + (int64_t)j * d.v_stride[1] + 8 * c, d.head_dim - 8 * c);
            }
            Ti::put(lds_k, r, c, kv);
            Ti::put(lds_v, r, c, vv);
        }
        __syncthreads();
        f32x16 s[2];
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
            s[kt] = f32x16{};
#pragma unroll
            for (int c = 0; c < kSteps; ++c) s[kt] = mma(Ti::rows(lds_k, 32 * kt, c, lane), qf[c], s[kt]);
        }
        float m = top;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                if (!see(j0 + 32 * kt + tile_row(lane, r))) s[kt][r] = -INFINITY;
                m = fmaxf(m, s[kt][r]);
            }
        m = fmaxf(m, __shfl_xor(m, 32));
        const float mc = m == -INFINITY ? 0.f : m * c2;
        const bool large = __any(!(fabsf(mc) < kLarge));
        float keep = exp2_fast(top * c2 - mc);
        if (large) keep = top == -INFINITY ? 0.f : exp2_fast((top - m) * c2);
        top = m;
        float sum = 0.f;
        if (large) {
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const float x = s[kt][r];
                    s[kt][r] = m == -INFINITY || x == -INFINITY ? 0.f : exp2_fast((x - m) * c2);
                    sum += s[kt][r];
                }
        } else {
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[kt][r] = exp2_fast(fmaf(s[kt][r], c2, -mc));
                sum += s[kt][r];
            }
        }
        total = total * keep + sum + __shfl_xor(sum, 32);
#pragma unroll
        for (int t = 0; t < kDT; ++t) o[t] *= keep;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const Frag<T> p = as_frag<T>(s[kt], c);
#pragma unroll
                for (int t = 0; t < kDT; ++t) o[t] = mma(Ti::cols(lds_v, 32 * kt + 16 * c, t, lane), p, o[t]);
            }
    }

    float* lse = a.lse ? a.lse + ((int64_t)b * d.heads_q + hq) * d.q_len + qi : nullptr;
    T* out = static_cast<T*>(a.out) + b * d.out_stride[0] + qi * d.out_stride[1] + hq * d.out_stride[2];
    const float inv = total == 0.f ? 0.f : 1.f / total;
    bool odd = false;
#pragma unroll
    for (int t = 0; t < kDT; ++t) {
        o[t] = total == 0.f ? f32x16{} : o[t] * inv;
#pragma unroll
        for (int r = 0; r < 16; ++r) odd = odd || !(fabsf(o[t][r]) < INFINITY);
    }
    odd = odd && real;
    const uint64_t both = __ballot(odd);
    uint32_t again = (uint32_t)both | (uint32_t)(both >> 32);
    if (real && !((again >> (lane & 31)) & 1)) {
#pragma unroll
        for (int t = 0; t < kDT; ++t)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int e = 32 * t + 8 * g + 4 * h;
                store4(out + e, d.head_dim - e, f32x4{o[t][4 * g], o[t][4 * g + 1], o[t][4 * g + 2], o[t][4 * g + 3]});
            }
        if (lse && h == 0) *lse = log_sum(top, fabsf(d.scale), total);
    }
    while (again) {
        const int w = __ffs(again) - 1, rr = row0 + w;
        again &= again - 1;
        const int i = rr / group, hh = hk * group + rr % group;
        attend_row<T>(a, static_cast<const T*>(a.q) + b * d.q_stride[0] + i * d.q_stride[1] + hh * d.q_stride[2], kb, vb,
                      sees(d, seq, i), static_cast<T*>(a.out) + b * d.out_stride[0] + i * d.out_stride[1] + hh * d.out_stride[2],
                      a.lse ? a.lse + ((int64_t)b * d.heads_q + hh) * d.q_len + i : nullptr);
    }
}

template <typename T, int DP>
void attention_t(const AttentionArgs& a, hipStream_t s) {
    const int group = a.d.heads_q / a.d.heads_kv;
    const int64_t rows = (int64_t)a.d.q_len * group;
    hipLaunchKernelGGL((k_attention<T, DP>), dim3((unsigned)((rows + 127) / 128), a.d.heads_kv, a.d.batch), dim3(256), 0, s, a);
    PD_HIP(hipGetLastError());
}
template <typename T>
void attention_dim(const AttentionArgs& a, hipStream_t s) {
    if (a.d.head_dim <= 32) return attention_t<T, 32>(a, s);
    if (a.d.head_dim <= 64) return attention_t<T, 64>(a, s);
    if (a.d.head_dim <= 96) return attention_t<T, 96>(a, s);
    attention_t<T, 128>(a, s);
}

}  // namespace

int64_t attention_scratch_bytes(const pd_attention_desc&) { return 0; }

void launch_attention(const AttentionArgs& a, hipStream_t s) {
    a.d.dtype == PD_F32 ? attention_dim<float>(a, s) : attention_dim<bf16>(a, s);
}

}  // namespace pd
