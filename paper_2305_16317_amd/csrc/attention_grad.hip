// Attention with a sliding window and sinks, backward.
//
//   p_ij = e^(scale q_i k_j - lse_i),  dp_ij = do_i v_j,  delta_i = do_i o_i,
//   ds_ij = p_ij (dp_ij - delta_i):
//   dq_i = scale sum_j ds_ij k_j,  dk_j = scale sum_i ds_ij q_i,  dv_j = sum_i p_ij do_i
//
// Two kernels, each summing into its own registers: dq over a block of queries
// (which also leaves delta for the other), dk and dv over a block of keys and all
// query heads that read them.  The scores are formed twice (14 D operations a pair
// and head in place of 10), and in exchange there is no atomic and no order that
// varies from run to run.
#include "attention_tile.h"

namespace pd {
namespace {

using namespace attn;

constexpr int kBN = 64;          // keys a tile of the dq kernel
constexpr int kBR = 32;          // rows a tile of the dk, dv kernel

// p = e^(scale s - lse): one fused multiply-add in base 2 while |lse| is under 1024;
// beyond, where rounding lse log2 e would show, from the difference itself, which
// is not above 0 (a score of 10^8 has a unit in the last place of 8).
constexpr float kLarge = 1024.f;
__device__ inline float probability(bool large, float s, float c2, float lse2, float scale, float lse) {
    if (!large) return exp2_fast(fmaf(s, c2, -lse2));
    const float x = (s * scale - lse) * kLog2e;
    return exp2_fast(x > 0.f ? 0.f : x);
}

// What the backward kernels read of one (sequence, key head).
template <typename T>
struct Views {
    const T *k, *v;              // of the key head
    const T *q, *out, *dout;     // of the group's first query head
    const float *lse, *delta;    // [group][q_len]
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
                    a.lse + at, a.scratch + at, group};
}

// p and ds of one pair, from memory
template <typename T>
__device__ inline void pair_grad(const AttentionArgs& a, const Views<T>& w, int i, int g, int j, float* p, float* ds) {
    const pd_attention_desc& d = a.d;
    const T* q = w.q + i * d.q_stride[1] + g * d.q_stride[2];
    const T* go = w.dout + i * d.dout_stride[1] + g * d.dout_stride[2];
    const T* k = w.k + j * d.k_stride[1];
    const T* v = w.v + j * d.v_stride[1];
    float s = 0.f, dp = 0.f;
    for (int e = 0; e < d.head_dim; ++e) {
        s = fmaf((float)q[e], (float)k[e], s);
        dp = fmaf((float)go[e], (float)v[e], dp);
    }
    const int64_t at = (int64_t)g * d.q_len + i;
    *p = probability(true, s, 0.f, 0.f, d.scale, w.lse[at]);
    *ds = *p * (dp - w.delta[at]);
}

// A row of dq from its visible keys alone (see attend_row in attention.hip).
template <typename T>
__device__ void dq_row(const AttentionArgs& a, const Views<T>& w, int i, int g, const See see, T* dq) {
    const int lane = threadIdx.x & 63, D = a.d.head_dim;
    float acc[2] = {0.f, 0.f};
    for (int part = 0; part < 2; ++part) {
        const int j0 = part == 0 ? 0 : max(see.lo, see.sk), j1 = part == 0 ? see.sk : see.hi;
        for (int jb = j0; jb < j1; jb += 64) {
            const int count = min(64, j1 - jb);
            float p = 0.f, ds = 0.f;
            if (lane < count) pair_grad(a, w, i, g, jb + lane, &p, &ds);
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
        if (seen) pair_grad(a, w, i, g, j, &p, &ds);
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

template <typename T, int DP>
__global__ __launch_bounds__(256) void k_attention_dq(const AttentionArgs a) {
    using Ti = Tile<T, DP>;
    constexpr int kSteps = DP / 16, kDT = DP / 32;
    __shared__ __align__(16) char lds_k[kBN * Ti::kPitch];
    __shared__ __align__(16) char lds_v[kBN * Ti::kPitch];
    const pd_attention_desc& d = a.d;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = lane >> 5;
    const int b = blockIdx.z, hk = blockIdx.y;
    const Seq seq = sequence(a, b);
    const Views<T> w = views<T>(a, b, hk);
    const int rows_all = d.q_len * w.group;
    const int row0 = blockIdx.x * 128 + wave * 32, row = row0 + (lane & 31);
    const bool real = row < rows_all;
    const int qi = real ? row / w.group : 0, g = row % w.group;
    const See see = real ? sees(d, seq, qi) : See{0, 0, 0};

    Frag<T> qf[kSteps], gf[kSteps];
    float delta = 0.f;
#pragma unroll
    for (int c = 0; c < kSteps; ++c) {
        const int e = 16 * c + 8 * h;
        qf[c] = Frag<T>{};
        gf[c] = Frag<T>{};
        if (see.none()) continue;
        qf[c] = load8(w.q + qi * d.q_stride[1] + g * d.q_stride[2] + e, d.head_dim - e);
        gf[c] = load8(w.dout + qi * d.dout_stride[1] + g * d.dout_stride[2] + e, d.head_dim - e);
        const f32x8 x = widen(gf[c]), y = widen(load8(w.out + qi * d.out_stride[1] + g * d.out_stride[2] + e, d.head_dim - e));
#pragma unroll
        for (int f = 0; f < 8; ++f) delta = fmaf(x[f], y[f], delta);
    }
    delta += __shfl_xor(delta, 32);
    const int64_t at = (int64_t)g * d.q_len + qi;
    if (real && h == 0) const_cast<float*>(w.delta)[at] = delta;
    const float c2 = d.scale * kLog2e;
    const float lse = see.none() ? 0.f : w.lse[at], lse2 = lse * kLog2e;
    const bool large = __any(!(fabsf(lse) < kLarge));

    const int i0 = blockIdx.x * 128 / w.group, i1 = min((blockIdx.x * 128 + 127) / w.group, seq.n - 1);
    See any{0, 0, 0};
    if (i0 <= i1) any = sees_any(d, seq, i0, i1);
    const int sink_tiles = (any.sk + kBN - 1) / kBN;
    const int first = max(any.lo / kBN, sink_tiles), end = max((any.hi + kBN - 1) / kBN, first);
    const int tiles = sink_tiles + end - first;

    f32x16 o[kDT];
#pragma unroll
    for (int t = 0; t < kDT; ++t) o[t] = f32x16{};
    for (int it = 0; it < tiles; ++it) {
        const int j0 = (it < sink_tiles ? it : first + it - sink_tiles) * kBN;
        __syncthreads();
        for (int u = threadIdx.x; u < kBN * (DP / 8); u += 256) {
            const int r = u / (DP / 8), c = u % (DP / 8), j = j0 + r;
            Frag<T> kv = {}, vv = {};
            if (any(j)) {
                kv = load8(w.k + (int64_t)j * d.k_stride[1] + 8 * c, d.head_dim - 8 * c);
                vv = load8(w.v + (int64_t)j * d.v_stride[1] + 8 * c, d.head_dim - 8 * c);
            }
            Ti::put(lds_k, r, c, kv);
            Ti::put(lds_v, r, c, vv);
        }
        __syncthreads();
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
            f32x16 s = {}, dp = {};
#pragma unroll
            for (int c = 0; c < kSteps; ++c) {
                s = mma(Ti::rows(lds_k, 32 * kt, c, lane), qf[c], s);
                dp = mma(Ti::rows(lds_v, 32 * kt, c, lane), gf[c], dp);
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const float p = probability(large, s[r], c2, lse2, d.scale, lse);
                s[r] = see(j0 + 32 * kt + tile_row(lane, r)) ? p * (dp[r] - delta) : 0.f;
            }
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const Frag<T> ds = as_frag<T>(s, c);
#pragma unroll
                for (int t = 0; t < kDT; ++t) o[t] = mma(Ti::cols(lds_k, 32 * kt + 16 * c, t, lane), ds, o[t]);
            }
        }
    }

    T* dq = static_cast<T*>(a.dq) + b * d.dq_stride[0] + hk * w.group * d.dq_stride[2];
    bool odd = false;
#pragma unroll
    for (int t = 0; t < kDT; ++t) {
        o[t] = see.none() ? f32x16{} : o[t] * d.scale;
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

template <typename T, int DP>
__global__ __launch_bounds__(256) void k_attention_dkv(const AttentionArgs a) {
    using Ti = Tile<T, DP>;
    constexpr int kSteps = DP / 16, kDT = DP / 32;
    __shared__ __align__(16) char lds_q[kBR * Ti::kPitch];
    __shared__ __align__(16) char lds_g[kBR * Ti::kPitch];
    __shared__ __align__(16) float lds_lse[kBR], lds_delta[kBR];
    __shared__ __align__(16) See lds_see[kBR];
    __shared__ bool lds_large;
    const pd_attention_desc& d = a.d;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = lane >> 5;
    const int b = blockIdx.z, hk = blockIdx.y;
    const Seq seq = sequence(a, b);
    const Views<T> w = views<T>(a, b, hk);
    const int key0 = blockIdx.x * 128, wkey0 = key0 + wave * 32, key = wkey0 + (lane & 31);
    const bool live = key < seq.m;

    Frag<T> kf[kSteps], vf[kSteps];
#pragma unroll
    for (int c = 0; c < kSteps; ++c) {
        const int e = 16 * c + 8 * h;
        kf[c] = Frag<T>{};
        vf[c] = Frag<T>{};
        if (!live) continue;
        kf[c] = load8(w.k + (int64_t)key * d.k_stride[1] + e, d.head_dim - e);
        vf[c] = load8(w.v + (int64_t)key * d.v_stride[1] + e, d.head_dim - e);
    }
    // the queries that may see a key of the block: first .. last
    const int k1 = min(key0 + 127, seq.m - 1), off = seq.m - seq.n;      // t = off + i
    int first = 0, last = key0 < seq.m ? seq.n - 1 : -1;
    if (d.causal) first = max(first, key0 - off);
    if (d.window && key0 >= d.sinks) {
        last = min(last, k1 + d.window - 1 - off);
        if (!d.causal) first = max(first, key0 - d.window + 1 - off);
    }
    const float c2 = d.scale * kLog2e;
    f32x16 dk[kDT], dv[kDT];
#pragma unroll
    for (int t = 0; t < kDT; ++t) dk[t] = dv[t] = f32x16{};
    const int r_end = (last + 1) * w.group;
    for (int r0 = first * w.group; r0 < r_end; r0 += kBR) {
        __syncthreads();
        for (int u = threadIdx.x; u < kBR * (DP / 8); u += 256) {
            const int r = u / (DP / 8), c = u % (DP / 8), row = r0 + r;
            Frag<T> qv = {}, gv = {};
            if (row < r_end) {
                const int i = row / w.group, g = row % w.group;
                if (!sees(d, seq, i).none()) {
                    qv = load8(w.q + i * d.q_stride[1] + g * d.q_stride[2] + 8 * c, d.head_dim - 8 * c);
                    gv = load8(w.dout + i * d.dout_stride[1] + g * d.dout_stride[2] + 8 * c, d.head_dim - 8 * c);
                }
            }
            Ti::put(lds_q, r, c, qv);
            Ti::put(lds_g, r, c, gv);
        }
        if (threadIdx.x < kBR) {
            const int row = r0 + threadIdx.x;
            See see{0, 0, 0};
            float lse = 0.f, delta = 0.f;
            if (row < r_end) {
                const int i = row / w.group, g = row % w.group;
                see = sees(d, seq, i);
                if (!see.none()) {
                    lse = w.lse[(int64_t)g * d.q_len + i];
                    delta = w.delta[(int64_t)g * d.q_len + i];
                }
            }
            lds_see[threadIdx.x] = see;
            lds_lse[threadIdx.x] = lse;
            lds_delta[threadIdx.x] = delta;
            const uint64_t far = __ballot(!(fabsf(lse) < kLarge));
            if (threadIdx.x == 0) lds_large = far != 0;
        }
        __syncthreads();
        const bool large = lds_large;
        f32x16 s = {}, dp = {};
#pragma unroll
        for (int c = 0; c < kSteps; ++c) {
            s = mma(Ti::rows(lds_q, 0, c, lane), kf[c], s);
            dp = mma(Ti::rows(lds_g, 0, c, lane), vf[c], dp);
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int row = tile_row(lane, r);
            const bool seen = live && lds_see[row](key);
            const float lse = lds_lse[row];
            const float p = probability(large, s[r], c2, lse * kLog2e, d.scale, lse);
            s[r] = seen ? p : 0.f;
            dp[r] = seen ? p * (dp[r] - lds_delta[row]) : 0.f;
        }
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const Frag<T> p = as_frag<T>(s, c), ds = as_frag<T>(dp, c);
#pragma unroll
            for (int t = 0; t < kDT; ++t) {
                dv[t] = mma(Ti::cols(lds_g, 16 * c, t, lane), p, dv[t]);
                dk[t] = mma(Ti::cols(lds_q, 16 * c, t, lane), ds, dk[t]);
            }
        }
    }

    bool odd = false;
#pragma unroll
    for (int t = 0; t < kDT; ++t) {
        dk[t] *= d.scale;
#pragma unroll
        for (int r = 0; r < 16; ++r) odd = odd || !(fabsf(dk[t][r]) < INFINITY) || !(fabsf(dv[t][r]) < INFINITY);
    }
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

template <typename T, int DP>
void attention_grad_t(const AttentionArgs& a, hipStream_t s) {
    const int64_t rows = (int64_t)a.d.q_len * (a.d.heads_q / a.d.heads_kv);
    if (rows) {
        hipLaunchKernelGGL((k_attention_dq<T, DP>), dim3((unsigned)((rows + 127) / 128), a.d.heads_kv, a.d.batch), dim3(256),
                           0, s, a);
        PD_HIP(hipGetLastError());
    }
    if (!a.d.kv_len) return;
    hipLaunchKernelGGL((k_attention_dkv<T, DP>), dim3((unsigned)(((int64_t)a.d.kv_len + 127) / 128), a.d.heads_kv, a.d.batch),
                       dim3(256), 0, s, a);
    PD_HIP(hipGetLastError());
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
    return (int64_t)d.batch * d.heads_q * d.q_len * (int64_t)sizeof(float);      // delta
}

void launch_attention_grad(const AttentionArgs& a, hipStream_t s) {
    a.d.dtype == PD_F32 ? attention_grad_dim<float>(a, s) : attention_grad_dim<bf16>(a, s);
}

}  // namespace pd
