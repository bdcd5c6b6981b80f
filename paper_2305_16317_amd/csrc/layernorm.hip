// Layer norm with the residual's addition and a weight and bias for each run of rows
// (a sequence's modulation), forward and backward.
//
//   s = x + r,  mu = mean s,  rstd = (mean (s - mu)^2 + eps)^-1/2,  n = (s - mu) rstd
//   y = n w_g + b_g,  g = row / span
//   a = dy w_g:  dx = dsum + rstd (a - mean a - n mean(a n)),
//   dw_g = sum over the rows of g of dy n,  db_g = the same of dy
//
// Bound by memory: 4 values move per element each way.  A row stays in registers from
// its one read to its writes, eight values a lane and step, so the squares are summed
// around the mean itself and an offset common to the row costs no digits.  Rows up to
// 2048 values belong to one wave, longer ones to a block of 256 or 1024 lanes.  Backward a
// lane keeps its columns over many rows, so that dw and db are summed in registers.
//
// Measured: 36864 x 1024 bfloat16 in 64 runs 49 us (6.1 TB/s; a large copy reaches 5.0, this
// fits the last cache), backward 70 us, of which dx alone 56 (5.4 TB/s); 12432 x 1001 in 16 runs
// backward 33 us (3.1 TB/s: rows that begin at no multiple of 16 bytes; 1024 values 27).
#include "ops.h"

namespace pd {
namespace {

// Sums of two values over the TPR lanes of a row; `slot` holds two values a wave.
template <int TPR>
__device__ inline void row_sums(float& u, float& v, float* slot) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        u += __shfl_xor(u, o);
        v += __shfl_xor(v, o);
    }
    if constexpr (TPR > 64) {
        __syncthreads();                     // the last use of slot is over
        if ((threadIdx.x & 63) == 0) {
            slot[2 * (threadIdx.x >> 6)] = u;
            slot[2 * (threadIdx.x >> 6) + 1] = v;
        }
        __syncthreads();
        u = slot[0], v = slot[1];
#pragma unroll
        for (int w = 1; w < TPR / 64; ++w) {
            u += slot[2 * w];
            v += slot[2 * w + 1];
        }
    }
}
template <int TPR>
__device__ inline float row_sum(float v, float* slot) {
    float none = 0.f;
    row_sums<TPR>(v, none, slot);
    return v;
}

// ------------------------------------------------------------------ rows of any width
// Eight values from column c on, of a row of `width`.  Every lane reads eight of the row's,
// those past its end its last eight, so that no read waits for a test; `settle` then brings
// them down by how much later they begin and puts zeros behind (so a row of an odd width
// has one read a lane as any other: a read a value took 33 us where this takes 25).
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x8 __attribute__((ext_vector_type(8)));
// (TINY: rows of fewer than eight values.)
template <bool TINY, typename T>
__device__ __forceinline__ typename Vec8<T>::type eight_of(const T* row, int c, int width) {
    if constexpr (TINY) return load8(row + c, width - c);
    else return *reinterpret_cast<const typename Vec8<T>::unaligned*>(row + (c < width - 8 ? c : width - 8));
}
__device__ __forceinline__ bf16x8 settle(bf16x8 v, int c, int width) {
    const int k = c - (width - 8);                       // values that are not this lane's
    u32x4 w = __builtin_bit_cast(u32x4, v);
    if (k > 0) {
        if (k & 4) w = u32x4{w[2], w[3], 0, 0};
        if (k & 2) w = u32x4{w[1], w[2], w[3], 0};
        if (k & 1) w = u32x4{w[0] >> 16 | w[1] << 16, w[1] >> 16 | w[2] << 16, w[2] >> 16 | w[3] << 16, w[3] >> 16};
        if (k > 7) w = u32x4{};
    }
    return __builtin_bit_cast(bf16x8, w);
}
__device__ __forceinline__ f32x8 settle(f32x8 v, int c, int width) {
    const int k = c - (width - 8);
    if (k > 0) {
        if (k & 4) v = f32x8{v[4], v[5], v[6], v[7], 0.f, 0.f, 0.f, 0.f};
        if (k & 2) v = f32x8{v[2], v[3], v[4], v[5], v[6], v[7], 0.f, 0.f};
        if (k & 1) v = f32x8{v[1], v[2], v[3], v[4], v[5], v[6], v[7], 0.f};
        if (k > 7) v = f32x8{};
    }
    return v;
}
// Stores the first n of eight: in runs of four, two and one.
template <typename T>
__device__ __forceinline__ void store_first(T* p, int n, typename Vec8<T>::type v) {
    if (n >= 8) {
        *reinterpret_cast<typename Vec8<T>::unaligned*>(p) = v;
        return;
    }
    typedef T four __attribute__((ext_vector_type(4), aligned(sizeof(T))));
    typedef T two __attribute__((ext_vector_type(2), aligned(sizeof(T))));
    if (n <= 0) return;
    if (n & 4) {
        *reinterpret_cast<four*>(p) = four{v[0], v[1], v[2], v[3]};
        v[0] = v[4], v[1] = v[5], v[2] = v[6];
        p += 4;
    }
    if (n & 2) {
        *reinterpret_cast<two*>(p) = two{v[0], v[1]};
        v[0] = v[2];
        p += 2;
    }
    if (n & 1) *p = v[0];
}

// 1 / sqrt(v), within a little more than half a unit of the last place: the rounded root's quotient,
// and a Newton step from its exact residual (0 and infinity, whose residual is NaN, as they are).
__device__ __forceinline__ float one_over_sqrt(float v) {
    const float r = 1.f / sqrtf(v), t = v * r;
    const float residual = fmaf(-t, r, 1.f) - fmaf(v, r, -t) * r, better = fmaf(0.5f * r, residual, r);
    return better == better ? better : r;
}

// TPR lanes a row, NV steps of eight values a lane.
template <typename T, int TPR, int NV, bool TINY>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void k_layernorm(const LayerNormArgs a) {
    constexpr int kRows = TPR < 256 ? 256 / TPR : 1;      // rows a block
    __shared__ float slot[32];
    const int lane = threadIdx.x % TPR;
    const int64_t row = (int64_t)blockIdx.x * kRows + (kRows > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / TPR) : 0);   // (a wave's)
    if (row >= a.d.rows) return;             // whole waves; with TPR > 64 there is one row a block
    const int width = (int)a.d.width;
    const T* x = static_cast<const T*>(a.x) + row * a.d.x_stride;
    const T* r = a.residual ? static_cast<const T*>(a.residual) + row * a.d.residual_stride : nullptr;
    f32x8 v[NV];
    float sum = 0.f;
    {
        typename Vec8<T>::type vx[NV], vr[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) vx[i] = eight_of<TINY>(x, (i * TPR + lane) * 8, width);
        if (r)
#pragma unroll
            for (int i = 0; i < NV; ++i) vr[i] = eight_of<TINY>(r, (i * TPR + lane) * 8, width);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const bool whole = TINY || (i + 1) * TPR * 8 <= width;  // (uniform)
            const int c = (i * TPR + lane) * 8;
            v[i] = widen(whole ? vx[i] : settle(vx[i], c, width));
            if (r) v[i] += widen(whole ? vr[i] : settle(vr[i], c, width));
        }
    }
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += v[i][e];
    const float mean = row_sum<TPR>(sum, slot) / (float)width;
    if (a.sum) {                             // (all of the row has been read: sum may lie over x or residual)
        T* h = static_cast<T*>(a.sum) + row * a.d.sum_stride;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * TPR + lane) * 8;
            store_first(h + c, width - c, narrow<T>(v[i]));
        }
    }
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int n = width - (i * TPR + lane) * 8;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            v[i][e] = e < n ? v[i][e] - mean : 0.f;
            ss = fmaf(v[i][e], v[i][e], ss);
        }
    }
    const float rstd = one_over_sqrt(row_sum<TPR>(ss, slot) / (float)width + a.d.eps);
    if (lane == 0) {
        if (a.mean) a.mean[row] = mean;
        if (a.rstd) a.rstd[row] = rstd;
    }
    const int64_t g = (uint32_t)(a.first + row) / (uint32_t)a.d.span;
    const float* w = a.weight ? a.weight + g * a.d.weight_stride : nullptr;
    const float* b = a.bias ? a.bias + g * a.d.bias_stride : nullptr;
    T* y = static_cast<T*>(a.y) + row * a.d.y_stride;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * TPR + lane) * 8;
        const bool whole = TINY || (i + 1) * TPR * 8 <= width;
        f32x8 o = v[i] * rstd;
        if (w) {
            const f32x8 q = eight_of<TINY>(w, c, width);
            o = o * (whole ? q : settle(q, c, width));
        }
        if (b) {
            const f32x8 q = eight_of<TINY>(b, c, width);
            o = o + (whole ? q : settle(q, c, width));
        }
        store_first(y + c, width - c, narrow<T>(o));
    }
}

// Backward.  Item i of the grid's loop is part i % parts of run i / parts: its rows are
// every parts-th of the run.  A lane keeps its columns over all of them, so dw and db are
// summed in registers, then over the block's rows in LDS, and over the parts by
// k_layernorm_join: a fixed order.  SUMS false:
// dx alone.
template <typename T, int TPR, int NV, bool TINY, bool SUMS, int BLOCKS>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR, BLOCKS) void k_layernorm_grad(const LayerNormGradArgs a) {
    constexpr int kRows = TPR < 256 ? 256 / TPR : 1;
    constexpr bool KEEP = NV == 1 || (TPR < 1024 && NV * sizeof(T) < 16);   // the row stays in registers (else it is read again, from the cache)
    __shared__ float slot[32];
    __shared__ float part[SUMS && kRows > 1 ? (kRows - 1) * TPR * NV * 8 : 1];
    // (sub is a wave's: its rows' addresses and statistics stay in scalar registers)
    const int lane = threadIdx.x % TPR, sub = kRows > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / TPR) : 0;
    const int width = (int)a.d.width;
    for (int64_t item = blockIdx.x; item < (int64_t)a.groups * a.parts; item += gridDim.x) {
        const int64_t g = item / a.parts, first = g * a.d.span;
        const float* weight = a.weight ? a.weight + g * a.d.weight_stride : nullptr;
        const auto read = [&](const T* p, int i) { return eight_of<TINY>(p, (i * TPR + lane) * 8, width); };
        const auto wide = [&](typename Vec8<T>::type v, int i) {
            return widen(TINY || (i + 1) * TPR * 8 <= width ? v : settle(v, (i * TPR + lane) * 8, width));
        };
        const auto weights = [&](int i) {
            if (!weight) return f32x8{1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
            const int c = (i * TPR + lane) * 8;
            const f32x8 w = eight_of<TINY>(weight, c, width);
            return TINY || (i + 1) * TPR * 8 <= width ? w : settle(w, c, width);
        };
        f32x8 dw[SUMS ? NV : 1], db[SUMS ? NV : 1];
#pragma unroll
        for (int i = 0; i < (SUMS ? NV : 1); ++i) dw[i] = db[i] = f32x8{};
        // a row as it is read; the next one's reads begin before this one's sums
        struct Row {
            typename Vec8<T>::type dy[KEEP ? NV : 1], h[KEEP ? NV : 1], ds[KEEP ? NV : 1];
            float rstd, mean;
        } next;
        const auto fetch = [&](int64_t row) {
            next.rstd = a.rstd[row], next.mean = a.mean[row];
            if constexpr (KEEP) {
                const T* dy = static_cast<const T*>(a.dy) + row * a.d.y_stride;
                const T* h = static_cast<const T*>(a.sum) + row * a.d.sum_stride;
#pragma unroll
                for (int i = 0; i < NV; ++i) next.dy[i] = read(dy, i);
#pragma unroll
                for (int i = 0; i < NV; ++i) next.h[i] = read(h, i);
                if (a.dsum) {
                    const T* ds = static_cast<const T*>(a.dsum) + row * a.d.residual_stride;
#pragma unroll
                    for (int i = 0; i < NV; ++i) next.ds[i] = read(ds, i);
                }
            }
        };
        const int64_t begin = (item - g * a.parts) * kRows + sub, step = (int64_t)a.parts * kRows;
        if (begin < a.d.span) fetch(first + begin);
        for (int64_t at = begin; at < a.d.span; at += step) {
            const int64_t row = first + at;
            const T* dy = static_cast<const T*>(a.dy) + row * a.d.y_stride;
            const T* h = static_cast<const T*>(a.sum) + row * a.d.sum_stride;
            const T* ds = a.dsum ? static_cast<const T*>(a.dsum) + row * a.d.residual_stride : nullptr;
            T* dx = static_cast<T*>(a.dx) + row * a.d.x_stride;
            const Row now = next;
            if (at + step < a.d.span) fetch(row + step);
            const float rstd = now.rstd, mean = now.mean;
            float dot = 0.f, sum = 0.f;
            // (past the row's end dy is 0, and what it meets a number wherever the row's values are)
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const f32x8 g = wide(KEEP ? now.dy[KEEP ? i : 0] : read(dy, i), i), w = weights(i);
                const f32x8 nn = (wide(KEEP ? now.h[KEEP ? i : 0] : read(h, i), i) - mean) * rstd;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    if (SUMS) {
                        dw[SUMS ? i : 0][e] = fmaf(g[e], nn[e], dw[SUMS ? i : 0][e]);
                        db[SUMS ? i : 0][e] += g[e];
                    }
                    sum = fmaf(g[e], w[e], sum);
                    dot = fmaf(g[e] * w[e], nn[e], dot);
                }
            }
            row_sums<TPR>(dot, sum, slot);
            dot /= (float)width;
            sum /= (float)width;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = (i * TPR + lane) * 8;
                f32x8 g, nn, o = {};
                if constexpr (KEEP) {
                    g = wide(now.dy[i], i);
                    nn = wide(now.h[i], i);
                    if (ds) o = wide(now.ds[i], i);
                } else {                     // (its own values alone: dx may lie over dy or dsum)
                    g = widen(load8(dy + c, width - c));
                    nn = widen(load8(h + c, width - c));
                    if (ds) o = widen(load8(ds + c, width - c));
                }
                const f32x8 w = weights(i);
                nn = (nn - mean) * rstd;
#pragma unroll
                for (int e = 0; e < 8; ++e) o[e] = fmaf(rstd, fmaf(-nn[e], dot, fmaf(g[e], w[e], -sum)), o[e]);
                store_first(dx + c, width - c, narrow<T>(o));
            }
        }
        if constexpr (SUMS) {
            // the parts' sums, or with one part the results themselves
            float* to_w = a.parts == 1 ? a.dweight : a.partial;
            float* to_b = a.parts == 1 ? a.dbias : a.partial + (int64_t)a.groups * a.parts * width;
#pragma unroll
            for (int which = 0; which < 2; ++which) {
                float* to = which ? to_b : to_w;
                f32x8* d = which ? db : dw;
                if (which ? !a.dbias : !a.dweight) continue;
                if constexpr (kRows > 1) {
                    __syncthreads();                     // the last use of part is over
                    if (sub > 0)
#pragma unroll
                        for (int i = 0; i < NV; ++i)
#pragma unroll
                            for (int e = 0; e < 8; ++e) part[(((sub - 1) * NV + i) * 8 + e) * TPR + lane] = d[i][e];
                    __syncthreads();
                    if (sub == 0)
#pragma unroll
                        for (int s = 0; s < kRows - 1; ++s)
#pragma unroll
                            for (int i = 0; i < NV; ++i)
#pragma unroll
                                for (int e = 0; e < 8; ++e) d[i][e] += part[((s * NV + i) * 8 + e) * TPR + lane];
                }
                if (sub == 0)
#pragma unroll
                    for (int i = 0; i < NV; ++i) {
                        const int c = (i * TPR + lane) * 8, n = width - c;
                        if (n > 0) store8(to + item * width + c, n, d[i]);
                    }
            }
        }
    }
}

// The gradients of weight and bias alone, for rows too wide to keep their sums in
// registers: 32 lanes side by side take 256 columns, 8 rows at a time.
template <typename T>
__global__ __launch_bounds__(256) void k_layernorm_columns(const LayerNormGradArgs a) {
    __shared__ float part[7][256][2];
    const int lane = threadIdx.x & 31, sub = threadIdx.x >> 5;
    const int width = (int)a.d.width, c = blockIdx.x * 256 + lane * 8, n = width - c;
    for (int64_t item = blockIdx.y; item < (int64_t)a.groups * a.parts; item += gridDim.y) {
        const int64_t g = item / a.parts, first = g * a.d.span;
        f32x8 dw = {}, db = {};
        if (n > 0)
            for (int64_t at = (item - g * a.parts) * 8 + sub; at < a.d.span; at += (int64_t)a.parts * 8) {
                const int64_t row = first + at;
                const f32x8 dy = widen(load8(static_cast<const T*>(a.dy) + row * a.d.y_stride + c, n));
                const f32x8 nn = (widen(load8(static_cast<const T*>(a.sum) + row * a.d.sum_stride + c, n)) - a.mean[row]) * a.rstd[row];
#pragma unroll
                for (int e = 0; e < 8; ++e) dw[e] = fmaf(dy[e], nn[e], dw[e]);
                db += dy;
            }
        __syncthreads();                     // the last use of part is over
        if (sub > 0)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                part[sub - 1][e * 32 + lane][0] = dw[e];
                part[sub - 1][e * 32 + lane][1] = db[e];
            }
        __syncthreads();
        if (sub == 0 && n > 0) {
#pragma unroll
            for (int s = 0; s < 7; ++s)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    dw[e] += part[s][e * 32 + lane][0];
                    db[e] += part[s][e * 32 + lane][1];
                }
            float* to_w = a.parts == 1 ? a.dweight : a.partial;
            float* to_b = a.parts == 1 ? a.dbias : a.partial + (int64_t)a.groups * a.parts * width;
            if (a.dweight) store8(to_w + item * width + c, n, dw);
            if (a.dbias) store8(to_b + item * width + c, n, db);
        }
    }
}

// The sums over a run's parts: COLS columns a block, each of whose 1024 / COLS lanes take
// every so many parts, four reads at a time.  Grid row 2 g is run g's weight, 2 g + 1 its bias.
// (16 runs of 32 parts of 1001: 64 columns 4 us, 16 columns 8.5; one run of 512 parts: 13 and 4.)
template <int COLS>
__global__ __launch_bounds__(1024) void k_layernorm_join(const LayerNormGradArgs a) {
    constexpr int SUBS = 1024 / COLS;
    __shared__ float part[SUBS][COLS];
    const int col = threadIdx.x % COLS, sub = threadIdx.x / COLS, c = blockIdx.x * COLS + col, width = (int)a.d.width;
    for (int64_t at = blockIdx.y; at < 2 * (int64_t)a.groups; at += gridDim.y) {
        const int64_t g = at >> 1;
        float* to = (at & 1) ? a.dbias : a.dweight;
        if (!to) continue;
        const float* from = a.partial + ((at & 1) * (int64_t)a.groups + g) * a.parts * width;
        float v[4] = {0.f, 0.f, 0.f, 0.f};
        if (c < width)
            for (int b = sub; b < a.parts; b += 4 * SUBS) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (b + SUBS * i < a.parts) v[i] += from[(int64_t)(b + SUBS * i) * width + c];
            }
        __syncthreads();                     // the last use of part is over
        part[sub][col] = (v[0] + v[1]) + (v[2] + v[3]);
        __syncthreads();
#pragma unroll
        for (int half = SUBS / 2; half > 0; half >>= 1) {
            if (sub < half) part[sub][col] += part[sub + half][col];
            __syncthreads();
        }
        if (sub == 0 && c < width) to[g * width + c] = part[0][col];
    }
}

// dweight and dbias of no rows
__global__ __launch_bounds__(256) void k_layernorm_zero(float* dweight, float* dbias, int64_t n) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        if (dweight) dweight[i] = 0.f;
        if (dbias) dbias[i] = 0.f;
    }
}

// lanes and steps of a row by its width
#define PD_LAYERNORM_SHAPES(X) \
    X(7, 64, 1)                \
    X(512, 64, 1)              \
    X(1024, 64, 2)             \
    X(2048, 64, 4)             \
    X(4096, 256, 2)            \
    X(8192, 256, 4)            \
    X(16384, 1024, 2)          \
    X(32768, 1024, 4)          \
    X(65536, 1024, 8)

template <typename T>
void layernorm_t(const LayerNormArgs& a, hipStream_t s) {
#define X(W, TPR, NV)                                                                                            \
    if (a.d.width <= W) {                                                                                        \
        constexpr int rows = TPR < 256 ? 256 / TPR : 1;                                                          \
        hipLaunchKernelGGL((k_layernorm<T, TPR, NV, (W < 8)>), dim3((unsigned)((a.d.rows + rows - 1) / rows)),            \
                           dim3(TPR < 256 ? 256 : TPR), 0, s, a);                                                \
        return;                                                                                                  \
    }
    PD_LAYERNORM_SHAPES(X)
#undef X
}

// The same where the gradients of weight and bias are summed as well, with how many blocks
// a compute unit takes (bfloat16, float32): their sums stay in registers, so rows are spread
// over more lanes.
#define PD_LAYERNORM_SUM_SHAPES(X) \
    X(7, 64, 1, 4, 3)              \
    X(512, 64, 1, 4, 3)            \
    X(1024, 64, 2, 3, 2)           \
    X(2048, 256, 1, 4, 4)          \
    X(4096, 512, 1, 2, 2)          \
    X(8192, 1024, 1, 1, 1)
// above this width a pass of its own sums them, in blocks of 256 columns
constexpr int64_t kFusedWidth = 8192;
constexpr int64_t kMostBlocks = (int64_t)1 << 20;

template <typename T>
void layernorm_grad_t(const LayerNormGradArgs& a, hipStream_t s) {
    const int64_t items = (int64_t)a.groups * a.parts;
    if ((a.dweight || a.dbias) && a.d.width <= kFusedWidth) {
        const dim3 grid((unsigned)(items < kMostBlocks ? items : kMostBlocks));
#define X(W, TPR, NV, B16, B32)                                                                                      \
    if (a.d.width <= W) {                                                                                            \
        constexpr int BLOCKS = sizeof(T) == 2 ? B16 : B32;                                                           \
        hipLaunchKernelGGL((k_layernorm_grad<T, TPR, NV, (W < 8), true, BLOCKS>), grid, dim3(TPR < 256 ? 256 : TPR), 0, s, a); \
        return;                                                                                                      \
    }
        PD_LAYERNORM_SUM_SHAPES(X)
#undef X
    }
    if (a.dweight || a.dbias) {                          // before dx, which may lie over dy
        hipLaunchKernelGGL(k_layernorm_columns<T>, dim3((unsigned)((a.d.width + 255) / 256), (unsigned)(items < 16384 ? items : 16384)),
                           dim3(256), 0, s, a);
        PD_HIP(hipGetLastError());
    }
    LayerNormGradArgs b = a;                             // dx alone: 16 waves a compute unit
#define X(W, TPR, NV)                                                                                                \
    if (a.d.width <= W) {                                                                                            \
        constexpr int rows = TPR < 256 ? 256 / TPR : 1;                                                              \
        const int64_t need = (a.d.span + rows - 1) / rows, most = (4 * kCus * 256 / (TPR < 256 ? 256 : TPR) + a.groups - 1) / a.groups; \
        b.parts = (int)(need < most ? need : most);                                                                  \
        const int64_t all = (int64_t)b.groups * b.parts;                                                             \
        hipLaunchKernelGGL((k_layernorm_grad<T, TPR, NV, (W < 8), false, 1>), dim3((unsigned)(all < kMostBlocks ? all : kMostBlocks)), \
                           dim3(TPR < 256 ? 256 : TPR), 0, s, b);                                                    \
        return;                                                                                                      \
    }
    PD_LAYERNORM_SHAPES(X)
#undef X
}

}  // namespace

// A launch holds fewer than 2^32 threads: 2^21 rows (of up to 1024 lanes) at a time.
constexpr int64_t kLaunchRows = (int64_t)1 << 21;

void launch_layernorm(const LayerNormArgs& all, hipStream_t s) {
    const int64_t elem = all.d.dtype == PD_F32 ? 4 : 2;
    for (int64_t r0 = 0; r0 < all.d.rows; r0 += kLaunchRows) {
        LayerNormArgs a = all;
        a.d.rows = all.d.rows - r0 < kLaunchRows ? all.d.rows - r0 : kLaunchRows;
        a.first = r0;
        a.x = static_cast<const char*>(a.x) + r0 * a.d.x_stride * elem;
        if (a.residual) a.residual = static_cast<const char*>(a.residual) + r0 * a.d.residual_stride * elem;
        if (a.sum) a.sum = static_cast<char*>(a.sum) + r0 * a.d.sum_stride * elem;
        a.y = static_cast<char*>(a.y) + r0 * a.d.y_stride * elem;
        if (a.mean) a.mean += r0;
        if (a.rstd) a.rstd += r0;
        a.d.dtype == PD_F32 ? layernorm_t<float>(a, s) : layernorm_t<bf16>(a, s);
        PD_HIP(hipGetLastError());
    }
}

int layernorm_grad_parts(const pd_layernorm_desc& d) {
    // all runs' parts together: as many blocks as the chip takes; never more than a run has rows for
    if (d.rows == 0) return 1;
    const int64_t groups = d.rows / d.span;
    int64_t blocks = 4 * kCus, rows = 8;                 // (the pass over columns: eight rows at a time)
    if (d.width > kFusedWidth) blocks = (blocks + (d.width + 255) / 256 - 1) / ((d.width + 255) / 256);
#define X(W, TPR, NV, B16, B32)                              \
    else if (d.width <= W) {                                 \
        blocks = (d.dtype == PD_F32 ? B32 : B16) * kCus;     \
        rows = TPR < 256 ? 256 / TPR : 1;                    \
    }
    PD_LAYERNORM_SUM_SHAPES(X)
#undef X
    const int64_t need = (d.span + rows - 1) / rows, most = (blocks + groups - 1) / groups;
    return (int)(need < most ? need : most);
}

void launch_layernorm_grad(const LayerNormGradArgs& a, hipStream_t s) {
    if (a.d.rows == 0) {
        const int64_t n = (int64_t)a.groups * a.d.width;
        hipLaunchKernelGGL(k_layernorm_zero, dim3((unsigned)((n + 255) / 256 < 4096 ? (n + 255) / 256 : 4096)), dim3(256), 0, s,
                           a.dweight, a.dbias, n);
        PD_HIP(hipGetLastError());
        return;
    }
    a.d.dtype == PD_F32 ? layernorm_grad_t<float>(a, s) : layernorm_grad_t<bf16>(a, s);
    PD_HIP(hipGetLastError());
    if ((!a.dweight && !a.dbias) || a.parts == 1) return;
    const int64_t rows = 2 * (int64_t)a.groups;
    const unsigned high = (unsigned)(rows < 512 ? rows : 512);
    if (a.parts > 64)
        hipLaunchKernelGGL(k_layernorm_join<16>, dim3((unsigned)((a.d.width + 15) / 16), high), dim3(1024), 0, s, a);
    else
        hipLaunchKernelGGL(k_layernorm_join<64>, dim3((unsigned)((a.d.width + 63) / 64), high), dim3(1024), 0, s, a);
    PD_HIP(hipGetLastError());
}

}  // namespace pd
