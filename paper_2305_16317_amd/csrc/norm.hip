// Root-mean-square norm with the residual's addition, forward and backward.
//
//   s = x + r,  rstd = (mean s^2 + eps)^-1/2,  y = s rstd w
//   a = dy w, n = s rstd:  dx = dsum + rstd (a - n mean(a n)),  dw = sum_rows dy n
//
// Bound by memory: 3 or 4 values move per element and a dozen operations.  A row
// stays in registers from its one read to its writes, eight values a lane and
// step; rows up to 2048 values belong to one wave (no barrier, four rows a
// block), longer ones to a block of 256 or 1024 lanes.  (1500 values: a wave 57.8 us for
// 16384 rows, a block of 256 65.2; 2048 values: 57.4 and 49.1.)
//
// Measured: 36864 x 1024 bfloat16 with residual to e4m3, a scale for 128 values, 56 us (4.7
// TB/s; a large copy reaches 4.8); backward on 12432 x 1001 34 us (2.9 TB/s), of which
// 24 for the rows and 4 for the weight's gradient.
#include "ops.h"

namespace pd {
namespace {

constexpr float kE4m3Max = 448.f;
constexpr float kMinNormal = 1.17549435e-38f;

__device__ inline float wave_sum(float v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    return v;
}
// The largest of values >= 0 by their bits, in which a NaN is above infinity.
__device__ inline uint32_t wave_max(uint32_t v, int width) {
    for (int o = width >> 1; o > 0; o >>= 1) {
        const uint32_t w = (uint32_t)__shfl_xor((int)v, o);
        v = v > w ? v : w;
    }
    return v;
}
// Sum over the TPR lanes of a row; `slot` holds one value a wave.
template <int TPR>
__device__ inline float row_sum(float v, float* slot) {
    v = wave_sum(v);
    if constexpr (TPR > 64) {
        __syncthreads();                     // the last use of slot is over
        if ((threadIdx.x & 63) == 0) slot[threadIdx.x >> 6] = v;
        __syncthreads();
        v = slot[0];
#pragma unroll
        for (int w = 1; w < TPR / 64; ++w) v += slot[w];
    }
    return v;
}
template <int TPR>
__device__ inline uint32_t row_max(uint32_t v, float* slot) {
    v = wave_max(v, 64);
    if constexpr (TPR > 64) {
        uint32_t* u = reinterpret_cast<uint32_t*>(slot);
        __syncthreads();
        if ((threadIdx.x & 63) == 0) u[threadIdx.x >> 6] = v;
        __syncthreads();
        v = u[0];
#pragma unroll
        for (int w = 1; w < TPR / 64; ++w) v = v > u[w] ? v : u[w];
    }
    return v;
}

typedef uint32_t u32x2_u __attribute__((ext_vector_type(2), aligned(1)));

// eight values as e4m3, to nearest even (values are within +-448, or NaN)
__device__ inline void store_e4m3(uint8_t* p, int n, f32x8 v) {
    int lo = 0, hi = 0;
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], lo, false);
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], lo, true);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(v[4], v[5], hi, false);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(v[6], v[7], hi, true);
    if (n >= 8) {
        u32x2_u w = {(uint32_t)lo, (uint32_t)hi};
        *reinterpret_cast<u32x2_u*>(p) = w;
        return;
    }
#pragma unroll
    for (int e = 0; e < 7; ++e)
        if (e < n) p[e] = (uint8_t)((e < 4 ? lo : hi) >> (8 * (e & 3)));
}

// TPR lanes a row, NV steps of eight values a lane.
template <typename T, bool F8, int TPR, int NV>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void k_rmsnorm(const NormArgs a) {
    constexpr int kRows = TPR < 256 ? 256 / TPR : 1;      // rows a block
    __shared__ float slot[16];
    const int lane = threadIdx.x % TPR;
    const int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / TPR;
    if (row >= a.d.rows) return;             // whole waves; with TPR > 64 there is one row a block
    const int width = (int)a.d.width;
    const T* x = static_cast<const T*>(a.x) + row * a.d.x_stride;
    const T* r = a.residual ? static_cast<const T*>(a.residual) + row * a.d.residual_stride : nullptr;
    f32x8 v[NV];
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * TPR + lane) * 8, n = width - c;
        v[i] = f32x8{};
        if (n <= 0) continue;
        v[i] = widen(load8(x + c, n));
        if (r) v[i] += widen(load8(r + c, n));
    }
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) ss = fmaf(v[i][e], v[i][e], ss);
    const float rstd = 1.f / sqrtf(row_sum<TPR>(ss, slot) / (float)width + a.d.eps);
    if (a.rstd && lane == 0) a.rstd[row] = rstd;
    if (a.sum) {
        T* h = static_cast<T*>(a.sum) + row * a.d.sum_stride;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * TPR + lane) * 8, n = width - c;
            if (n > 0) store8(h + c, n, narrow<T>(v[i]));
        }
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * TPR + lane) * 8, n = width - c;
        if (n > 0) v[i] = v[i] * rstd * load8(a.weight + c, n);
    }
    if constexpr (!F8) {
        T* y = static_cast<T*>(a.y) + row * a.d.y_stride;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * TPR + lane) * 8, n = width - c;
            if (n > 0) store8(y + c, n, narrow<T>(v[i]));
        }
    } else {
        uint8_t* y = static_cast<uint8_t*>(a.y) + row * a.d.y_stride;
        const int group = a.d.group;
        const int per_row = group ? (width + group - 1) / group : 1;
        uint32_t top[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            top[i] = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t b = __float_as_uint(v[i][e]) & 0x7fffffffu;
                top[i] = top[i] > b ? top[i] : b;
            }
        }
        if (!group) {
            uint32_t m = top[0];
#pragma unroll
            for (int i = 1; i < NV; ++i) m = m > top[i] ? m : top[i];
            m = row_max<TPR>(m, slot);
#pragma unroll
            for (int i = 0; i < NV; ++i) top[i] = m;
        } else {                             // a group: group / 8 neighbouring lanes of one step
#pragma unroll
            for (int i = 0; i < NV; ++i) top[i] = wave_max(top[i], group >> 3);
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * TPR + lane) * 8, n = width - c;
            if (n <= 0) continue;
            float scale = __uint_as_float(top[i]) / kE4m3Max;
            if (scale < kMinNormal) scale = 0.f;
            if (group ? c % group == 0 : c == 0) a.scale[row * per_row + (group ? c / group : 0)] = scale;
            f32x8 q;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                q[e] = scale == 0.f ? 0.f : v[i][e] / scale;
                // the quotient's rounding may pass 448, which is no value of the format
                q[e] = q[e] > kE4m3Max ? kE4m3Max : (q[e] < -kE4m3Max ? -kE4m3Max : q[e]);
            }
            store_e4m3(y + c, n, q);
        }
    }
}

// Backward: a lane keeps its columns over all rows of its wave (or block), so dw
// is summed in registers, then over the block's rows in LDS, and the blocks'
// sums by k_norm_dweight: a fixed order.
template <typename T, int TPR, int NV>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void k_rmsnorm_grad(const NormGradArgs a) {
    constexpr int kRows = TPR < 256 ? 256 / TPR : 1;
    __shared__ float slot[16];
    __shared__ float part[kRows > 1 ? (kRows - 1) * TPR * NV * 8 : 1];
    const int lane = threadIdx.x % TPR, sub = threadIdx.x / TPR;
    const int width = (int)a.d.width;
    f32x8 w[NV], dw[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * TPR + lane) * 8, n = width - c;
        dw[i] = f32x8{};
        w[i] = f32x8{};
        if (n > 0) w[i] = load8(a.weight + c, n);
    }
    for (int64_t row = (int64_t)blockIdx.x * kRows + sub; row < a.d.rows; row += (int64_t)gridDim.x * kRows) {
        const T* dy = static_cast<const T*>(a.dy) + row * a.d.y_stride;
        const T* h = static_cast<const T*>(a.sum) + row * a.d.sum_stride;
        const T* ds = a.dsum ? static_cast<const T*>(a.dsum) + row * a.d.residual_stride : nullptr;
        T* dx = static_cast<T*>(a.dx) + row * a.d.x_stride;
        const float rstd = a.rstd[row];
        typename Vec8<T>::type vdy[NV], vh[NV], vds[NV];
        float dot = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * TPR + lane) * 8, n = width - c;
            vdy[i] = typename Vec8<T>::type{};
            vh[i] = typename Vec8<T>::type{};
            vds[i] = typename Vec8<T>::type{};
            if (n <= 0) continue;
            vdy[i] = load8(dy + c, n);
            vh[i] = load8(h + c, n);
            if (ds) vds[i] = load8(ds + c, n);
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const f32x8 g = widen(vdy[i]), nn = widen(vh[i]) * rstd;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                dw[i][e] = fmaf(g[e], nn[e], dw[i][e]);
                dot = fmaf(g[e] * w[i][e], nn[e], dot);
            }
        }
        const float mean = row_sum<TPR>(dot, slot) / (float)width;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * TPR + lane) * 8, n = width - c;
            if (n <= 0) continue;
            const f32x8 g = widen(vdy[i]), nn = widen(vh[i]) * rstd;
            f32x8 o = widen(vds[i]);
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = fmaf(rstd, fmaf(-nn[e], mean, g[e] * w[i][e]), o[e]);
            store8(dx + c, n, narrow<T>(o));
        }
    }
    if (!a.dweight) return;
    if constexpr (kRows > 1) {
        if (sub > 0)
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) part[(((sub - 1) * NV + i) * 8 + e) * TPR + lane] = dw[i][e];
        __syncthreads();
        if (sub > 0) return;
#pragma unroll
        for (int s = 0; s < kRows - 1; ++s)
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) dw[i][e] += part[((s * NV + i) * 8 + e) * TPR + lane];
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * TPR + lane) * 8, n = width - c;
        if (n > 0) store8(a.partial + (int64_t)blockIdx.x * width + c, n, dw[i]);
    }
}

// dweight[c] = sum over blocks: 16 columns a block and 64 lanes down each, which take
// every 64th row of the sums, four loads at a time (a chain of loads one after the other
// took 20 us over 512 x 1001 sums; so, 4 us).
__global__ __launch_bounds__(1024) void k_norm_dweight(const float* partial, int blocks, int width, float* dweight) {
    __shared__ float part[64][17];
    const int col = threadIdx.x & 15, sub = threadIdx.x >> 4, c = blockIdx.x * 16 + col;
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    if (c < width)
        for (int b = sub; b < blocks; b += 256) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (b + 64 * i < blocks) v[i] += partial[(int64_t)(b + 64 * i) * width + c];
        }
    part[sub][col] = (v[0] + v[1]) + (v[2] + v[3]);
    __syncthreads();
    // a wave of the 16 takes one column
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const float sum = wave_sum(part[lane][wave]);
    if (lane == 0 && blockIdx.x * 16 + wave < width) dweight[blockIdx.x * 16 + wave] = sum;
}

// lanes and steps of a row by its width
#define PD_NORM_SHAPES(X)      \
    X(512, 64, 1)              \
    X(1024, 64, 2)             \
    X(2048, 64, 4)             \
    X(4096, 256, 2)            \
    X(8192, 256, 4)            \
    X(16384, 1024, 2)          \
    X(32768, 1024, 4)          \
    X(65536, 1024, 8)

template <typename T, bool F8>
void rmsnorm_t(const NormArgs& a, hipStream_t s) {
#define X(W, TPR, NV)                                                                              \
    if (a.d.width <= W) {                                                                          \
        constexpr int rows = TPR < 256 ? 256 / TPR : 1;                                            \
        hipLaunchKernelGGL((k_rmsnorm<T, F8, TPR, NV>), dim3((unsigned)((a.d.rows + rows - 1) / rows)), \
                           dim3(TPR < 256 ? 256 : TPR), 0, s, a);                                  \
        return;                                                                                    \
    }
    PD_NORM_SHAPES(X)
#undef X
}
template <typename T>
void rmsnorm_grad_t(const NormGradArgs& a, int blocks, hipStream_t s) {
#define X(W, TPR, NV)                                                                                   \
    if (a.d.width <= W) {                                                                               \
        hipLaunchKernelGGL((k_rmsnorm_grad<T, TPR, NV>), dim3(blocks), dim3(TPR < 256 ? 256 : TPR), 0, s, a); \
        return;                                                                                         \
    }
    PD_NORM_SHAPES(X)
#undef X
}

}  // namespace

// A launch holds fewer than 2^32 threads: 2^21 rows (of up to 1024 lanes) at a time.
constexpr int64_t kLaunchRows = (int64_t)1 << 21;

void launch_rmsnorm(const NormArgs& all, hipStream_t s) {
    const bool f8 = all.d.out_dtype == PD_F8E4M3;
    const int64_t elem = all.d.dtype == PD_F32 ? 4 : 2;
    const int64_t scales = all.d.group ? (all.d.width + all.d.group - 1) / all.d.group : 1;
    for (int64_t r0 = 0; r0 < all.d.rows; r0 += kLaunchRows) {
        NormArgs a = all;
        a.d.rows = all.d.rows - r0 < kLaunchRows ? all.d.rows - r0 : kLaunchRows;
        a.x = static_cast<const char*>(a.x) + r0 * a.d.x_stride * elem;
        if (a.residual) a.residual = static_cast<const char*>(a.residual) + r0 * a.d.residual_stride * elem;
        if (a.sum) a.sum = static_cast<char*>(a.sum) + r0 * a.d.sum_stride * elem;
        a.y = static_cast<char*>(a.y) + r0 * a.d.y_stride * (f8 ? 1 : elem);
        if (a.scale) a.scale += r0 * scales;
        if (a.rstd) a.rstd += r0;
        if (a.d.dtype == PD_F32)
            f8 ? rmsnorm_t<float, true>(a, s) : rmsnorm_t<float, false>(a, s);
        else
            f8 ? rmsnorm_t<bf16, true>(a, s) : rmsnorm_t<bf16, false>(a, s);
        PD_HIP(hipGetLastError());
    }
}

int norm_grad_blocks(const pd_rmsnorm_desc& d) {
    // two blocks a compute unit; never more than there are rows for
    const int64_t per = d.width <= 2048 ? 4 : 1, need = (d.rows + per - 1) / per, most = 2 * device_cus();
    return (int)(need < 1 ? 1 : need < most ? need : most);
}

void launch_rmsnorm_grad(const NormGradArgs& a, hipStream_t s) {
    const int blocks = norm_grad_blocks(a.d);
    a.d.dtype == PD_F32 ? rmsnorm_grad_t<float>(a, blocks, s) : rmsnorm_grad_t<bf16>(a, blocks, s);
    PD_HIP(hipGetLastError());
    if (!a.dweight) return;
    hipLaunchKernelGGL(k_norm_dweight, dim3((unsigned)((a.d.width + 15) / 16)), dim3(1024), 0, s, a.partial, blocks,
                       (int)a.d.width, a.dweight);
    PD_HIP(hipGetLastError());
}

}  // namespace pd
