// Dropout by a counter-based generator, with the residual's addition.
//
//   y = r + (u >= t ? x 65536 / (65536 - t) : 0),  t = p in steps of 2^-16
//
// Eight neighbouring values of a row take one 128-bit block of Philox4x32-10 (philox.h),
// 16 bits u each, so the mask follows from the seed and the place alone: it is never
// stored, and the gradient is the same call on dy.
//
// Bound by memory: two or three values move per element, and the generator's 20 products
// for eight values pass beside them.  Measured: 36864 x 1024 bfloat16 with a residual 33 us (6.9
// TB/s: it fits the last cache; a large copy reaches 5.0), 131072 x 1024 without one 88 us (6.1).
#include "ops.h"
#include "philox.h"

namespace pd {
namespace {

// Lane: eight values (unit `id` of the launch's rows x `per`).  FLAT: every tensor is one
// run of whole units, so that no unit's row is needed.
template <typename T, bool FLAT>
__global__ __launch_bounds__(256) void k_dropout(const DropoutArgs a, uint32_t units, uint32_t per) {
    const uint32_t id = blockIdx.x * 256 + threadIdx.x;
    if (id >= units) return;
    uint32_t row = 0, c = id;
    if constexpr (!FLAT) {
        row = id / per;
        c = id - row * per;
    }
    const int n = FLAT ? 8 : (int)(a.d.width - 8 * (int64_t)c < 8 ? a.d.width - 8 * (int64_t)c : 8);
    const T* x = static_cast<const T*>(a.x) + (int64_t)row * a.d.x_stride + 8 * (int64_t)c;
    const typename Vec8<T>::type xv = load8(x, n);
    typename Vec8<T>::type rv = {};
    if (a.residual) rv = load8(static_cast<const T*>(a.residual) + (int64_t)row * a.d.residual_stride + 8 * (int64_t)c, n);
    const uint64_t q = (uint64_t)(a.first * (int64_t)per) + id;
    uint32_t w[4] = {(uint32_t)q, (uint32_t)(q >> 32), a.d.rng_stream, a.d.step + 1 + (a.step ? *a.step : 0)};
    philox4x32_10(w[0], w[1], w[2], w[3], (uint32_t)a.d.seed, (uint32_t)(a.d.seed >> 32));
    const f32x8 v = widen(xv), r = widen(rv);
    f32x8 o;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t u = (e & 1) ? w[e >> 1] >> 16 : w[e >> 1] & 0xffffu;
        o[e] = u >= a.under ? v[e] * a.scale : 0.f;       // (a dropped value is not read: infinity and NaN give 0 too)
        if (a.residual) o[e] += r[e];
    }
    store8(static_cast<T*>(a.y) + (int64_t)row * a.d.y_stride + 8 * (int64_t)c, n, narrow<T>(o));
}

template <typename T>
void dropout_t(const DropoutArgs& all, hipStream_t s) {
    const int64_t per = (all.d.width + 7) / 8;
    const int64_t most = ((int64_t)1 << 30) / per;       // rows a launch (per <= 2^28)
    for (int64_t r0 = 0; r0 < all.d.rows; r0 += most) {
        DropoutArgs a = all;
        const int64_t rows = all.d.rows - r0 < most ? all.d.rows - r0 : most;
        a.first = all.d.first_row + r0;
        a.x = static_cast<const T*>(a.x) + r0 * a.d.x_stride;
        if (a.residual) a.residual = static_cast<const T*>(a.residual) + r0 * a.d.residual_stride;
        a.y = static_cast<T*>(a.y) + r0 * a.d.y_stride;
        const auto whole = [&](int64_t stride) { return rows == 1 || stride == a.d.width; };
        const bool flat = a.d.width % 8 == 0 && whole(a.d.x_stride) && whole(a.d.y_stride) && (!a.residual || whole(a.d.residual_stride));
        const uint32_t units = (uint32_t)(rows * per);
        if (flat)
            hipLaunchKernelGGL((k_dropout<T, true>), dim3((units + 255) / 256), dim3(256), 0, s, a, units, (uint32_t)per);
        else
            hipLaunchKernelGGL((k_dropout<T, false>), dim3((units + 255) / 256), dim3(256), 0, s, a, units, (uint32_t)per);
        PD_HIP(hipGetLastError());
    }
}

}  // namespace

void launch_dropout(const DropoutArgs& a, hipStream_t s) { a.d.dtype == PD_F32 ? dropout_t<float>(a, s) : dropout_t<bf16>(a, s); }

}  // namespace pd
