// Rotary positions: the table of (cos, sin) and the turn of q and k by it.
//
//   pair k of a head at position p:  (a, b) -> (a c - b s, a s + b c),  (c, s) = table[p][k]
//
// Bound by memory (each value read and written once; the table's row is shared
// by a token's heads).  A lane holds the (cos, sin) of a unit's pairs in registers and
// turns that unit in several heads.  A unit is eight pairs with halves (two runs of eight
// values), four with pairs side by side (one run), and eight values where they are
// copied: neighbouring lanes load neighbouring 16 bytes of bfloat16.  q and k go in one
// launch.
//
// Measured: 16381 tokens of 32 + 8 heads of 128 bfloat16 values, 96 of them turned, pairs
// side by side, 73 us (4.7 TB/s; a large copy reaches 4.8).
#include "ops.h"

namespace pd {
namespace {

__global__ __launch_bounds__(256) void k_rotary_table(const pd_rotary_table_desc d, int64_t first, int64_t rows,
                                                      float* table) {
    const int half = d.rotary_dim / 2;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= rows * half) return;
    const int k = (int)(i % half);
    double base = d.base;
    if (d.scaling == PD_ROTARY_BASE && d.rotary_dim > 2)
        base *= pow(d.factor, (double)d.rotary_dim / (double)(d.rotary_dim - 2));
    double f = pow(base, -2.0 * k / (double)d.rotary_dim);
    if (d.scaling == PD_ROTARY_LINEAR) f /= d.factor;
    if (d.scaling == PD_ROTARY_BY_PARTS) {
        const double turns = d.original_length * f / 6.283185307179586477;
        double g = (turns - d.turns_low) / (d.turns_high - d.turns_low);
        g = g < 0.0 ? 0.0 : (g > 1.0 ? 1.0 : g);
        f = g * f + (1.0 - g) * f / d.factor;
    }
    double sn, cs;
    sincos((double)(first + i / half) * f, &sn, &cs);
    table[2 * i] = (float)(cs * d.magnitude);
    table[2 * i + 1] = (float)(sn * d.magnitude);
}

// One lane: unit u of a token (pairs while u < pair_units, then values to copy) in the
// heads hs, hs + lanes_h, ...; the heads of q, then of k.
template <typename T, bool HALF>
__global__ __launch_bounds__(256) void k_rotary(const RotaryArgs a, int units, int pair_units, int lanes_h, int64_t lanes) {
    constexpr int kPairs = HALF ? 8 : 4;
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (id >= lanes) return;
    const int per_token = units * lanes_h;
    const int64_t token = id / per_token;
    const int rest = (int)(id - token * per_token);
    const int hs = rest / units, u = rest - hs * units;
    const int64_t b = token / a.d.length, i = token - b * a.d.length;
    const int R = a.d.rotary_dim, half = R / 2;
    const bool turn = u < pair_units;
    // first element of the run (halves: and of the second), and how many of each count
    int e0, n0;
    float cs[kPairs], sn[kPairs];
    if (turn) {
        const int k0 = u * kPairs, pairs = min(half - k0, kPairs);
        e0 = HALF ? k0 : 2 * k0;
        n0 = HALF ? pairs : 2 * pairs;
        int64_t pos = a.positions[b * a.d.position_stride + i];
        pos = pos < 0 ? 0 : (pos >= a.d.table_rows ? a.d.table_rows - 1 : pos);
        const float* t = a.table + (pos * half + k0) * 2;
#pragma unroll
        for (int r = 0; r < kPairs / 4; ++r) {
            const f32x8 v = load8(t + 8 * r, 2 * pairs - 8 * r);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                cs[4 * r + e] = v[2 * e];
                sn[4 * r + e] = a.d.backward ? -v[2 * e + 1] : v[2 * e + 1];
            }
        }
    } else {
        e0 = R + (u - pair_units) * 8;
        n0 = a.d.head_dim - e0;
    }
    const int heads = a.d.heads_q + a.d.heads_k;
    for (int h = hs; h < heads; h += lanes_h) {
        const bool is_k = h >= a.d.heads_q;
        const int hh = is_k ? h - a.d.heads_q : h;
        const int64_t* st = is_k ? a.d.k_stride : a.d.q_stride;
        const int64_t* so = is_k ? a.d.k_out_stride : a.d.q_out_stride;
        const T* x = static_cast<const T*>(is_k ? a.k : a.q) + b * st[0] + i * st[1] + hh * st[2] + e0;
        T* y = static_cast<T*>(is_k ? a.k_out : a.q_out) + b * so[0] + i * so[1] + hh * so[2] + e0;
        typename Vec8<T>::type p = load8(x, n0);
        if (!turn) {
            store8(y, n0, p);
            continue;
        }
        const f32x8 v = widen(p);
        f32x8 ra;
        if constexpr (HALF) {
            const f32x8 w = widen(load8(x + half, n0));
            f32x8 rb;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                ra[e] = v[e] * cs[e] - w[e] * sn[e];
                rb[e] = v[e] * sn[e] + w[e] * cs[e];
            }
            store8(y + half, n0, narrow<T>(rb));
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                ra[2 * e] = v[2 * e] * cs[e] - v[2 * e + 1] * sn[e];
                ra[2 * e + 1] = v[2 * e] * sn[e] + v[2 * e + 1] * cs[e];
            }
        }
        store8(y, n0, narrow<T>(ra));
    }
}

template <typename T>
void rotary_t(const RotaryArgs& a, hipStream_t s) {
    const pd_rotary_desc& d = a.d;
    const int pairs = d.layout == PD_ROTARY_HALF ? 8 : 4;
    const int pair_units = (d.rotary_dim / 2 + pairs - 1) / pairs, units = pair_units + (d.head_dim - d.rotary_dim + 7) / 8;
    const int heads = d.heads_q + d.heads_k;
    const int64_t tokens = d.batch * d.length;
    // heads a lane: as many as leave 16 waves a compute unit, at most 8 (the case above
    // with one head a lane: 95 us)
    int per = 1;
    while (per < 8 && per < heads && tokens * units * ((heads + 2 * per - 1) / (2 * per)) >= (int64_t)device_cus() * 1024) per *= 2;
    const int lanes_h = (heads + per - 1) / per;
    const int64_t lanes = tokens * units * lanes_h;
    const dim3 grid((unsigned)((lanes + 255) / 256)), block(256);
    if (d.layout == PD_ROTARY_HALF)
        hipLaunchKernelGGL((k_rotary<T, true>), grid, block, 0, s, a, units, pair_units, lanes_h, lanes);
    else
        hipLaunchKernelGGL((k_rotary<T, false>), grid, block, 0, s, a, units, pair_units, lanes_h, lanes);
    PD_HIP(hipGetLastError());
}

}  // namespace

void launch_rotary(const RotaryArgs& a, hipStream_t s) {
    a.d.dtype == PD_F32 ? rotary_t<float>(a, s) : rotary_t<bf16>(a, s);
}

void launch_rotary_table(const pd_rotary_table_desc& d, int64_t first, int64_t rows, float* table, hipStream_t s) {
    const int64_t n = rows * (d.rotary_dim / 2);
    hipLaunchKernelGGL(k_rotary_table, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s, d, first, rows, table);
    PD_HIP(hipGetLastError());
}

}  // namespace pd
