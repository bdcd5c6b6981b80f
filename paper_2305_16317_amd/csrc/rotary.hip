// Rotary positions: the table of (cos, sin) and the turn of q and k by it.
//
//   pair k of a head at position p:  (a, b) -> (a c - b s, a s + b c),  (c, s) = table[p][k]
//
// With several axes a token has a position on each, and p is that of the axis which pair k
// belongs to (AxisMap: two bits a pair).
//
// Bound by memory (each value read and written once; the table's row is shared
// by a token's heads).  A lane holds the (cos, sin) of a unit's pairs in registers and
// turns that unit in several heads.  A unit is eight pairs with halves (two runs of eight
// values), four with pairs side by side (one run), and eight values where they are
// copied: neighbouring lanes load neighbouring 16 bytes of bfloat16.  q and k go in one
// launch.
//
// Measured: 16381 tokens of 32 + 8 heads of 128 bfloat16 values, 96 of them turned, pairs
// side by side, 70 to 72 us (4.7 TB/s; a large copy reaches 4.8 to 5.0); 16384 tokens of a video's
// three axes in turn, 32 + 8 heads of 128, 70 us (4.8 TB/s; with one head's values at a time,
// read after the table, 86).
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

// The table of several axes: pair k of axis a, the i-th of the axis's n, turns by
// base_a^(-i / n) scale_a, or with `shared` by base_a^(-k / pairs) scale_a.
__global__ __launch_bounds__(256) void k_rotary_axes_table(const pd_rotary_axes_table_desc d, const AxisMap map, int64_t first,
                                                           int64_t rows, float* table) {
    const int half = d.rotary_dim / 2;
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (at >= rows * half) return;
    const int k = (int)(at % half), a = map.axis(k);
    int i = 0;
    for (int j = 0; j < k; ++j) i += map.axis(j) == a;
    const double part = d.shared ? (double)k / half : (double)i / d.sections[a];
    double sn, cs;
    sincos((double)(first + at / half) * (pow(d.base[a], -part) * d.scale[a]), &sn, &cs);
    table[2 * at] = (float)cs;
    table[2 * at + 1] = (float)sn;
}

// One lane: unit u of a token (pairs while u < pair_units, then values to copy) in the
// heads hs, hs + lanes_h, ...; the heads of q, then of k.
template <typename T, bool HALF, class Args>
__global__ __launch_bounds__(256) void k_rotary(const Args a, int units, int pair_units, int lanes_h, uint32_t lanes) {
    constexpr int kPairs = HALF ? 8 : 4;
    const uint32_t id = blockIdx.x * 256 + threadIdx.x;        // (fewer than 2^32 lanes)
    if (id >= lanes) return;
    const uint32_t per_token = units * lanes_h, token = id / per_token;
    const int rest = (int)(id - token * per_token);
    const int hs = rest / units, u = rest - hs * units;
    int64_t b = 0, i = token;
    if (a.d.batch > 1) b = token / (uint32_t)a.d.length, i = token - b * a.d.length;
    const int R = a.d.rotary_dim, half = R / 2;
    const bool turn = u < pair_units;
    // first element of the run (halves: and of the second), and how many of each count
    const int k0 = u * kPairs, pairs = min(half - k0, kPairs);
    const int e0 = !turn ? R + (u - pair_units) * 8 : HALF ? k0 : 2 * k0, n0 = !turn ? a.d.head_dim - e0 : HALF ? pairs : 2 * pairs;
    const int heads = a.d.heads_q + a.d.heads_k;
    // four heads' values at a time; the first four are on the way while the table is read
    constexpr int kBatch = 4;
    typename Vec8<T>::type p[kBatch], w[kBatch];
    const auto fetch = [&](int first) {
#pragma unroll
        for (int c = 0; c < kBatch; ++c) {
            const int h = first + c * lanes_h;
            if (h >= heads) break;
            const bool is_k = h >= a.d.heads_q;
            const int hh = is_k ? h - a.d.heads_q : h;
            const int64_t* st = is_k ? a.d.k_stride : a.d.q_stride;
            const T* x = static_cast<const T*>(is_k ? a.k : a.q) + b * st[0] + i * st[1] + hh * st[2] + e0;
            p[c] = load8(x, n0);
            if (HALF && turn) w[c] = load8(x + half, n0);
        }
    };
    fetch(hs);
    float cs[kPairs], sn[kPairs];
    if (turn) {
        const auto clamped = [&](int64_t pos) { return pos < 0 ? 0 : (pos >= a.d.table_rows ? a.d.table_rows - 1 : pos); };
        const auto set = [&](int e, float c, float s) {
            cs[e] = c;
            sn[e] = a.d.backward ? -s : s;
        };
        const auto row = [&](int64_t pos) {                // the unit's pairs from one row of the table
            const float* t = a.table + (clamped(pos) * half + k0) * 2;
#pragma unroll
            for (int r = 0; r < kPairs / 4; ++r) {
                const f32x8 v = load8(t + 8 * r, 2 * pairs - 8 * r);
#pragma unroll
                for (int e = 0; e < 4; ++e) set(4 * r + e, v[2 * e], v[2 * e + 1]);
            }
        };
        if constexpr (!Args::kAxes) {
            row(a.positions[b * a.d.position_stride + i]);
        } else {
            const int32_t* at = a.positions + b * a.position_strides[0] + i * a.position_strides[1];
            const uint32_t axes = a.map.word[k0 >> 4] >> (2 * (k0 & 15)), mine = (1u << (2 * pairs)) - 1, one = axes & 3;
            if (((axes ^ (one * 0x5555u)) & mine) == 0) {
                row(at[one * a.position_strides[2]]);
            } else {
#pragma unroll
                for (int e = 0; e < kPairs; ++e) {
                    const int64_t pos = clamped(at[((axes >> (2 * e)) & 3) * a.position_strides[2]]);
                    const int k = e < pairs ? k0 + e : k0;
                    const float* t = a.table + (pos * half + k) * 2;
                    set(e, t[0], t[1]);
                }
            }
        }
    }
    for (int first = hs; first < heads; first += kBatch * lanes_h) {
        if (first != hs) fetch(first);
#pragma unroll
        for (int c = 0; c < kBatch; ++c) {
            const int h = first + c * lanes_h;
            if (h >= heads) break;
            const bool is_k = h >= a.d.heads_q;
            const int hh = is_k ? h - a.d.heads_q : h;
            const int64_t* so = is_k ? a.d.k_out_stride : a.d.q_out_stride;
            T* y = static_cast<T*>(is_k ? a.k_out : a.q_out) + b * so[0] + i * so[1] + hh * so[2] + e0;
            if (!turn) {
                store8(y, n0, p[c]);
                continue;
            }
            const f32x8 v = widen(p[c]);
            f32x8 ra;
            if constexpr (HALF) {
                const f32x8 vw = widen(w[c]);
                f32x8 rb;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    ra[e] = v[e] * cs[e] - vw[e] * sn[e];
                    rb[e] = v[e] * sn[e] + vw[e] * cs[e];
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
}

template <typename T, class Args>
void rotary_t(const Args& a, hipStream_t s) {
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
        hipLaunchKernelGGL((k_rotary<T, true, Args>), grid, block, 0, s, a, units, pair_units, lanes_h, (uint32_t)lanes);
    else
        hipLaunchKernelGGL((k_rotary<T, false, Args>), grid, block, 0, s, a, units, pair_units, lanes_h, (uint32_t)lanes);
    PD_HIP(hipGetLastError());
}

}  // namespace

void launch_rotary(const RotaryArgs& a, hipStream_t s) {
    a.d.dtype == PD_F32 ? rotary_t<float>(a, s) : rotary_t<bf16>(a, s);
}

void launch_rotary_axes(const RotaryAxesArgs& a, hipStream_t s) {
    a.d.dtype == PD_F32 ? rotary_t<float>(a, s) : rotary_t<bf16>(a, s);
}

void launch_rotary_axes_table(const pd_rotary_axes_table_desc& d, const AxisMap& map, int64_t first, int64_t rows, float* table,
                              hipStream_t s) {
    const int64_t n = rows * (d.rotary_dim / 2);
    hipLaunchKernelGGL(k_rotary_axes_table, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s, d, map, first, rows, table);
    PD_HIP(hipGetLastError());
}

void launch_rotary_table(const pd_rotary_table_desc& d, int64_t first, int64_t rows, float* table, hipStream_t s) {
    const int64_t n = rows * (d.rotary_dim / 2);
    hipLaunchKernelGGL(k_rotary_table, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s, d, first, rows, table);
    PD_HIP(hipGetLastError());
}

}  // namespace pd
