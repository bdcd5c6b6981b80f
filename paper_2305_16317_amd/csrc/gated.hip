// The gated product of a feed-forward block, forward and backward.
//
//   g = x Wg, u = x Wu, h = act(g) u
//   dg = dh u act'(g), du = dh act(g);  dx = dg Wg^T + du Wu^T,  dWg = x^T dg, dWu = x^T du
//
// All products run in one kernel (k_product) over bfloat16 operands: blocks of BM rows
// and twice HN columns, the two halves being gate and up, or neighbours of one matrix.
// Operands are read as they lie, along the sum (units of a row are fragments) or across
// it (transposing LDS reads).  float32 operands are split into three bfloat16 parts first,
// and the six products of parts that count are six segments of the sum, small ones first.
// Operands that copies of 16 bytes cannot read (alignment, odd sizes) are laid out first.
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
    int segs, k, steps;                  // steps of 64 a segment
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
__device__ inline float sigmoid(float v) { return 1.f / (1.f + expf(-v)); }
__device__ inline float activate(int act, float g) {
    switch (act) {
        case PD_ACT_SILU: return g / (1.f + expf(-g));
        case PD_ACT_GELU: return 0.5f * g * (1.f + erff(g * 0.707106781f));
        case PD_ACT_GELU_TANH: return 0.5f * g * (1.f + tanhf(0.797884561f * (g + 0.044715f * g * g * g)));
        case PD_ACT_SIGMOID: return sigmoid(g);
        default: return g > 0.f ? g : (g != g ? g : 0.f);
    }
}
// (act, its slope) at g
__device__ inline void activate_grad(int act, float g, float& a, float& slope) {
    switch (act) {
        case PD_ACT_SILU: {
            const float s = sigmoid(g);
            a = g * s;
            slope = s * (1.f + g * (1.f - s));
            return;
        }
        case PD_ACT_GELU: {
            const float p = 0.5f * (1.f + erff(g * 0.707106781f));
            a = g * p;
            slope = p + g * expf(-0.5f * g * g) * 0.398942280f;
            return;
        }
        case PD_ACT_GELU_TANH: {
            const float t = tanhf(0.797884561f * (g + 0.044715f * g * g * g));
            a = 0.5f * g * (1.f + t);
            slope = 0.5f * (1.f + t) + 0.5f * g * (1.f - t * t) * 0.797884561f * (1.f + 0.134145f * g * g);
            return;
        }
        case PD_ACT_SIGMOID: {
            const float s = sigmoid(g);
            a = s;
            slope = s * (1.f - s);
            return;
        }
        default:
            a = g > 0.f ? g : (g != g ? g : 0.f);
            slope = g > 0.f ? 1.f : (g != g ? g : 0.f);
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

// A tile of ROWS rows of UNITS units of 16 bytes, copied by 256 threads in Tile's order.
// ACROSS: its rows run along the sum, else its units do.
template <int ROWS, int UNITS, bool ACROSS>
struct Operand {
    using Ti = Tile<bf16, UNITS * 8>;
    static constexpr int kCopies = ROWS * UNITS / 256, kBytes = ROWS * UNITS * 16;
    static_assert(ROWS * UNITS % 256 == 0, "whole copies");
    uint32_t off[kCopies];                 // from the tile's first element
    uint32_t to;
    static __device__ __forceinline__ int row_of(int i, int thread) { return (i * 256 + thread) / UNITS; }
    static __device__ __forceinline__ int unit_of(int i, int thread) {
        return ((i * 256 + thread) % UNITS) ^ Ti::swz(row_of(i, thread));
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
    // the tile at `base`, of whose 64 steps `k` are left
    __device__ __forceinline__ void copy(const bf16* base, const char* lds, int k, int thread) const {
        const uint32_t at = __builtin_amdgcn_readfirstlane(lds_address(lds) + to);
        if (k >= 64) {
            const uint64_t from = uniform_address(base);
#pragma unroll
            for (int i = 0; i < kCopies; ++i) copy16(from, off[i], at + i * 4096);
        } else {
#pragma unroll
            for (int i = 0; i < kCopies; ++i) {
                const bool real = ACROSS ? row_of(i, thread) < k : unit_of(i, thread) * 8 < k;
                copy16_from(real ? reinterpret_cast<const char*>(base) + off[i] : reinterpret_cast<const char*>(kZeros), at + i * 4096);
            }
        }
    }
    // rows (ACROSS: columns) 32 t .. 32 t + 31 as a fragment, step c of 16: lane l has
    // row l % 32 and of the step the eight values from 8 (l / 32)
    static __device__ __forceinline__ bf16x8 read(const char* lds, int t, int c, int lane) {
        if constexpr (!ACROSS) {
            return Ti::rows(lds, 32 * t, c, lane);
        } else {
            const int i = lane & 15, row = 16 * c + 8 * (lane >> 5) + (i >> 2);
            const int unit = 4 * t + 2 * ((lane >> 4) & 1) + ((i & 3) >> 1);
            typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
            const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(lds + Ti::at(row, unit) + 8 * (i & 1)));
            const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(lds + Ti::at(row + 4, unit) + 8 * (i & 1)));
            typedef short s16x8 __attribute__((ext_vector_type(8)));
            return __builtin_bit_cast(bf16x8, s16x8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]});
        }
    }
};

// ------------------------------------------------------------------ the product
enum Out { kGated, kStore, kPartial };

// WM x 4/WM waves of 32 MT rows and in each half 16 NT columns.
template <int MT, int NT, int WM, bool AC, bool BC, Out OUT, typename TO>
__global__ __launch_bounds__(256) void k_product(const Product p) {
    constexpr int WN = 4 / WM, BM = 32 * MT * WM, HT = NT / 2, HN = 32 * HT * WN;
    using A = std::conditional_t<AC, Operand<64, BM / 8, true>, Operand<BM, 8, false>>;
    using B = std::conditional_t<BC, Operand<64, HN / 8, true>, Operand<HN, 8, false>>;
    constexpr int kBuffer = A::kBytes + 2 * B::kBytes;
    __shared__ __attribute__((aligned(256))) char lds[2 * kBuffer];
    const int thread = threadIdx.x, lane = thread & 63, wave = __builtin_amdgcn_readfirstlane(thread >> 6);
    const int wm = wave / WN, wn = wave % WN;
    // the block's tile: neighbours on a die share rows of a and columns of b
    const int per = p.tiles_m * p.tiles_n;
    int id = near_blocks(blockIdx.x, per * p.groups * p.splits);
    const int z = id / (per * p.groups);
    id -= z * per * p.groups;
    const int group = id / per;
    id -= group * per;
    constexpr int kStrip = 4;
    const int strip = id / (kStrip * p.tiles_n), in = id - strip * kStrip * p.tiles_n;
    const int high = min(kStrip, p.tiles_m - strip * kStrip);
    const int m0 = (strip * kStrip + in % high) * BM, tn = in / high;
    const int n0 = tn * (p.apart ? HN : 2 * HN);                 // first column of the first half
    const int n1 = p.apart ? n0 : n0 + HN;
    // steps of this split
    const int all = p.segs * p.steps, first = (int)((int64_t)all * z / p.splits), last = (int)((int64_t)all * (z + 1) / p.splits);
    A a;
    B b0, b1;
    a.plan(p.lda, p.m - m0, thread);
    b0.plan(p.ldb, p.n - n0, thread);
    const bool two = n1 < p.n;                                   // (else the second half repeats the first)
    b1.plan(p.ldb, two ? p.n - n1 : p.n - n0, thread);
    const auto fill = [&](int t, char* to) {
        const int s = t / p.steps, k0 = (t - s * p.steps) * 64, k = p.k - k0;
        a.copy(p.a[s] + group * p.a_group + (AC ? (int64_t)k0 * p.lda + m0 : (int64_t)m0 * p.lda + k0), to, k, thread);
        b0.copy(p.b0[s] + (BC ? (int64_t)k0 * p.ldb + n0 : (int64_t)n0 * p.ldb + k0), to + A::kBytes, k, thread);
        const int n = two ? n1 : n0;
        b1.copy(p.b1[s] + (BC ? (int64_t)k0 * p.ldb + n : (int64_t)n * p.ldb + k0), to + A::kBytes + B::kBytes, k, thread);
    };
    f32x16 acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = f32x16{};
    if (first < last) fill(first, lds);
    wait_copies();
    lds_barrier();
    for (int t = first; t < last; ++t) {
        const char* now = lds + ((t - first) & 1) * kBuffer;
        if (t + 1 < last) fill(t + 1, lds + ((t - first + 1) & 1) * kBuffer);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            bf16x8 fa[MT], fb[NT];
#pragma unroll
            for (int i = 0; i < MT; ++i) fa[i] = A::read(now, wm * MT + i, c, lane);
#pragma unroll
            for (int j = 0; j < NT; ++j) fb[j] = B::read(now + A::kBytes + (j / HT) * B::kBytes, wn * HT + j % HT, c, lane);
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j) acc[i][j] = mma(fa[i], fb[j], acc[i][j]);
        }
        wait_copies();
        lds_barrier();
    }
    // results, 32 rows of the wave at a time through LDS, so that a lane has eight neighbours
    // of a row (in a product's result it has one column)
    constexpr int kCols = 32 * HT, kPitch = 2 * kCols + 4;       // floats: both halves, and 4 against bank conflicts
    static_assert(4 * 32 * kPitch * 4 <= 2 * kBuffer, "four waves' rows fit");
    float* stage = reinterpret_cast<float*>(lds) + wave * 32 * kPitch;
    const int unit = lane % (kCols / 8), sub = lane / (kCols / 8);
    const int at0 = n0 + wn * kCols + 8 * unit, at1 = n1 + wn * kCols + 8 * unit;
    const int left0 = p.n - at0, left1 = p.n - at1;
#pragma unroll
    for (int i = 0; i < MT; ++i) {
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) stage[tile_row(lane, r) * kPitch + 32 * j + (lane & 31)] = acc[i][j][r];
#pragma unroll 1
        for (int r0 = sub; r0 < 32; r0 += 64 / (kCols / 8)) {
            const int64_t row = m0 + (wm * MT + i) * 32 + r0;
            if (row >= p.m) break;
            const f32x4* from = reinterpret_cast<const f32x4*>(stage + r0 * kPitch + 8 * unit);
            const f32x4 g0 = from[0], g1 = from[1], u0 = from[kCols / 4], u1 = from[kCols / 4 + 1];
            const f32x8 v0 = {g0[0], g0[1], g0[2], g0[3], g1[0], g1[1], g1[2], g1[3]};
            const f32x8 v1 = {u0[0], u0[1], u0[2], u0[3], u1[0], u1[1], u1[2], u1[3]};
            if constexpr (OUT == kGated) {
                if (left0 <= 0) break;
                f32x8 h;
#pragma unroll
                for (int e = 0; e < 8; ++e) h[e] = activate(p.act, v0[e]) * v1[e];
                store8(static_cast<TO*>(p.c[0]) + row * p.ldc[0] + at0, left0, narrow<TO>(h));
                if (p.gate) store8(static_cast<TO*>(p.gate) + row * p.ld_gate + at0, left0, narrow<TO>(v0));
                if (p.up) store8(static_cast<TO*>(p.up) + row * p.ld_up + at0, left0, narrow<TO>(v1));
            } else {
                const int h0 = p.apart ? 0 : group, h1 = p.apart ? 1 : group;
                TO *to0, *to1;
                if constexpr (OUT == kStore) {
                    to0 = static_cast<TO*>(p.c[h0]) + row * p.ldc[h0];
                    to1 = static_cast<TO*>(p.c[h1]) + row * p.ldc[h1];
                } else {
                    const int64_t size = (int64_t)p.m * p.n, count = p.apart ? 2 : p.groups;
                    to0 = p.partial + (z * count + h0) * size + row * p.n;
                    to1 = p.partial + (z * count + h1) * size + row * p.n;
                }
                if (left0 > 0) store8(to0 + at0, left0, narrow<TO>(v0));
                if (left1 > 0) store8(to1 + at1, left1, narrow<TO>(v1));
            }
        }
    }
}

// The splits' sums together, in their order, and what comes after them.
template <bool GATED, typename TO>
__global__ __launch_bounds__(256) void k_product_join(const Product p) {
    const int64_t size = (int64_t)p.m * p.n, each = (p.apart ? 2 : p.groups) * size;
    const int64_t count = GATED ? size : each;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < count; i += (int64_t)gridDim.x * 256) {
        const int64_t matrix = i / size, in = i - matrix * size, row = in / p.n;
        const int n = (int)(in - row * p.n);
        float v0 = 0.f, v1 = 0.f;
        for (int z = 0; z < p.splits; ++z) {
            v0 += p.partial[z * each + i];
            if (GATED) v1 += p.partial[z * each + size + i];
        }
        if constexpr (GATED) {
            static_cast<TO*>(p.c[0])[row * p.ldc[0] + n] = (TO)(activate(p.act, v0) * v1);
            if (p.gate) static_cast<TO*>(p.gate)[row * p.ld_gate + n] = (TO)v0;
            if (p.up) static_cast<TO*>(p.up)[row * p.ld_up + n] = (TO)v1;
        } else {
            static_cast<TO*>(p.c[matrix])[row * p.ldc[matrix] + n] = (TO)v0;
        }
    }
}

// ------------------------------------------------------------------ layouts
// A float32 in three parts, as split() makes them, but that values past the largest bfloat16
// (3.39e38) keep a finite first part.
constexpr float kMostBf16 = 3.38953139e38f;
__device__ inline Split split_any(f32x8 x) {
    f32x8 y;
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = fminf(fmaxf(x[e], -kMostBf16), kMostBf16);
    Split s;
    s.h = narrow<bf16>(y);
    const f32x8 r = x - widen(s.h);          // (NaN stays in it)
    s.m = narrow<bf16>(r);
    s.l = narrow<bf16>(r - widen(s.m));
    return s;
}
// [rows][cols] as bfloat16 [rows][pitch], zeros past cols; float32: three parts, each a
// matrix.
template <typename T>
__device__ inline void store_parts(bf16* to, int64_t plane, f32x8 v) {
    if constexpr (sizeof(T) == 2) {
        *reinterpret_cast<bf16x8*>(to) = narrow<bf16>(v);
    } else {
        const Split s = split_any(v);
        *reinterpret_cast<bf16x8*>(to) = s.h;
        *reinterpret_cast<bf16x8*>(to + plane) = s.m;
        *reinterpret_cast<bf16x8*>(to + 2 * plane) = s.l;
    }
}
template <typename T>
__global__ __launch_bounds__(256) void k_lay_out(const T* from, int64_t stride, int64_t rows, int cols, int pitch, bf16* to) {
    const int64_t units = rows * (pitch / 8);
    for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < units; u += (int64_t)gridDim.x * 256) {
        const int64_t row = u / (pitch / 8);
        const int c = (int)(u - row * (pitch / 8)) * 8;
        f32x8 v = {};
        if (c < cols) v = widen(load8(from + row * stride + c, cols - c));
        store_parts<T>(to + row * pitch + c, rows * pitch, v);
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
template <typename T>
__global__ __launch_bounds__(256) void k_gated_slopes(const SlopeArgs a) {
    const int64_t units = a.rows * (a.pitch / 8);
    for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < units; u += (int64_t)gridDim.x * 256) {
        const int64_t row = u / (a.pitch / 8);
        const int c = (int)(u - row * (a.pitch / 8)) * 8, n = a.cols - c;
        f32x8 dg = {}, du = {}, h = {};
        if (n > 0) {
            const f32x8 g = widen(load8(static_cast<const T*>(a.gate) + row * a.ld_gate + c, n));
            const f32x8 up = widen(load8(static_cast<const T*>(a.up) + row * a.ld_up + c, n));
            const f32x8 dh = widen(load8(static_cast<const T*>(a.dh) + row * a.ld_dh + c, n));
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (e >= n) continue;
                float act, slope;
                activate_grad(a.act, g[e], act, slope);
                dg[e] = dh[e] * up[e] * slope;
                du[e] = dh[e] * act;
                h[e] = act * up[e];
            }
            if (a.h) store8(static_cast<T*>(a.h) + row * a.ld_h + c, n, narrow<T>(h));
        }
        if (!a.dg) continue;
        bf16* to = a.dg + row * a.pitch + c;
        store_parts<T>(to, a.rows * a.pitch, dg);
        store_parts<T>(to + a.du, a.rows * a.pitch, du);
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
int parts_of(int dtype) { return dtype == PD_F32 ? 3 : 1; }
int64_t layout_bytes(int dtype, int64_t rows, int64_t cols) { return rows * up_to(cols, 64) * 2 * parts_of(dtype); }
// Copies of 16 bytes read the matrix as it lies.
bool as_it_lies(int dtype, const void* p, int64_t stride, int64_t rows, int64_t cols) {
    return dtype == PD_BF16 && (uintptr_t)p % 16 == 0 && cols % 8 == 0 && (rows == 1 || (stride % 8 == 0 && stride < (1 << 22)));
}
Matrix laid_out(int dtype, const void* p, int64_t stride, int64_t rows, int64_t cols, char* to, hipStream_t s, bool lies) {
    if (lies) return Matrix{{static_cast<const bf16*>(p)}, rows == 1 ? cols : stride};
    const int64_t pitch = up_to(cols, 64);
    bf16* q = reinterpret_cast<bf16*>(to);
    const dim3 grid(blocks_for(rows * pitch / 8)), block(256);
    if (dtype == PD_F32)
        hipLaunchKernelGGL(k_lay_out<float>, grid, block, 0, s, static_cast<const float*>(p), stride, rows, (int)cols, (int)pitch, q);
    else
        hipLaunchKernelGGL(k_lay_out<bf16>, grid, block, 0, s, static_cast<const bf16*>(p), stride, rows, (int)cols, (int)pitch, q);
    PD_HIP(hipGetLastError());
    return Matrix{{q, q + rows * pitch, q + 2 * rows * pitch}, pitch};
}
// Appends the segments of a times (b0, b1) to p.
void add_segments(Product& p, int dtype, const Matrix& a, const Matrix& b0, const Matrix& b1) {
    static const int pa[6] = {2, 0, 1, 1, 0, 0}, pb[6] = {0, 2, 1, 0, 1, 0};
    for (int i = dtype == PD_F32 ? 0 : 5; i < 6; ++i) {
        p.a[p.segs] = a.part[pa[i]];
        p.b0[p.segs] = b0.part[pb[i]];
        p.b1[p.segs] = b1.part[pb[i]];
        ++p.segs;
    }
    p.lda = a.ld;
    p.ldb = b0.ld;
}

// How a product is cut: the block's shape, and into how many sums.
enum Shape { kLarge, kSmall, kFew };
struct Cut {
    Shape shape;
    int tiles_m, tiles_n, splits;
};
Cut cut(int64_t m, int64_t n, bool apart, int groups, int64_t steps, bool across) {
    static const int bm[3] = {256, 128, 32}, hn[3] = {128, 64, 128};
    Cut c{};
    const auto tiles = [&](Shape s) {
        c.shape = s;
        c.tiles_m = (int)((m + bm[s] - 1) / bm[s]);
        const int wide = apart ? hn[s] : 2 * hn[s];
        c.tiles_n = (int)((n + wide - 1) / wide);
        return (int64_t)c.tiles_m * c.tiles_n * groups;
    };
    int64_t count;
    if (m <= 32 && !across) count = tiles(kFew);        // (`across`: a runs across the sum)
    else if ((count = tiles(kLarge)) < kCus) count = tiles(kSmall);
    c.splits = 1;
    while (count * c.splits * 2 <= 2 * kCus && steps / (c.splits * 2) >= 4) c.splits *= 2;
    return c;
}
int64_t partial_bytes(const Cut& c, int64_t m, int64_t n, bool apart, int groups) {
    return c.splits == 1 ? 0 : (int64_t)c.splits * groups * (apart ? 2 : 1) * m * n * 4;
}

template <bool AC, bool BC, Out OUT, typename TO>
void launch_shape(const Product& p, Shape shape, hipStream_t s) {
    const dim3 grid((unsigned)(p.tiles_m * p.tiles_n * p.groups * p.splits)), block(256);
    if (shape == kLarge)
        hipLaunchKernelGGL((k_product<4, 4, 2, AC, BC, OUT, TO>), grid, block, 0, s, p);
    else if (shape == kSmall)
        hipLaunchKernelGGL((k_product<2, 2, 2, AC, BC, OUT, TO>), grid, block, 0, s, p);
    else if constexpr (!AC)
        hipLaunchKernelGGL((k_product<1, 2, 1, AC, BC, OUT, TO>), grid, block, 0, s, p);
    PD_HIP(hipGetLastError());
}
template <bool AC, bool BC, bool GATED, typename TO>
void launch_product(Product& p, float* partial, hipStream_t s) {
    p.steps = (p.k + 63) / 64;
    const Cut c = cut(p.m, p.n, p.apart, p.groups, (int64_t)p.steps * p.segs, AC);
    p.tiles_m = c.tiles_m, p.tiles_n = c.tiles_n, p.splits = c.splits;
    p.partial = partial;
    if (c.splits == 1) return launch_shape<AC, BC, GATED ? kGated : kStore, TO>(p, c.shape, s);
    launch_shape<AC, BC, kPartial, float>(p, c.shape, s);
    hipLaunchKernelGGL((k_product_join<GATED, TO>), dim3(blocks_for((int64_t)p.m * p.n * (GATED || !p.apart ? 1 : 2) * p.groups)),
                       dim3(256), 0, s, p);
    PD_HIP(hipGetLastError());
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
    const int64_t segs = d.dtype == PD_F32 ? 6 : 1;
    l.x = take(layout_bytes(d.dtype, d.rows, d.width));
    l.w = take(2 * (in_out ? layout_bytes(d.dtype, d.width, d.hidden) : layout_bytes(d.dtype, d.hidden, d.width)));
    int64_t partial = 0;
    const auto more = [&](int64_t m, int64_t n, bool apart, int groups, int64_t k, int64_t s, bool across) {
        const int64_t b = partial_bytes(cut(m, n, apart, groups, (k + 63) / 64 * s, across), m, n, apart, groups);
        partial = b > partial ? b : partial;
    };
    if (!backward) {
        more(d.rows, d.hidden, true, 1, d.width, segs, false);
    } else {
        l.slopes = take(2 * layout_bytes(d.dtype, d.rows, d.hidden));
        more(d.rows, d.width, false, 1, d.hidden, 2 * segs, false);
        if (in_out) more(d.width, d.hidden, true, 1, d.rows, segs, true);
        else more(d.hidden, d.width, false, 2, d.rows, segs, true);
    }
    l.partial = take(partial);
    l.total = at;
    return l;
}

Matrix inputs(const GatedArgs& a, const Layout& l, hipStream_t s) {
    const pd_gated_desc& d = a.d;
    return laid_out(d.dtype, a.x, d.x_stride, d.rows, d.width, a.scratch + l.x, s,
                    as_it_lies(d.dtype, a.x, d.x_stride, d.rows, d.width));
}
// Both weights lie alike, as the kernel has one distance of rows for them.
void weights(const GatedArgs& a, const Layout& l, Matrix& gate, Matrix& up, hipStream_t s) {
    const pd_gated_desc& d = a.d;
    const bool in_out = d.weight_layout == PD_WEIGHTS_IN_OUT;
    const int64_t rows = in_out ? d.width : d.hidden, cols = in_out ? d.hidden : d.width;
    const bool lie = as_it_lies(d.dtype, a.w_gate, d.w_gate_stride, rows, cols) &&
                     as_it_lies(d.dtype, a.w_up, d.w_up_stride, rows, cols) && (rows == 1 || d.w_gate_stride == d.w_up_stride);
    gate = laid_out(d.dtype, a.w_gate, d.w_gate_stride, rows, cols, a.scratch + l.w, s, lie);
    up = laid_out(d.dtype, a.w_up, d.w_up_stride, rows, cols, a.scratch + l.w + layout_bytes(d.dtype, rows, cols), s, lie);
}

template <typename T>
void gated_t(const GatedArgs& a, hipStream_t s) {
    const pd_gated_desc& d = a.d;
    const Layout l = layout(d, false);
    const Matrix x = inputs(a, l, s);
    Matrix wg, wu;
    weights(a, l, wg, wu, s);
    Product p{};
    add_segments(p, d.dtype, x, wg, wu);
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
    g.du = parts_of(d.dtype) * plane;
    hipLaunchKernelGGL(k_gated_slopes<T>, dim3(blocks_for(d.rows * pitch / 8)), dim3(256), 0, s, g);
    PD_HIP(hipGetLastError());
    const Matrix dg{{g.dg, g.dg + plane, g.dg + 2 * plane}, pitch}, du{{g.dg + g.du, g.dg + g.du + plane, g.dg + g.du + 2 * plane}, pitch};
    float* partial = reinterpret_cast<float*>(a.scratch + l.partial);
    if (a.dx) {
        Matrix wg, wu;
        weights(a, l, wg, wu, s);
        Product p{};
        add_segments(p, d.dtype, dg, wg, wg);
        add_segments(p, d.dtype, du, wu, wu);
        p.k = d.hidden, p.m = (int)d.rows, p.n = d.width;
        p.apart = 0, p.groups = 1;
        p.c[0] = a.dx, p.ldc[0] = d.dx_stride;
        if (in_out) launch_product<false, false, false, T>(p, partial, s);
        else launch_product<false, true, false, T>(p, partial, s);
    }
    if (a.dw_gate) {
        const Matrix x = inputs(a, l, s);
        Product p{};
        if (in_out) {
            add_segments(p, d.dtype, x, dg, du);
            p.m = d.width, p.n = d.hidden;
            p.apart = 1, p.groups = 1;
        } else {
            add_segments(p, d.dtype, dg, x, x);
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

int64_t gated_scratch_bytes(const pd_gated_desc& d) { return d.rows ? layout(d, false).total : 0; }
void launch_gated(const GatedArgs& a, hipStream_t s) { a.d.dtype == PD_F32 ? gated_t<float>(a, s) : gated_t<bf16>(a, s); }
int64_t gated_grad_scratch_bytes(const pd_gated_desc& d) { return d.rows ? layout(d, true).total : 0; }
void launch_gated_grad(const GatedArgs& a, hipStream_t s) { a.d.dtype == PD_F32 ? gated_grad_t<float>(a, s) : gated_grad_t<bf16>(a, s); }

}  // namespace pd
