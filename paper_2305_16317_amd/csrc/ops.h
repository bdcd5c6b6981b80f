// Shared by the transformer operators (norm.hip, layernorm.hip, rotary.hip, dropout.hip,
// gated.hip, attention.hip, attention_grad.hip) and their C entry points (operators.cpp).
#pragma once

#include "pd_internal.h"

namespace pd {

using bf16 = __bf16;

// ---------------------------------------------------------------- eight values
// A lane's unit of memory traffic: eight consecutive elements (16 bytes of
// bfloat16, 32 of float32).  The accesses promise the element's alignment only,
// which the hardware takes for global memory, so any stride and offset runs the
// same code.
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef f32x8 f32x8_u __attribute__((aligned(4)));
typedef bf16x8 bf16x8_u __attribute__((aligned(2)));
template <typename T>
struct Vec8;
template <>
struct Vec8<float> {
    using type = f32x8;
    using unaligned = f32x8_u;
};
template <>
struct Vec8<bf16> {
    using type = bf16x8;
    using unaligned = bf16x8_u;
};

__device__ inline f32x8 widen(f32x8 v) { return v; }
__device__ inline f32x8 widen(bf16x8 v) { return __builtin_convertvector(v, f32x8); }
template <typename T>
__device__ inline typename Vec8<T>::type narrow(f32x8 v) {
    return __builtin_convertvector(v, typename Vec8<T>::type);   // to nearest even
}

// eight elements at p, of which the first n count (the others: 0)
template <typename T>
__device__ inline typename Vec8<T>::type load8(const T* p, int n) {
    if (n >= 8) return *reinterpret_cast<const typename Vec8<T>::unaligned*>(p);
    typename Vec8<T>::type v = {};
#pragma unroll
    for (int e = 0; e < 7; ++e)
        if (e < n) v[e] = p[e];
    return v;
}
template <typename T>
__device__ inline void store8(T* p, int n, typename Vec8<T>::type v) {
    if (n >= 8) {
        *reinterpret_cast<typename Vec8<T>::unaligned*>(p) = v;
        return;
    }
#pragma unroll
    for (int e = 0; e < 7; ++e)
        if (e < n) p[e] = v[e];
}

// ---------------------------------------------------------------- launches
struct NormArgs {
    pd_rmsnorm_desc d;
    const void* x;
    const void* residual;
    const float* weight;
    void* sum;
    void* y;
    float* scale;
    float* rstd;
};
void launch_rmsnorm(const NormArgs& a, hipStream_t s);
struct NormGradArgs {
    pd_rmsnorm_desc d;
    const void* dy;
    const void* sum;
    const float* weight;
    const float* rstd;
    const void* dsum;
    void* dx;
    float* dweight;
    float* partial;      // [norm_grad_blocks][width], or nullptr without dweight
};
int norm_grad_blocks(const pd_rmsnorm_desc& d);
void launch_rmsnorm_grad(const NormGradArgs& a, hipStream_t s);

// Compute units of an MI355X: how much scratch a call needs does not depend on a device.
constexpr int kCus = 256;

struct LayerNormArgs {
    pd_layernorm_desc d;     // (span as the kernels take it: at least 1)
    const void* x;
    const void* residual;
    const float* weight;     // or nullptr: ones
    const float* bias;       // or nullptr: zeros
    void* sum;
    void* y;
    float* mean;
    float* rstd;
    int64_t first;           // row that the launch begins at
};
void launch_layernorm(const LayerNormArgs& a, hipStream_t s);
struct LayerNormGradArgs {
    pd_layernorm_desc d;
    const void* dy;
    const void* sum;
    const float* weight;
    const float* mean;
    const float* rstd;
    const void* dsum;
    void* dx;
    float* dweight;
    float* dbias;
    float* partial;          // [2][groups][parts][width]; not used with one part
    int64_t groups;
    int parts;
};
int layernorm_grad_parts(const pd_layernorm_desc& d);
void launch_layernorm_grad(const LayerNormGradArgs& a, hipStream_t s);

struct DropoutArgs {
    pd_dropout_desc d;
    const void* x;
    const void* residual;
    const uint32_t* step;
    void* y;
    uint32_t under;          // a value is kept where its 16 bits are not under this
    float scale;             // 65536 / (65536 - under)
    int64_t first;           // row that the launch begins at, for the counters
};
void launch_dropout(const DropoutArgs& a, hipStream_t s);

struct RotaryArgs {
    static constexpr bool kAxes = false;
    pd_rotary_desc d;
    const void* q;
    const void* k;
    const int32_t* positions;
    const float* table;
    void* q_out;
    void* k_out;
};
void launch_rotary(const RotaryArgs& a, hipStream_t s);
// the axis of each pair, two bits a pair
struct AxisMap {
    uint32_t word[32];
    __host__ __device__ int axis(int k) const { return (word[k >> 4] >> (2 * (k & 15))) & 3; }
};
struct RotaryAxesArgs {
    static constexpr bool kAxes = true;
    pd_rotary_desc d;
    const void* q;
    const void* k;
    const int32_t* positions;
    const float* table;
    void* q_out;
    void* k_out;
    int64_t position_strides[3];   // batch, token, axis
    AxisMap map;
};
void launch_rotary_axes(const RotaryAxesArgs& a, hipStream_t s);
void launch_rotary_axes_table(const pd_rotary_axes_table_desc& d, const AxisMap& map, int64_t first, int64_t rows, float* table,
                              hipStream_t s);
void launch_rotary_table(const pd_rotary_table_desc& d, int64_t first, int64_t rows, float* table, hipStream_t s);

struct AttentionArgs {
    pd_attention_desc d;
    const void* q;
    const void* k;
    const void* v;
    const int32_t* q_lens;
    const int32_t* kv_lens;
    void* out;
    float* lse;
    // backward
    const void* dout;
    void* dq;
    void* dk;
    void* dv;
    float* scratch;
};
int64_t attention_scratch_bytes(const pd_attention_desc& d);
void launch_attention(const AttentionArgs& a, hipStream_t s);
int64_t attention_grad_scratch_bytes(const pd_attention_desc& d);
void launch_attention_grad(const AttentionArgs& a, hipStream_t s);

struct GatedArgs {
    pd_gated_desc d;
    const void* x;
    const void* w_gate;
    const void* w_up;
    void* gate;              // forward: or nullptr
    void* up;
    void* h;                 // backward: or nullptr
    // backward
    const void* dh;
    void* dx;                // or nullptr
    void* dw_gate;           // or nullptr
    void* dw_up;
    char* scratch;
};
int64_t gated_scratch_bytes(const pd_gated_desc& d);
void launch_gated(const GatedArgs& a, hipStream_t s);
int64_t gated_grad_scratch_bytes(const pd_gated_desc& d);
// How a call's products are cut, four numbers each: the form (256, 192, 128 by 256, 128 by 128, 32 by 256), parts of
// the sum, tiles, blocks at once; returns how many products there are.  For tests, which reach all of them.
int gated_forms(const pd_gated_desc& d, bool backward, int* out);
void launch_gated_grad(const GatedArgs& a, hipStream_t s);

}  // namespace pd
