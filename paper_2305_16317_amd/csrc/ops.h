// Shared by the transformer operators (norm.hip, rotary.hip, attention.hip,
// attention_grad.hip) and their C entry points (operators.cpp).
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

struct RotaryArgs {
    pd_rotary_desc d;
    const void* q;
    const void* k;
    const int32_t* positions;
    const float* table;
    void* q_out;
    void* k_out;
};
void launch_rotary(const RotaryArgs& a, hipStream_t s);
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

}  // namespace pd
