// C entry points of the transformer operators: argument checks on the host,
// then the launches.  Empty work (no rows, no tokens) is PD_OK with nothing
// launched, but for gradients that are sums over nothing.
#include <algorithm>
#include <cmath>
#include <cstring>

#include "api_guard.h"
#include "ops.h"

using namespace pd;

namespace {

// Every call checks the device it runs on; the answer for a device is kept.
void require_gfx950() {
    static thread_local int known = -1;
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess) fail(PD_ERR_DEVICE, "no HIP device is available");
    if (dev == known) return;
    hipDeviceProp_t prop;
    PD_HIP(hipGetDeviceProperties(&prop, dev));
    if (std::strncmp(prop.gcnArchName, "gfx950", 6) != 0)
        fail(PD_ERR_DEVICE, std::string("this library is built for gfx950, device is ") + prop.gcnArchName);
    known = dev;
}

void check_dtype(int32_t dtype) { require(dtype == PD_F32 || dtype == PD_BF16, "dtype must be PD_F32 or PD_BF16"); }

void check_scratch(const void* scratch, int64_t have, int64_t need) {
    if (need == 0) return;
    require(scratch != nullptr && have >= need, "scratch is smaller than the matching scratch call says");
    require(reinterpret_cast<uintptr_t>(scratch) % 16 == 0, "scratch must be 16-byte aligned");
}

// Rows from 0 to count - 1 at a stride must not reach past 2^62 elements, and not
// overlap where they are written.
constexpr int64_t kMostStride = (int64_t)1 << 40;
void check_stride(int64_t s) { require(s >= 0 && s < kMostStride, "a stride is out of range"); }

// The rows of `row` elements of an output at three strides: none may share an element
// with another.
bool rows_apart(const int64_t* stride, int64_t batch, int64_t tokens, int64_t heads, int64_t row) {
    typedef __int128 wide;                                // (a stride times a count can pass 2^63)
    struct Axis {
        int64_t stride, count;
    } axes[3] = {{stride[0], batch}, {stride[1], tokens}, {stride[2], heads}};
    std::sort(axes, axes + 3, [](const Axis& a, const Axis& b) { return a.stride < b.stride; });
    // usually each step passes what the smaller steps cover
    bool nested = true;
    wide covered = row;
    for (const Axis& x : axes) {
        if (x.count <= 1) continue;
        if (x.stride < row) return false;
        nested = nested && x.stride >= covered;
        covered += (wide)x.stride * (x.count - 1);
    }
    if (nested) return true;
    // else the axes interleave: two rows share an element where some difference of places is
    // under `row`; the longest axis is solved for, the others are gone through
    std::sort(axes, axes + 3, [](const Axis& a, const Axis& b) { return a.count < b.count; });
    const Axis &p = axes[0], &q = axes[1], &l = axes[2];
    for (int64_t i = 0; i < p.count; ++i)
        for (int64_t j = i ? 1 - q.count : 0; j < q.count; ++j) {
            const wide at = (wide)i * p.stride + (wide)j * q.stride;
            const wide back = -at / l.stride;             // (the nearest of the longest axis: this, or one beside it)
            for (wide k = back - 1; k <= back + 1; ++k) {
                if (k <= -(wide)l.count || k >= l.count || (i == 0 && j == 0 && k == 0)) continue;
                const wide off = at + k * l.stride;
                if (off < row && -off < row) return false;
            }
        }
    return true;
}
void check_apart(const char* what, const int64_t* stride, int64_t batch, int64_t tokens, int64_t heads, int64_t row) {
    require(rows_apart(stride, batch, tokens, heads, row), std::string(what) + ": rows of an output share elements");
}

// ------------------------------------------------------------------ norm
void check_norm(const pd_rmsnorm_desc& d, bool backward) {
    check_dtype(d.dtype);
    require(d.rows >= 0 && d.rows <= (int64_t)1 << 31, "rows out of range");
    require(d.width >= 1 && d.width <= 65536, "width must be in [1, 65536]");
    require(d.eps >= 0.f && std::isfinite(d.eps), "eps must be finite and >= 0");
    for (int64_t s : {d.x_stride, d.residual_stride, d.sum_stride, d.y_stride}) check_stride(s);
    if (backward) {
        require(d.out_dtype == d.dtype, "the backward pass takes out_dtype = dtype");
        require(d.rows <= 1 || d.x_stride >= d.width, "x_stride (of dx) must be >= width");
        return;
    }
    require(d.out_dtype == d.dtype || d.out_dtype == PD_F8E4M3, "out_dtype must be dtype or PD_F8E4M3");
    require(d.rows <= 1 || d.y_stride >= d.width, "y_stride must be >= width");
    const int g = d.group;
    require(g == 0 || (g >= 16 && g <= 512 && (g & (g - 1)) == 0), "group must be 0 or a power of two from 16 to 512");
}

// The desc as the kernels take it: runs of at least a row, which divide the rows.
pd_layernorm_desc check_layernorm(const pd_layernorm_desc* p, bool backward) {
    require(p != nullptr, "desc must not be NULL");
    pd_layernorm_desc d = *p;
    check_dtype(d.dtype);
    require(d.rows >= 0 && d.rows <= (int64_t)1 << 31, "rows out of range");
    require(d.width >= 1 && d.width <= 65536, "width must be in [1, 65536]");
    require(d.eps >= 0.f && std::isfinite(d.eps), "eps must be finite and >= 0");
    require(d.span >= 0 && (d.span == 0 || d.rows % d.span == 0), "span must be >= 0 and divide rows");
    for (int64_t s : {d.x_stride, d.residual_stride, d.sum_stride, d.y_stride, d.weight_stride, d.bias_stride}) check_stride(s);
    if (backward) require(d.rows <= 1 || d.x_stride >= d.width, "x_stride (of dx) must be >= width");
    else require(d.rows <= 1 || d.y_stride >= d.width, "y_stride must be >= width");
    if (d.span == 0) {
        d.span = d.rows ? d.rows : 1;
        d.weight_stride = d.bias_stride = 0;
    }
    return d;
}
// runs that have gradients: one of span 0 without rows
int64_t layernorm_groups(const pd_layernorm_desc& given) { return given.span ? given.rows / given.span : 1; }

// ------------------------------------------------------------------ rotary
// What rotary calls have in common, and the desc as the kernels take it.
pd_rotary_desc check_rotary(const pd_rotary_desc& given, const void* k) {
    pd_rotary_desc d = given;
    check_dtype(d.dtype);
    require(d.layout == PD_ROTARY_HALF || d.layout == PD_ROTARY_INTERLEAVED,
            "layout must be PD_ROTARY_HALF or PD_ROTARY_INTERLEAVED");
    require(d.batch >= 0 && d.length >= 0, "batch and length must be >= 0");
    if (!k) d.heads_k = 0;
    require(d.heads_q >= 1 && d.heads_q <= 65536 && d.heads_k >= 0 && d.heads_k <= 65536, "heads out of range");
    require(d.head_dim >= 2 && d.head_dim <= 1024, "head_dim must be in [2, 1024]");
    require(d.rotary_dim >= 2 && d.rotary_dim <= d.head_dim && d.rotary_dim % 2 == 0,
            "rotary_dim must be even and in [2, head_dim]");
    require(d.position_stride >= 0, "position_stride must be >= 0");
    for (int i = 0; i < 3; ++i)
        for (int64_t s : {d.q_stride[i], d.k_stride[i], d.q_out_stride[i], d.k_out_stride[i]}) check_stride(s);
    require(d.batch <= (int64_t)1 << 31 && d.length <= (int64_t)1 << 31, "batch or length out of range");
    // a launch holds fewer than 2^32 threads (at least a unit of 8 values of 8 heads each)
    const int64_t units = d.head_dim / 8 + 2, heads8 = ((int64_t)d.heads_q + d.heads_k + 7) / 8;
    if (d.length && d.batch > ((int64_t)1 << 31) / (units * heads8) / d.length)
        fail(PD_ERR_UNSUPPORTED, "so many tokens in one call are not implemented");
    return d;
}
void check_rotary_memory(const pd_rotary_desc& d, const void* q, const void* k, const int32_t* positions, const float* table,
                         void* q_out, void* k_out) {
    require(q && positions && table && q_out && (!k || k_out), "NULL device pointer");
    require(d.table_rows >= 1, "table_rows must be >= 1");
    check_apart("q_out", d.q_out_stride, d.batch, d.length, d.heads_q, d.head_dim);
    if (d.heads_k) check_apart("k_out", d.k_out_stride, d.batch, d.length, d.heads_k, d.head_dim);
}
// The axis of each pair.
AxisMap axis_map(int axes, int order, const int32_t* sections, int rotary_dim) {
    require(axes >= 1 && axes <= 4, "axes must be in [1, 4]");
    require(order == PD_AXES_RUNS || order == PD_AXES_TURNS, "order must be PD_AXES_RUNS or PD_AXES_TURNS");
    int left[4] = {0, 0, 0, 0};
    int64_t sum = 0;
    for (int a = 0; a < axes; ++a) {
        require(sections[a] >= 0, "sections must be >= 0");
        sum += left[a] = sections[a];
    }
    require(sum == rotary_dim / 2, "sections must add up to rotary_dim / 2");
    AxisMap map{};
    for (int k = 0, a = 0; k < rotary_dim / 2; ++k) {
        while (left[a] == 0) a = (a + 1) % axes;
        map.word[k >> 4] |= (uint32_t)a << (2 * (k & 15));
        --left[a];
        if (order == PD_AXES_TURNS) a = (a + 1) % axes;
    }
    return map;
}

// ------------------------------------------------------------------ gated product
void check_gated(const pd_gated_desc& d) {
    check_dtype(d.dtype);
    require(d.rows >= 0, "rows must be >= 0");
    require(d.width >= 1 && d.width <= 1 << 20 && d.hidden >= 1 && d.hidden <= 1 << 20, "width and hidden must be in [1, 2^20]");
    require(d.activation >= PD_ACT_SILU && d.activation <= PD_ACT_RELU, "activation must be a PD_ACT_* kind");
    require(d.weight_layout == PD_WEIGHTS_IN_OUT || d.weight_layout == PD_WEIGHTS_OUT_IN,
            "weight_layout must be PD_WEIGHTS_IN_OUT or PD_WEIGHTS_OUT_IN");
    for (int64_t s : {d.x_stride, d.w_gate_stride, d.w_up_stride, d.gate_stride, d.up_stride, d.h_stride, d.dh_stride, d.dx_stride,
                      d.dw_gate_stride, d.dw_up_stride})
        check_stride(s);
    if (d.rows > (int64_t)1 << 24) fail(PD_ERR_UNSUPPORTED, "more than 2^24 rows are not implemented");
    // tiles are counted in 32 bits
    const int64_t m = d.rows / 64 + 1, n = d.hidden / 64 + 1, k = d.width / 64 + 1;
    if (m * n > 1 << 28 || m * k > 1 << 28 || n * k > 1 << 28)
        fail(PD_ERR_UNSUPPORTED, "products of more than 2^28 tiles of 64 x 64 are not implemented");
}
void check_alignment(const pd_gated_desc& d, const void* x, const void* w_gate, const void* w_up) {
    if (!d.aligned) return;
    for (const void* p : {x, w_gate, w_up})
        require((uintptr_t)p % 16 == 0, "x, w_gate and w_up do not all begin at multiples of 16 bytes, as aligned says");
}
void check_rows_of(const char* what, const void* p, int64_t stride, int64_t rows, int64_t cols) {
    if (p && rows > 1 && stride < cols) fail(PD_ERR_INVALID_ARG, std::string(what) + ": rows of an output share elements");
}

// ------------------------------------------------------------------ attention
// The desc as the kernels take it: a window that hides nothing becomes 0, and
// sinks count up to the keys there are.
pd_attention_desc check_attention(const pd_attention_desc* p) {
    require(p != nullptr, "desc must not be NULL");
    pd_attention_desc d = *p;
    check_dtype(d.dtype);
    require(d.batch >= 0 && d.heads_q >= 1 && d.heads_kv >= 1, "batch must be >= 0, heads_q and heads_kv >= 1");
    require(d.heads_q % d.heads_kv == 0, "heads_q must be a multiple of heads_kv");
    require(d.head_dim >= 1, "head_dim must be >= 1");
    require(d.q_len >= 0 && d.kv_len >= 0, "q_len and kv_len must be >= 0");
    require(d.window >= 0 && d.sinks >= 0, "window and sinks must be >= 0");
    require(std::isfinite(d.scale), "scale must be finite");
    for (int i = 0; i < 3; ++i)
        for (int64_t s : {d.q_stride[i], d.k_stride[i], d.v_stride[i], d.out_stride[i]}) check_stride(s);
    if (d.head_dim > 128) fail(PD_ERR_UNSUPPORTED, "head_dim above 128 is not implemented");
    const int64_t rows = (int64_t)d.q_len * (d.heads_q / d.heads_kv);
    if (rows > (int64_t)1 << 28 || d.kv_len > 1 << 28)
        fail(PD_ERR_UNSUPPORTED, "more than 2^28 keys, or queries of one key head, are not implemented");
    // a launch holds fewer than 2^32 threads, 512 a block
    const int64_t longest = rows > d.kv_len ? rows : d.kv_len;
    if ((int64_t)d.batch * d.heads_kv > ((int64_t)1 << 22) / (longest / 128 + 1))
        fail(PD_ERR_UNSUPPORTED, "more than 2^22 tiles of 128 queries or keys are not implemented");
    if ((int64_t)d.window >= (int64_t)d.q_len + d.kv_len) d.window = 0;
    if (d.sinks > d.kv_len) d.sinks = d.kv_len;
    if (!d.window) d.sinks = 0;
    return d;
}
void check_attention_grad(const pd_attention_desc& d) {
    for (int i = 0; i < 3; ++i)
        for (int64_t s : {d.dq_stride[i], d.dk_stride[i], d.dv_stride[i], d.dout_stride[i]}) check_stride(s);
}

}  // namespace

extern "C" pd_status pd_rmsnorm_forward(const pd_rmsnorm_desc* desc, const void* x, const void* residual,
                                        const float* weight, void* sum, void* y, float* scale, float* rstd,
                                        void* stream) {
    return guard([&] {
        require(desc != nullptr, "desc must not be NULL");
        check_norm(*desc, false);
        if (desc->rows == 0) return;
        require(x && weight && y, "x, weight and y must not be NULL");
        require(!sum || desc->rows <= 1 || desc->sum_stride >= desc->width, "sum_stride must be >= width");
        require(desc->out_dtype != PD_F8E4M3 || scale, "an output in 8 bits needs scale");
        require_gfx950();
        launch_rmsnorm(NormArgs{*desc, x, residual, weight, sum, y, scale, rstd}, static_cast<hipStream_t>(stream));
    });
}

static int64_t norm_grad_scratch(const pd_rmsnorm_desc& d) {
    return (int64_t)norm_grad_blocks(d) * d.width * (int64_t)sizeof(float);
}

extern "C" pd_status pd_rmsnorm_backward_scratch(const pd_rmsnorm_desc* desc, int64_t* bytes) {
    return guard([&] {
        require(desc != nullptr && bytes != nullptr, "desc and bytes must not be NULL");
        check_norm(*desc, true);
        *bytes = norm_grad_scratch(*desc);
    });
}

extern "C" pd_status pd_rmsnorm_backward(const pd_rmsnorm_desc* desc, const void* dy, const void* sum,
                                         const float* weight, const float* rstd, const void* dsum, void* dx,
                                         float* dweight, void* scratch, int64_t scratch_bytes, void* stream) {
    return guard([&] {
        require(desc != nullptr, "desc must not be NULL");
        check_norm(*desc, true);
        if (desc->rows == 0 && !dweight) return;
        require(weight != nullptr, "weight must not be NULL");
        require(desc->rows == 0 || (dy && sum && rstd && dx), "dy, sum, rstd and dx must not be NULL");
        if (dweight) check_scratch(scratch, scratch_bytes, norm_grad_scratch(*desc));
        require_gfx950();
        launch_rmsnorm_grad(NormGradArgs{*desc, dy, sum, weight, rstd, dsum, dx, dweight, static_cast<float*>(scratch)},
                            static_cast<hipStream_t>(stream));
    });
}

extern "C" pd_status pd_rotary_table(const pd_rotary_table_desc* desc, int64_t first, int64_t rows, float* table,
                                     void* stream) {
    return guard([&] {
        require(desc != nullptr, "desc must not be NULL");
        const pd_rotary_table_desc& d = *desc;
        require(d.rotary_dim >= 2 && d.rotary_dim <= 1024 && d.rotary_dim % 2 == 0, "rotary_dim must be even and in [2, 1024]");
        require(d.scaling >= PD_ROTARY_PLAIN && d.scaling <= PD_ROTARY_BY_PARTS, "scaling must be a PD_ROTARY_* kind");
        require(d.base > 1.0 && std::isfinite(d.base), "base must be finite and > 1");
        require(d.scaling == PD_ROTARY_PLAIN || (d.factor >= 1.0 && std::isfinite(d.factor)), "factor must be finite and >= 1");
        if (d.scaling == PD_ROTARY_BY_PARTS) {
            require(d.original_length > 0.0 && std::isfinite(d.original_length), "original_length must be finite and > 0");
            require(d.turns_low >= 0.0 && d.turns_high > d.turns_low && std::isfinite(d.turns_high),
                    "turns_low and turns_high must be finite with 0 <= low < high");
        }
        require(std::isfinite(d.magnitude), "magnitude must be finite");
        require(first >= 0 && first <= (int64_t)1 << 40 && rows >= 0 && rows <= (int64_t)1 << 28, "first or rows out of range");
        if (rows > ((int64_t)1 << 31) / (d.rotary_dim / 2))
            fail(PD_ERR_UNSUPPORTED, "a table of more than 2^31 pairs is not implemented");
        if (rows == 0) return;
        require(table != nullptr, "table must not be NULL");
        require_gfx950();
        launch_rotary_table(d, first, rows, table, static_cast<hipStream_t>(stream));
    });
}

extern "C" pd_status pd_rotary_apply(const pd_rotary_desc* desc, const void* q, const void* k,
                                     const int32_t* positions, const float* table, void* q_out, void* k_out,
                                     void* stream) {
    return guard([&] {
        require(desc != nullptr, "desc must not be NULL");
        const pd_rotary_desc d = check_rotary(*desc, k);
        if (d.batch == 0 || d.length == 0) return;
        check_rotary_memory(d, q, k, positions, table, q_out, k_out);
        require_gfx950();
        launch_rotary(RotaryArgs{d, q, k, positions, table, q_out, k_out}, static_cast<hipStream_t>(stream));
    });
}

extern "C" pd_status pd_attention_forward_scratch(const pd_attention_desc* desc, int64_t* bytes) {
    return guard([&] {
        require(bytes != nullptr, "bytes must not be NULL");
        *bytes = attention_scratch_bytes(check_attention(desc));
    });
}

extern "C" pd_status pd_attention_forward(const pd_attention_desc* desc, const void* q, const void* k, const void* v,
                                          const int32_t* q_lens, const int32_t* kv_lens, void* out, float* lse,
                                          void* scratch, int64_t scratch_bytes, void* stream) {
    return guard([&] {
        const pd_attention_desc d = check_attention(desc);
        if (d.batch == 0 || d.q_len == 0) return;
        require(q && out && (d.kv_len == 0 || (k && v)), "NULL device pointer");
        check_apart("out", d.out_stride, d.batch, d.q_len, d.heads_q, d.head_dim);
        check_scratch(scratch, scratch_bytes, attention_scratch_bytes(d));
        require_gfx950();
        AttentionArgs a{};
        a.d = d;
        a.q = q, a.k = k, a.v = v;
        a.q_lens = q_lens, a.kv_lens = kv_lens;
        a.out = out, a.lse = lse;
        a.scratch = static_cast<float*>(scratch);
        launch_attention(a, static_cast<hipStream_t>(stream));
    });
}

extern "C" pd_status pd_attention_backward_scratch(const pd_attention_desc* desc, int64_t* bytes) {
    return guard([&] {
        require(bytes != nullptr, "bytes must not be NULL");
        *bytes = attention_grad_scratch_bytes(check_attention(desc));
    });
}

extern "C" pd_status pd_attention_backward(const pd_attention_desc* desc, const void* q, const void* k, const void* v,
                                           const void* out, const float* lse, const void* dout,
                                           const int32_t* q_lens, const int32_t* kv_lens, void* dq, void* dk, void* dv,
                                           void* scratch, int64_t scratch_bytes, void* stream) {
    return guard([&] {
        const pd_attention_desc d = check_attention(desc);
        check_attention_grad(d);
        if (d.batch == 0 || (d.q_len == 0 && d.kv_len == 0)) return;
        require(d.q_len == 0 || (q && out && lse && dout && dq), "NULL device pointer");
        require(d.kv_len == 0 || (k && v && dk && dv), "NULL device pointer");
        check_apart("dq", d.dq_stride, d.batch, d.q_len, d.heads_q, d.head_dim);
        check_apart("dk", d.dk_stride, d.batch, d.kv_len, d.heads_kv, d.head_dim);
        check_apart("dv", d.dv_stride, d.batch, d.kv_len, d.heads_kv, d.head_dim);
        check_scratch(scratch, scratch_bytes, attention_grad_scratch_bytes(d));
        require_gfx950();
        AttentionArgs a{};
        a.d = d;
        a.q = q, a.k = k, a.v = v;
        a.q_lens = q_lens, a.kv_lens = kv_lens;
        a.out = const_cast<void*>(out), a.lse = const_cast<float*>(lse);
        a.dout = dout, a.dq = dq, a.dk = dk, a.dv = dv;
        a.scratch = static_cast<float*>(scratch);
        launch_attention_grad(a, static_cast<hipStream_t>(stream));
    });
}

extern "C" pd_status pd_layernorm_forward(const pd_layernorm_desc* desc, const void* x, const void* residual,
                                          const float* weight, const float* bias, void* sum, void* y, float* mean,
                                          float* rstd, void* stream) {
    return guard([&] {
        const pd_layernorm_desc d = check_layernorm(desc, false);
        if (d.rows == 0) return;
        require(x && y, "x and y must not be NULL");
        require(!sum || d.rows <= 1 || d.sum_stride >= d.width, "sum_stride must be >= width");
        require_gfx950();
        launch_layernorm(LayerNormArgs{d, x, residual, weight, bias, sum, y, mean, rstd, 0}, static_cast<hipStream_t>(stream));
    });
}

static int64_t layernorm_grad_scratch(const pd_layernorm_desc& d, int64_t groups) {
    const int64_t parts = layernorm_grad_parts(d);
    return parts == 1 ? 0 : 2 * groups * parts * d.width * (int64_t)sizeof(float);
}

extern "C" pd_status pd_layernorm_backward_scratch(const pd_layernorm_desc* desc, int64_t* bytes) {
    return guard([&] {
        require(bytes != nullptr, "bytes must not be NULL");
        const pd_layernorm_desc d = check_layernorm(desc, true);
        *bytes = layernorm_grad_scratch(d, layernorm_groups(*desc));
    });
}

extern "C" pd_status pd_layernorm_backward(const pd_layernorm_desc* desc, const void* dy, const void* sum,
                                           const float* weight, const float* mean, const float* rstd, const void* dsum,
                                           void* dx, float* dweight, float* dbias, void* scratch, int64_t scratch_bytes,
                                           void* stream) {
    return guard([&] {
        const pd_layernorm_desc d = check_layernorm(desc, true);
        const int64_t groups = layernorm_groups(*desc);
        if (groups == 0 || (d.rows == 0 && !dweight && !dbias)) return;
        require(d.rows == 0 || (dy && sum && mean && rstd && dx), "dy, sum, mean, rstd and dx must not be NULL");
        if (dweight || dbias) check_scratch(scratch, scratch_bytes, layernorm_grad_scratch(d, groups));
        require_gfx950();
        launch_layernorm_grad(LayerNormGradArgs{d, dy, sum, weight, mean, rstd, dsum, dx, dweight, dbias,
                                                static_cast<float*>(scratch), groups, layernorm_grad_parts(d)},
                              static_cast<hipStream_t>(stream));
    });
}

extern "C" pd_status pd_rotary_axes_table(const pd_rotary_axes_table_desc* desc, int64_t first, int64_t rows, float* table,
                                          void* stream) {
    return guard([&] {
        require(desc != nullptr, "desc must not be NULL");
        const pd_rotary_axes_table_desc& d = *desc;
        require(d.rotary_dim >= 2 && d.rotary_dim <= 1024 && d.rotary_dim % 2 == 0, "rotary_dim must be even and in [2, 1024]");
        const AxisMap map = axis_map(d.axes, d.order, d.sections, d.rotary_dim);
        for (int a = 0; a < d.axes; ++a) {
            require(d.base[a] > 1.0 && std::isfinite(d.base[a]), "base must be finite and > 1");
            require(std::isfinite(d.scale[a]), "scale must be finite");
        }
        require(first >= 0 && first <= (int64_t)1 << 40 && rows >= 0 && rows <= (int64_t)1 << 28, "first or rows out of range");
        if (rows > ((int64_t)1 << 31) / (d.rotary_dim / 2))
            fail(PD_ERR_UNSUPPORTED, "a table of more than 2^31 pairs is not implemented");
        if (rows == 0) return;
        require(table != nullptr, "table must not be NULL");
        require_gfx950();
        launch_rotary_axes_table(d, map, first, rows, table, static_cast<hipStream_t>(stream));
    });
}

extern "C" pd_status pd_rotary_axes_apply(const pd_rotary_axes_desc* desc, const void* q, const void* k,
                                          const int32_t* positions, const float* table, void* q_out, void* k_out,
                                          void* stream) {
    return guard([&] {
        require(desc != nullptr, "desc must not be NULL");
        const pd_rotary_desc d = check_rotary(desc->rotary, k);
        const AxisMap map = axis_map(desc->axes, desc->order, desc->sections, d.rotary_dim);
        for (int64_t s : desc->position_stride) check_stride(s);
        if (d.batch == 0 || d.length == 0) return;
        check_rotary_memory(d, q, k, positions, table, q_out, k_out);
        require_gfx950();
        launch_rotary_axes(RotaryAxesArgs{d, q, k, positions, table, q_out, k_out,
                                          {desc->position_stride[0], desc->position_stride[1], desc->position_stride[2]}, map},
                           static_cast<hipStream_t>(stream));
    });
}

extern "C" pd_status pd_dropout_apply(const pd_dropout_desc* desc, const void* x, const void* residual,
                                      const uint32_t* step_more, void* y, void* stream) {
    return guard([&] {
        require(desc != nullptr, "desc must not be NULL");
        const pd_dropout_desc& d = *desc;
        check_dtype(d.dtype);
        require(d.rows >= 0 && d.rows <= (int64_t)1 << 40 && d.first_row >= 0 && d.first_row <= (int64_t)1 << 40, "rows out of range");
        require(d.width >= 1 && d.width <= 0x7fffffff, "width must be in [1, 2^31 - 1]");
        require(d.rows <= ((int64_t)1 << 46) / d.width, "rows x width out of range");
        require(d.first_row + d.rows <= ((int64_t)1 << 60) / ((d.width + 7) / 8), "first_row out of range");
        require(d.p >= 0.0 && d.p <= 1.0, "p must be in [0, 1]");
        require(step_more || d.step != 0xffffffffu, "step must be below 2^32 - 1");
        for (int64_t s : {d.x_stride, d.residual_stride, d.y_stride}) check_stride(s);
        require(d.rows <= 1 || d.y_stride >= d.width, "y_stride must be >= width");
        if (d.rows == 0) return;
        require(x && y, "x and y must not be NULL");
        require_gfx950();
        DropoutArgs a{};
        a.d = d;
        a.x = x, a.residual = residual, a.step = step_more, a.y = y;
        a.under = (uint32_t)std::floor(65536.0 * d.p + 0.5);
        a.scale = a.under < 65536 ? (float)(65536.0 / (65536.0 - a.under)) : 0.f;
        launch_dropout(a, static_cast<hipStream_t>(stream));
    });
}

extern "C" pd_status pd_gated_forward_scratch(const pd_gated_desc* desc, int64_t* bytes) {
    return guard([&] {
        require(desc != nullptr && bytes != nullptr, "desc and bytes must not be NULL");
        check_gated(*desc);
        *bytes = gated_scratch_bytes(*desc);
    });
}

extern "C" pd_status pd_gated_forward(const pd_gated_desc* desc, const void* x, const void* w_gate, const void* w_up,
                                      void* gate, void* up, void* h, void* scratch, int64_t scratch_bytes, void* stream) {
    return guard([&] {
        require(desc != nullptr, "desc must not be NULL");
        const pd_gated_desc& d = *desc;
        check_gated(d);
        if (d.rows == 0) return;
        require(x && w_gate && w_up && h, "x, w_gate, w_up and h must not be NULL");
        check_alignment(d, x, w_gate, w_up);
        check_rows_of("h", h, d.h_stride, d.rows, d.hidden);
        check_rows_of("gate", gate, d.gate_stride, d.rows, d.hidden);
        check_rows_of("up", up, d.up_stride, d.rows, d.hidden);
        check_scratch(scratch, scratch_bytes, gated_scratch_bytes(d));
        require_gfx950();
        GatedArgs a{};
        a.d = d;
        a.x = x, a.w_gate = w_gate, a.w_up = w_up;
        a.gate = gate, a.up = up, a.h = h;
        a.scratch = static_cast<char*>(scratch);
        launch_gated(a, static_cast<hipStream_t>(stream));
    });
}

extern "C" pd_status pd_gated_backward_scratch(const pd_gated_desc* desc, int64_t* bytes) {
    return guard([&] {
        require(desc != nullptr && bytes != nullptr, "desc and bytes must not be NULL");
        check_gated(*desc);
        *bytes = gated_grad_scratch_bytes(*desc);
    });
}

extern "C" pd_status pd_gated_backward(const pd_gated_desc* desc, const void* x, const void* w_gate, const void* w_up,
                                       const void* gate, const void* up, const void* dh, void* h, void* dx,
                                       void* dw_gate, void* dw_up, void* scratch, int64_t scratch_bytes, void* stream) {
    return guard([&] {
        require(desc != nullptr, "desc must not be NULL");
        const pd_gated_desc& d = *desc;
        check_gated(d);
        require(!dw_gate == !dw_up, "dw_gate and dw_up come together");
        if (d.rows == 0 && !dw_gate) return;
        if (!h && !dx && !dw_gate) return;
        require(d.rows == 0 || (gate && up && dh), "gate, up and dh must not be NULL");
        require(d.rows == 0 || !dx || (w_gate && w_up), "w_gate and w_up must not be NULL");
        require(d.rows == 0 || !dw_gate || x, "x must not be NULL");
        check_alignment(d, x, w_gate, w_up);
        const bool in_out = d.weight_layout == PD_WEIGHTS_IN_OUT;
        check_rows_of("h", h, d.h_stride, d.rows, d.hidden);
        check_rows_of("dx", dx, d.dx_stride, d.rows, d.width);
        check_rows_of("dw_gate", dw_gate, d.dw_gate_stride, in_out ? d.width : d.hidden, in_out ? d.hidden : d.width);
        check_rows_of("dw_up", dw_up, d.dw_up_stride, in_out ? d.width : d.hidden, in_out ? d.hidden : d.width);
        if (dx || dw_gate) check_scratch(scratch, scratch_bytes, gated_grad_scratch_bytes(d));
        require_gfx950();
        GatedArgs a{};
        a.d = d;
        a.x = x, a.w_gate = w_gate, a.w_up = w_up;
        a.gate = const_cast<void*>(gate), a.up = const_cast<void*>(up), a.h = h;
        a.dh = dh, a.dx = dx, a.dw_gate = dw_gate, a.dw_up = dw_up;
        a.scratch = static_cast<char*>(scratch);
        launch_gated_grad(a, static_cast<hipStream_t>(stream));
    });
}
