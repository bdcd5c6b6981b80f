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
        pd_rotary_desc d = *desc;
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
        if (d.batch == 0 || d.length == 0) return;
        require(q && positions && table && q_out && (!k || k_out), "NULL device pointer");
        require(d.table_rows >= 1, "table_rows must be >= 1");
        check_apart("q_out", d.q_out_stride, d.batch, d.length, d.heads_q, d.head_dim);
        if (d.heads_k) check_apart("k_out", d.k_out_stride, d.batch, d.length, d.heads_k, d.head_dim);
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
