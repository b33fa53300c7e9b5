// C entry points of the transformer-block operators (vd_block.h): argument checks, then the launch.
#include <math.h>
#include <stdio.h>

#include "block_ops.h"

using namespace vd;

namespace {

vd_status refuse(vd_status s, const char* msg) {
    set_last_error(msg);
    return s;
}
vd_status done(cudaError_t e, const char* what) {
    if (e == cudaSuccess) return VD_OK;
    char msg[200];
    snprintf(msg, sizeof(msg), "%s: %s", what, cudaGetErrorString(e));
    set_last_error(msg);
    return VD_ERR_CUDA;
}
bool is_dtype(int d) { return d == VD_F32 || d == VD_BF16; }
bool aligned_to(const void* p, int dtype) { return ((uintptr_t)p & (dtype == VD_BF16 ? 1u : 3u)) == 0; }
bool fits(int64_t a, int64_t b, int64_t c) { return a == 0 || b == 0 || c == 0 || (a <= INT32_MAX / b && a * b <= INT32_MAX / c); }
// no element of an output lies on another one: each stride beyond the extent of the smaller ones
bool distinct(int64_t n0, int64_t s0, int64_t n1, int64_t s1, int64_t n2, int64_t s2, int64_t width) {
    struct { int64_t n, s; } d[3] = {{n0, s0}, {n1, s1}, {n2, s2}};
    for (int i = 0; i < 2; ++i)
        for (int j = 0; j < 2 - i; ++j)
            if (d[j].s > d[j + 1].s) { const auto t = d[j]; d[j] = d[j + 1]; d[j + 1] = t; }
    int64_t extent = width;
    for (const auto& e : d) {
        if (e.n <= 1) continue;
        if (e.s < extent || e.s > INT64_MAX / e.n / 2 - extent) return false;
        extent += (e.n - 1) * e.s;
    }
    return true;
}
bool not_negative(const int64_t* s, int n) {
    for (int i = 0; i < n; ++i)
        if (s[i] < 0) return false;
    return true;
}

const char* xattn_error(const vd_xattn_desc* d) {
    if (!d) return "NULL descriptor";
    if (d->struct_size != sizeof(vd_xattn_desc)) return "vd_xattn_desc: struct_size mismatch";
    if (!is_dtype(d->dtype)) return "bad dtype";
    if (d->batch < 0 || d->q_len < 0 || d->kv_len < 0 || d->heads < 1 || d->kv_heads < 1 || d->heads % d->kv_heads != 0 ||
        d->head_dim < 1 || d->head_dim > 256 || d->kv_len > 1 << 25 || !fits(d->batch, d->heads, d->q_len) ||
        (int64_t)d->batch * d->heads * d->q_len > 1 << 30)
        return "bad attention sizes";
    if (d->impl < VD_XATTN_AUTO || d->impl > VD_XATTN_PLAIN) return "bad impl";
    if (!(d->scale > 0.f && d->scale <= 8.5070592e37f)) return "scale must be positive, at most 2^126";     // (times log2 e it is still finite)
    if (!not_negative(&d->q_batch, 12)) return "negative stride";
    return nullptr;
}
XAttnArgs xattn_args(const vd_xattn_desc* d, const void* q, const void* k, const void* v, const int32_t* kv_lens, void* o) {
    return {q, k, v, o, kv_lens, d->dtype, d->batch, d->q_len, d->kv_len, d->heads, d->kv_heads, d->head_dim,
            {d->q_batch, d->q_token, d->q_head}, {d->k_batch, d->k_token, d->k_head}, {d->v_batch, d->v_token, d->v_head},
            {d->o_batch, d->o_token, d->o_head}, d->scale};
}
// the kernel that takes a call
auto kernel_of(const XAttnArgs& a) -> cudaError_t (*)(const XAttnArgs&, cudaStream_t) {
    const int64_t rows = (int64_t)a.Tq * (a.H / a.Hkv);       // of a key head
    // fp32, four rows of a key head at a time, against tiles of 128 rows (64 beyond 80 channels), us: 256 x 1500 of 64, 32 rows 201 / 342, 64 rows 384 / 344; of 80,
    // 32 rows 359 / 436; of 128, 16 rows 210 / 342, 32 rows 361 / 342; 256 x 50 of 128, 16 rows 18.7 / 20.8, 24 rows 25.2 / 20.9.
    const int few = a.dtype == VD_BF16 ? 16 : a.D <= 80 ? 32 : 16;
    // A few rows with a short context: streaming has not begun when it ends, and tiles mostly empty cost less (us, rows kernel / tiles: 1024 x 50, 8 rows of
    // 64 29 / 15; 32 x 100, 8 rows of 128 8.5 / 8.5; 32 x 300, 16 rows of 128 14.7 / 10.6; 256 x 300, 8 rows of 64 12.6 / 14.7; 32 x 1000, 16 rows of 64
    // 10.6 / 16.5).  With 9 to 16 rows of more than 64 channels in every SM the products bound the rows kernel (256 x 1000 of 128 38.6 / 35.1, of
    // 256 72 / 53; x 4000 of 128 90 / 102).
    const bool tiles = a.dtype == VD_BF16 && rows > 4 && (a.Tk <= 128 || (rows > 8 && (a.Tk <= 512 || (a.D > 64 && a.Tk <= 2048 && (int64_t)a.B * a.Hkv >= 148))));
    if (rows <= few && xattn_rows_supported(a) && !(tiles && xattn_tc_supported(a))) return launch_xattn_rows;
    return a.dtype == VD_BF16 && xattn_tc_supported(a) ? launch_xattn_tc : launch_xattn_f32;
}

}  // namespace

extern "C" {

vd_status vd_op_cross_attention(const vd_xattn_desc* d, const void* q, const void* k, const void* v, const int32_t* kv_lens, void* o,
                                void* cuda_stream) {
    if (const char* e = xattn_error(d)) return refuse(VD_ERR_INVALID_ARG, e);
    if (d->batch == 0 || d->q_len == 0) return VD_OK;
    if (!distinct(d->batch, d->o_batch, d->q_len, d->o_token, d->heads, d->o_head, d->head_dim))
        return refuse(VD_ERR_INVALID_ARG, "elements of the output overlap");
    if (!q || !o || (d->kv_len > 0 && (!k || !v))) return refuse(VD_ERR_INVALID_ARG, "NULL pointer");
    if (!aligned_to(q, d->dtype) || !aligned_to(k, d->dtype) || !aligned_to(v, d->dtype) || !aligned_to(o, d->dtype) || ((uintptr_t)kv_lens & 3))
        return refuse(VD_ERR_INVALID_ARG, "misaligned pointer");
    if (o == q || o == k || o == v) return refuse(VD_ERR_INVALID_ARG, "o is an input");
    const XAttnArgs a = xattn_args(d, q, k, v, kv_lens, o);
    const auto launch = d->impl == VD_XATTN_PLAIN ? launch_xattn_plain : kernel_of(a);
    return done(launch(a, (cudaStream_t)cuda_stream), "vd_op_cross_attention");
}

vd_status vd_debug_xattn_division(const vd_xattn_desc* d, int32_t* splits, int64_t* items, int64_t* whole, int64_t* blocks) {
    if (const char* e = xattn_error(d)) return refuse(VD_ERR_INVALID_ARG, e);
    if (!splits || !items || !whole || !blocks) return refuse(VD_ERR_INVALID_ARG, "NULL pointer");
    const uintptr_t at = 4096;
    const XAttnArgs a = xattn_args(d, (void*)at, (void*)at, (void*)at, nullptr, (void*)at);
    if (d->batch == 0 || d->q_len == 0 || d->impl != VD_XATTN_AUTO || kernel_of(a) != launch_xattn_tc)
        return refuse(VD_ERR_UNSUPPORTED, "another kernel takes this call");
    XAttnDivision div;
    const cudaError_t e = xattn_tc_division(a, &div);
    if (e != cudaSuccess) return done(e, "vd_debug_xattn_division");
    *splits = div.splits;
    *items = div.items;
    *whole = div.whole;
    *blocks = div.grid;
    return VD_OK;
}

vd_status vd_debug_xattn_meeting_limit(int64_t cycles) {
    xattn_tc_meeting_limit(cycles);
    return VD_OK;
}

static const char* rotary_axes_error(int rotary_dim, int axes, const int32_t* pairs) {
    if (rotary_dim < 0 || rotary_dim % 2 != 0) return "rotary_dim must be even";
    if (axes < 1 || axes > VD_ROTARY_MAX_AXES) return "bad number of axes";
    int64_t sum = 0;
    for (int i = 0; i < axes; ++i) {
        if (pairs[i] < 0) return "negative axis_pairs";
        sum += pairs[i];
    }
    return sum == rotary_dim / 2 ? nullptr : "axis_pairs do not add up to rotary_dim / 2";
}

vd_status vd_rotary_frequencies(const vd_rotary_freq_desc* d, double* freqs) {
    if (!d || !freqs) return refuse(VD_ERR_INVALID_ARG, "NULL pointer");
    if (d->struct_size != sizeof(vd_rotary_freq_desc)) return refuse(VD_ERR_INVALID_ARG, "vd_rotary_freq_desc: struct_size mismatch");
    if (const char* e = rotary_axes_error(d->rotary_dim, d->axes, d->axis_pairs)) return refuse(VD_ERR_INVALID_ARG, e);
    if (d->scaling < VD_ROTARY_SCALE_NONE || d->scaling > VD_ROTARY_SCALE_PARTS) return refuse(VD_ERR_INVALID_ARG, "bad scaling");
    if (!(d->base > 1.0) || isinf(d->base)) return refuse(VD_ERR_INVALID_ARG, "base must be above 1");
    if (d->scaling != VD_ROTARY_SCALE_NONE && (!(d->factor >= 1.0) || isinf(d->factor))) return refuse(VD_ERR_INVALID_ARG, "factor must be 1 or more");
    if (d->scaling == VD_ROTARY_SCALE_PARTS && (!(d->original_len > 0.0) || !(d->slow >= 0.0) || !(d->fast > d->slow) || isinf(d->fast) || isinf(d->original_len)))
        return refuse(VD_ERR_INVALID_ARG, "by parts: original_len > 0 and fast > slow >= 0");
    const double two_pi = 6.283185307179586476925;
    int at = 0;
    for (int axis = 0; axis < d->axes; ++axis) {
        const int n = d->axis_pairs[axis];
        const double base = d->scaling == VD_ROTARY_SCALE_BASE && n > 1 ? d->base * pow(d->factor, (double)n / (n - 1)) : d->base;
        for (int i = 0; i < n; ++i) {
            double f = pow(base, -(double)i / n) / two_pi;
            if (d->scaling == VD_ROTARY_SCALE_LINEAR) f /= d->factor;
            if (d->scaling == VD_ROTARY_SCALE_PARTS) {
                const double w = fmin(fmax((d->original_len * f - d->slow) / (d->fast - d->slow), 0.0), 1.0);
                f = f * w + f / d->factor * (1.0 - w);
            }
            freqs[at++] = f;
        }
    }
    return VD_OK;
}

vd_status vd_op_rotary(const vd_rotary_desc* d, const void* x, const int32_t* positions, const double* freqs, void* y, void* cuda_stream) {
    if (!d) return refuse(VD_ERR_INVALID_ARG, "NULL descriptor");
    if (d->struct_size != sizeof(vd_rotary_desc)) return refuse(VD_ERR_INVALID_ARG, "vd_rotary_desc: struct_size mismatch");
    if (!is_dtype(d->dtype)) return refuse(VD_ERR_INVALID_ARG, "bad dtype");
    if (d->batch < 0 || d->tokens < 0 || d->heads < 0 || d->heads > 1 << 30 || d->head_dim < 1 || d->head_dim > 1024 || d->rotary_dim > d->head_dim || !fits(d->batch, d->tokens, 1))
        return refuse(VD_ERR_INVALID_ARG, "bad rotary sizes");
    if (const char* e = rotary_axes_error(d->rotary_dim, d->axes, d->axis_pairs)) return refuse(VD_ERR_INVALID_ARG, e);
    if (d->layout != VD_ROTARY_HALF && d->layout != VD_ROTARY_INTERLEAVED) return refuse(VD_ERR_INVALID_ARG, "bad layout");
    if (!isfinite(d->amplitude)) return refuse(VD_ERR_INVALID_ARG, "amplitude must be finite");
    if (!not_negative(&d->x_batch, 8)) return refuse(VD_ERR_INVALID_ARG, "negative stride");
    if (d->batch == 0 || d->tokens == 0 || d->heads == 0) return VD_OK;
    if (!distinct(d->batch, d->y_batch, d->tokens, d->y_token, d->heads, d->y_head, d->head_dim))
        return refuse(VD_ERR_INVALID_ARG, "elements of the output overlap");
    if (!x || !y || (d->rotary_dim > 0 && !freqs)) return refuse(VD_ERR_INVALID_ARG, "NULL pointer");
    if (x == y && (d->x_batch != d->y_batch || d->x_token != d->y_token || d->x_head != d->y_head))
        return refuse(VD_ERR_INVALID_ARG, "in place with other strides");
    if (!positions && d->axes != 1) return refuse(VD_ERR_INVALID_ARG, "several axes need positions");
    if (!positions && (d->first_position < -(int64_t)1 << 40 || d->first_position > (int64_t)1 << 40))
        return refuse(VD_ERR_INVALID_ARG, "first_position beyond 2^40");
    if (!aligned_to(x, d->dtype) || !aligned_to(y, d->dtype) || ((uintptr_t)freqs & 7) || ((uintptr_t)positions & 3))
        return refuse(VD_ERR_INVALID_ARG, "misaligned pointer");
    RotaryArgs a{x, y, positions, freqs, d->dtype, d->batch, d->tokens, d->heads, d->head_dim, d->rotary_dim, d->layout == VD_ROTARY_INTERLEAVED,
                 d->axes, {}, d->amplitude, {d->x_batch, d->x_token, d->x_head}, {d->y_batch, d->y_token, d->y_head},
                 d->pos_batch, d->pos_token, d->first_position};
    int end = 0;
    for (int i = 0; i < VD_ROTARY_MAX_AXES; ++i) a.axis_end[i] = end += i < d->axes ? d->axis_pairs[i] : 0;
    return done(launch_rotary(a, (cudaStream_t)cuda_stream), "vd_op_rotary");
}

vd_status vd_op_gate_norm(const vd_gate_norm_desc* d, const void* x, const void* h, const float* post_weight, const void* gate, void* x_out,
                          const float* weight, const float* bias, const void* scale, const void* shift, void* y, void* cuda_stream) {
    if (!d) return refuse(VD_ERR_INVALID_ARG, "NULL descriptor");
    if (d->struct_size != sizeof(vd_gate_norm_desc)) return refuse(VD_ERR_INVALID_ARG, "vd_gate_norm_desc: struct_size mismatch");
    if (!is_dtype(d->x_dtype) || !is_dtype(d->h_dtype) || !is_dtype(d->y_dtype) || !is_dtype(d->mod_dtype)) return refuse(VD_ERR_INVALID_ARG, "bad dtype");
    if (d->batch < 0 || d->tokens < 0 || d->channels < 1 || d->channels > 16384 || d->mod_tokens < 1 || !fits(d->batch, d->tokens, 1))
        return refuse(VD_ERR_INVALID_ARG, "bad norm sizes");
    if (d->norm != VD_NORM_LAYER && d->norm != VD_NORM_RMS) return refuse(VD_ERR_INVALID_ARG, "bad norm kind");
    if (d->post_norm != 0 && d->post_norm != 1) return refuse(VD_ERR_INVALID_ARG, "post_norm must be 0 or 1");
    if (!(d->eps > 0.f) || isinf(d->eps)) return refuse(VD_ERR_INVALID_ARG, "eps must be positive and finite");
    if (!isfinite(d->residual_scale)) return refuse(VD_ERR_INVALID_ARG, "residual_scale must be finite");
    if (!not_negative(&d->x_batch, 14)) return refuse(VD_ERR_INVALID_ARG, "negative stride");
    if (d->batch == 0 || d->tokens == 0) return VD_OK;
    if (!h && (d->post_norm || post_weight || gate)) return refuse(VD_ERR_INVALID_ARG, "a gate or a norm of h without h");
    if (post_weight && !d->post_norm) return refuse(VD_ERR_INVALID_ARG, "post_weight without post_norm");
    if (!y && (weight || bias || scale || shift)) return refuse(VD_ERR_INVALID_ARG, "a modulated norm without y");
    if (!x_out && !y) return refuse(VD_ERR_INVALID_ARG, "nothing to write");
    if (!x) return refuse(VD_ERR_INVALID_ARG, "NULL pointer");
    if ((x_out && !distinct(d->batch, d->xo_batch, d->tokens, d->xo_token, 1, 0, d->channels)) ||
        (y && !distinct(d->batch, d->y_batch, d->tokens, d->y_token, 1, 0, d->channels)))
        return refuse(VD_ERR_INVALID_ARG, "elements of the output overlap");
    if (x_out && (x_out == h || x_out == y)) return refuse(VD_ERR_INVALID_ARG, "x_out is h or y");
    if (x_out == x && (d->x_batch != d->xo_batch || d->x_token != d->xo_token)) return refuse(VD_ERR_INVALID_ARG, "in place with other strides");
    if (y && (y == x || (y == h && (d->h_batch != d->y_batch || d->h_token != d->y_token || d->h_dtype != d->y_dtype))))
        return refuse(VD_ERR_INVALID_ARG, "y is x, or h with other strides or another type");
    if (!aligned_to(x, d->x_dtype) || !aligned_to(x_out, d->x_dtype) || !aligned_to(h, d->h_dtype) || !aligned_to(y, d->y_dtype) ||
        !aligned_to(gate, d->mod_dtype) || !aligned_to(scale, d->mod_dtype) || !aligned_to(shift, d->mod_dtype) ||
        (((uintptr_t)weight | (uintptr_t)bias | (uintptr_t)post_weight) & 3))
        return refuse(VD_ERR_INVALID_ARG, "misaligned pointer");
    GateNormArgs a{*d, x, h, post_weight, gate, x_out, weight, bias, scale, shift, y};
    return done(launch_gate_norm(a, (cudaStream_t)cuda_stream), "vd_op_gate_norm");
}

}  // extern "C"
