/*
 * vd_block.h - operators of a latent world model's transformer block.
 *
 * The decoder of vd.h turns latents into frames; the latents come from a transformer over latent patches (Section III-A,
 * Algorithm 1, "DistributedDiT"; Section IV-B, the shift, scale and gate of its modulated norms).  What is declared here
 * are the operators of one of its blocks that are no plain matrix product, as single calls on caller-provided device
 * tensors: a call enqueues kernels on `cuda_stream` and returns; it allocates nothing, keeps nothing, needs no workspace
 * and can be captured into a graph.  Calls on different streams do not touch one another.  The general rules of vd.h
 * apply.  Inference only: there are no gradients.
 *
 * Strides are in elements, between consecutive batch items, tokens and heads; channels lie side by side.  Inputs may
 * be slices of packed tensors and may have stride 0 (one tensor for the whole batch); outputs may be slices, whose
 * elements must all be distinct.  Unless said otherwise an output overlaps no input.
 */
#ifndef VD_BLOCK_H_
#define VD_BLOCK_H_

#include "vd.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ------------------------------------------------------------------------------------------
 * Attention of many heads to states of another length:
 *   o[b,t,h,:] = sum_{u < len[b]} softmax_u(scale * q[b,t,h,:].k[b,u,h/g,:]) v[b,u,h/g,:],   g = heads / kv_heads
 * len = kv_lens clamped to 0..kv_len, or kv_len where kv_lens is NULL.  Keys and values at or behind len are never used,
 * whatever they hold; a row without keys is zeros; one whose scores are all minus infinity, or one of them NaN or plus infinity, is NaN.
 * Sums and the softmax are fp32; VD_BF16 rounds the result to bf16 and may round the probabilities (relative to the row's
 * largest).  Bitwise reproducible.
 * Sums run over the keys in a row, relative to the largest score so far: |v| times the number of keys has to stay within fp32, and
 * what falls off a running sum grows with the keys.  With equal scores, values of 1.3125 throughout and keys that are not divided
 * among blocks (many rows or heads): bf16 exact at 2^20 keys, off by 1 % at 2^22 and 8 % at 2^24; fp32 by 3 % at 2^22.
 * Waits inside the kernels are bounded (a second; where blocks wait for one another longer, by the keys).  None of them ends so unless
 * the device or this library is at fault; the rows of the call that it concerns are then NaN, and there is no status to ask for.
 * ---------------------------------------------------------------------------------------- */
typedef enum {
    VD_XATTN_AUTO = 0,
    VD_XATTN_PLAIN = 1          /* the kernel without restrictions, a warp per row (cross-check path) */
} vd_xattn_impl;

typedef struct {
    uint32_t struct_size;
    int32_t dtype;              /* vd_dtype of q, k, v and o */
    int32_t batch, q_len, kv_len;       /* >= 0; batch * heads * q_len at most 2^30, kv_len at most 2^25 */
    int32_t heads, kv_heads;    /* heads a multiple of kv_heads */
    int32_t head_dim;           /* 1..256 */
    int32_t impl;               /* vd_xattn_impl */
    float scale;                /* > 0, at most 2^126 */
    int64_t q_batch, q_token, q_head;
    int64_t k_batch, k_token, k_head;
    int64_t v_batch, v_token, v_head;
    int64_t o_batch, o_token, o_head;
} vd_xattn_desc;

/* q, k, v, o device (k and v may be NULL where kv_len is 0); kv_lens device int32 [batch] or NULL. */
VD_API vd_status vd_op_cross_attention(const vd_xattn_desc* d, const void* q, const void* k, const void* v,
                                       const int32_t* kv_lens, void* o, void* cuda_stream);

/* Test hooks.
 *   vd_debug_xattn_division       how a bf16 call of the tensor-core kernel (aligned tensors) is shared out on the current device: of its
 *                                 `items` (up to 256 rows of a key head) the first `whole` are a thread block's each, in turn over the `blocks` launched, the
 *                                 others a cluster's of `splits` blocks, which divide the keys.  VD_ERR_UNSUPPORTED where
 *                                 another kernel takes the call.  Launches nothing.
 *   vd_debug_xattn_meeting_limit  SM clocks that blocks of a cluster wait for one another in the calls that follow, process-wide; 0: as many
 *                                 as the call needs (the default); negative: they give up at once, as if the others did not come, and the
 *                                 divided rows are NaN. */
VD_API vd_status vd_debug_xattn_division(const vd_xattn_desc* d, int32_t* splits, int64_t* items, int64_t* whole, int64_t* blocks);
VD_API vd_status vd_debug_xattn_meeting_limit(int64_t cycles);

/* ------------------------------------------------------------------------------------------
 * Rotary positions.  The first rotary_dim channels of a head are rotary_dim / 2 pairs; pair i of a token turns by
 * position[axis of i] * freqs[i]:   (a, b) -> amplitude * (a cos - b sin, a sin + b cos);   the other channels are copied.
 * The first axis_pairs[0] pairs belong to axis 0 (time, say), the next axis_pairs[1] to axis 1 (row), and so on.
 * Angles are formed and reduced in 64 bits, so that far positions keep their angle.
 * ---------------------------------------------------------------------------------------- */
#define VD_ROTARY_MAX_AXES 4
typedef enum {
    VD_ROTARY_HALF = 0,         /* pair i: channels i and i + rotary_dim / 2 */
    VD_ROTARY_INTERLEAVED = 1   /* pair i: channels 2i and 2i + 1 */
} vd_rotary_layout;

typedef struct {
    uint32_t struct_size;
    int32_t dtype;              /* vd_dtype of x and y */
    int32_t batch, tokens, heads;       /* >= 0; batch * tokens < 2^31, heads at most 2^30 */
    int32_t head_dim;           /* 1..1024 */
    int32_t rotary_dim;         /* even, 0..head_dim */
    int32_t layout;             /* vd_rotary_layout */
    int32_t axes;               /* 1..VD_ROTARY_MAX_AXES */
    int32_t axis_pairs[VD_ROTARY_MAX_AXES];     /* their sum over the axes: rotary_dim / 2 */
    float amplitude;            /* finite; 1: the pairs keep their length */
    int64_t x_batch, x_token, x_head;
    int64_t y_batch, y_token, y_head;
    int64_t pos_batch, pos_token;       /* of positions, whose axes lie side by side */
    int64_t first_position;     /* positions NULL (one axis): token t is at first_position + t */
} vd_rotary_desc;

/* x, y device; y may be x (same strides).  freqs device double [rotary_dim / 2], turns (of 2 pi) per position, as
 * vd_rotary_frequencies makes them; positions device int32 [batch, tokens, axes], or NULL. */
VD_API vd_status vd_op_rotary(const vd_rotary_desc* d, const void* x, const int32_t* positions, const double* freqs, void* y,
                              void* cuda_stream);

typedef enum {
    VD_ROTARY_SCALE_NONE = 0,   /* theta_i = base^(-i/n) radians per position for the axis's pair i of n */
    VD_ROTARY_SCALE_LINEAR = 1, /* theta_i / factor: positions are interpolated */
    VD_ROTARY_SCALE_BASE = 2,   /* base * factor^(n/(n-1)): the fastest pair as it was, the slowest one divided by factor */
    VD_ROTARY_SCALE_PARTS = 3   /* pairs that turn `fast` times or more within original_len positions as they were, those that turn
                                   `slow` times or less divided by factor, a linear blend by turns in between */
} vd_rotary_scaling;

typedef struct {
    uint32_t struct_size;
    int32_t rotary_dim, axes;
    int32_t axis_pairs[VD_ROTARY_MAX_AXES];
    int32_t scaling;            /* vd_rotary_scaling */
    double base;                /* > 1 */
    double factor;              /* >= 1; unused by NONE */
    double original_len;        /* > 0; PARTS only */
    double fast, slow;          /* fast > slow >= 0; PARTS only */
} vd_rotary_freq_desc;
/* Writes the rotary_dim / 2 frequencies, in turns per position, to HOST memory (host-only; touches no device). */
VD_API vd_status vd_rotary_frequencies(const vd_rotary_freq_desc* d, double* freqs);

/* ------------------------------------------------------------------------------------------
 * The seam between two blocks: the gated residual add of the one and the modulated norm of the next, in one pass.
 *   u = h, or norm(h) * post_weight where post_norm is set
 *   r = x + residual_scale * gate * u                     (x where h is NULL)        -> x_out
 *   y = (norm(r) * weight + bias) * (1 + scale) + shift                             -> y
 * norm over the channels of a token: VD_NORM_LAYER (z - mean) / sqrt(var + eps), VD_NORM_RMS z / sqrt(mean z^2 + eps).
 * All sums are fp32 and r is rounded once, into x_out; y is made from the unrounded r.  NULL: gate 1, weight 1, bias 0,
 * scale 0, shift 0, post_weight 1; x_out or y not written.
 * gate, scale, shift hold a row for every mod_tokens consecutive tokens of a batch item (a frame, say).
 * ---------------------------------------------------------------------------------------- */
typedef enum { VD_NORM_LAYER = 0, VD_NORM_RMS = 1 } vd_norm_kind;

typedef struct {
    uint32_t struct_size;
    int32_t batch, tokens;      /* >= 0; batch * tokens < 2^31 */
    int32_t channels;           /* 1..16384 */
    int32_t x_dtype;            /* vd_dtype of x and x_out (the residual stream) */
    int32_t h_dtype, y_dtype;
    int32_t mod_dtype;          /* of gate, scale and shift; weight, bias and post_weight are fp32 [channels] */
    int32_t norm;               /* vd_norm_kind */
    int32_t post_norm;          /* 1: h is normalised too */
    int32_t mod_tokens;         /* >= 1 */
    float eps;                  /* > 0 */
    float residual_scale;       /* finite */
    int64_t x_batch, x_token, h_batch, h_token, xo_batch, xo_token, y_batch, y_token;
    int64_t gate_batch, gate_group, scale_batch, scale_group, shift_batch, shift_group;
} vd_gate_norm_desc;

/* All device.  x_out may be x (same strides) and y may be h (same strides and type): a token is read before it is written. */
VD_API vd_status vd_op_gate_norm(const vd_gate_norm_desc* d, const void* x, const void* h, const float* post_weight,
                                 const void* gate, void* x_out, const float* weight, const float* bias, const void* scale,
                                 const void* shift, void* y, void* cuda_stream);

#ifdef __cplusplus
}
#endif
#endif /* VD_BLOCK_H_ */
