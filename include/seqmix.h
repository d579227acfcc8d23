/*
 * seqmix.h -- C ABI of the token-mixing operators of the MI355X (gfx950) library.
 *
 * What a layer runs around its projections (1x1 convolutions, conv2d.h) when it mixes along a
 * sequence of tokens:
 *
 *   seqmix_conv   causal depthwise convolution over tokens, with SiLU and a carried window
 *   seqmix_attn   linear attention with a decay for each head, with a carried state
 *   seqmix_norm   the norms after and before a block, fused with its gate, residual scale and sum
 *
 * Forward only, like the 2D convolution.  Prompts, packed prompts of different lengths, prompts
 * that continue and single tokens go through the same entry points.
 *
 * Conventions, beyond those of conv2d.h (statuses CONV2D_*, types CONV2D_F32 / CONV2D_BF16, device
 * pointers owned by the caller, `stream` a hipStream_t, nothing aborts or prints, calls return
 * without waiting, descriptors are made without a GPU):
 *   - Rows are tokens.  Sequence i holds rows [offsets[i], offsets[i+1]) of the packed rows, offsets
 *     being seqs + 1 ascending int64 on the device, first 0 and last `tokens`; a sequence may be empty.
 *     offsets NULL: sequences of equal length, tokens / seqs rows each.  The kernels clamp what they
 *     read there to [0, tokens], so bad offsets give wrong results but no access out of range.
 *   - What is carried (attention's state, the convolution's window) lies in a pool of `slots` entries.
 *     slot_index holds one int32 per sequence on the device; no two sequences of a call may name the
 *     same slot.  A sequence whose slot is outside [0, slots) is skipped: none of its outputs
 *     are written (the empty places of a batch of fixed size).  slot_index NULL: sequence i has slot i
 *     (slots >= seqs is required then).
 *   - *_in NULL: sequences start from zeros.  *_out NULL: what is left at their ends is not kept.
 *     *_in == *_out updates the pool in place; otherwise the two must not overlap.  An empty sequence
 *     carries its entry over unchanged.  Outputs must not overlap any other argument unless said.
 *   - Strides count elements.  Rows may lie apart (columns of a wider tensor); the last dimension is dense.
 *   - Any alignment of an element's size is accepted, at the same speed but for rows below 16 bytes.  Results are
 *     bitwise reproducible for the same descriptor parameters.
 *   - Every product is summed in fp32 and states are fp32; outputs are rounded once, to nearest even.  (Attention in bf16
 *     multiplies what it has computed in fp32, scores and states, as sums of bf16 parts: 2^-16 of each term is
 *     left out where outputs are bf16, 2^-24 where they are fp32.)
 *   - seqmix_conv and seqmix_norm descriptors are never written by a call: any number of threads and
 *     streams may use one at a time.  A seqmix_attn descriptor may own a workspace; like a conv2d
 *     descriptor it is used by one host thread at a time, and a call on another stream than the
 *     previous one makes its stream wait for that call (whose stream must still exist, and must not be
 *     under capture by then: E_HIP).
 *   - Under graph capture, calls of one capture wait for each other, on whatever streams of it, and not
 *     for calls outside it.  The library does not see when a graph is launched: launches of graphs that hold
 *     calls of one seqmix_attn descriptor, and its other calls, are kept in order by the caller (on one
 *     stream, or by events) where it owns a workspace.
 */
#ifndef SEQMIX_H
#define SEQMIX_H

#include "conv2d.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ------------------------------------------------------------------ linear attention
 * Per sequence and head h, with the q/k head h / (heads / qk_heads):
 *
 *   S_t = exp(g_t) S_{t-1} + k_t v_t^T      (dk x dv)        o_t = scale * q_t S_t
 *
 * g is the log of the decay.  -infinity clears the state (a document that starts inside a sequence);
 * values above 0 let it grow (by less than 2^100 over any 64 tokens, or results are not finite); decays that come to less
 * than 2^-126 within 64 tokens may count as 0.  What a token holds never reaches the outputs of tokens before it, also where
 * it is infinite or NaN; the infinities that follow from it may be NaN. */
enum {
    SEQMIX_DECAY_NONE = 0,  /* g = 0 */
    SEQMIX_DECAY_HEAD = 1,  /* g[heads], the same for every token */
    SEQMIX_DECAY_TOKEN = 2  /* g[tokens][heads] */
};

#define SEQMIX_MAX_HEAD_DIM 256

typedef struct {
    int64_t tokens, seqs, slots;
    int32_t heads;     /* heads of v, o and the state */
    int32_t qk_heads;  /* heads of q and k: divides heads */
    int32_t dk, dv;    /* 1 .. SEQMIX_MAX_HEAD_DIM */
    int32_t dtype;     /* q, k, v */
    int32_t o_dtype;   /* dtype, or CONV2D_F32 */
    int32_t decay;     /* SEQMIX_DECAY_*; g is always fp32 */
    float scale;
    /* elements from a token to the next, and from a head to the next */
    int64_t q_row, q_head, k_row, k_head, v_row, v_head, o_row, o_head;
} seqmix_attn_params;

/* Kernels of an attention call: token by token with the state in registers, or chunks of tokens on the
 * matrix cores (for long sequences in segments that run side by side, their states joined by a scan).  Chosen by the
 * sizes here, which of packed sequences are averages: many short ones with a few long ones among them are better called apart. */
enum { SEQMIX_KERNEL_TOKENS = 0, SEQMIX_KERNEL_CHUNKS = 1 };

typedef struct {
    int32_t kernel;           /* SEQMIX_KERNEL_* */
    int32_t chunk;            /* tokens per chunk (CHUNKS) */
    int64_t segment;          /* tokens per segment; 0: sequences are not cut */
    int64_t workspace_bytes;  /* states at the segments' starts, and their decays */
} seqmix_attn_plan_info;

typedef struct seqmix_attn_desc seqmix_attn_desc;

/* E_NULL, E_INVALID (sizes out of range, a stride below the dimension inside it, slots < 1,
 * tokens not a multiple of seqs is found at the call), E_UNSUPPORTED (dims over
 * SEQMIX_MAX_HEAD_DIM, unknown types, fp32 q with bf16 o, 2^31 tokens or more). */
int seqmix_attn_desc_create(const seqmix_attn_params* params, seqmix_attn_desc** out);
/* Frees the descriptor and its workspace (which waits for work queued on the device, and is not to be done under
 * capture; a graph that holds its calls must not be launched afterwards).  NULL is OK. */
int seqmix_attn_desc_destroy(seqmix_attn_desc* desc);
int seqmix_attn_plan_query(const seqmix_attn_desc* desc, seqmix_attn_plan_info* out);
/* Allocate the workspace on the current device now; calls then allocate nothing and can be captured
 * in a graph.  Without it the first call allocates.  E_NULL, E_ALLOC, E_HIP,
 * E_UNSUPPORTED (already on another device). */
int seqmix_attn_reserve(seqmix_attn_desc* desc);
/* q, k: [tokens][qk_heads][dk], v: [tokens][heads][dv], o: [tokens][heads][dv] by the strides given;
 * decay: fp32, NULL with SEQMIX_DECAY_NONE; state_in / state_out: fp32 [slots][heads][dk][dv], dense.
 * Errors: E_NULL, E_INVALID (offsets NULL and tokens not a multiple of seqs; slot_index NULL and
 * slots < seqs), E_ALLOC, E_HIP, E_UNSUPPORTED (workspace on another device). */
int seqmix_attn_fwd(seqmix_attn_desc* desc, const void* q, const void* k, const void* v, const float* decay,
                    const int64_t* offsets, const int32_t* slot_index, const float* state_in, float* state_out, void* o,
                    void* stream);

/* ------------------------------------------------------------------ causal convolution
 *
 *   y[t,c] = act(bias[c] + sum_{i < width} w[c,i] x[t - width + 1 + i, c])
 *
 * Rows before a sequence's start come from its window: the last width - 1 rows that went before, oldest first.
 * window_out receives the last width - 1 rows of window and sequence together. */
enum { SEQMIX_ACT_NONE = 0, SEQMIX_ACT_SILU = 1, SEQMIX_ACT_SIGMOID = 2, SEQMIX_ACT_LINEAR = 3 };

#define SEQMIX_MAX_CONV_WIDTH 8

typedef struct {
    int64_t tokens, seqs, slots, channels;
    int32_t width;          /* taps, 1 .. SEQMIX_MAX_CONV_WIDTH */
    int32_t dtype;          /* x, w, y and the windows; the bias is fp32 */
    int32_t act;            /* SEQMIX_ACT_NONE or SEQMIX_ACT_SILU */
    int32_t has_bias;
    int64_t x_row, y_row;   /* elements from a token to the next */
} seqmix_conv_params;

typedef struct seqmix_conv_desc seqmix_conv_desc;

/* E_NULL, E_INVALID, E_UNSUPPORTED (width over SEQMIX_MAX_CONV_WIDTH, unknown type or activation, 2^31 tokens or
 * channels or more). */
int seqmix_conv_desc_create(const seqmix_conv_params* params, seqmix_conv_desc** out);
int seqmix_conv_desc_destroy(seqmix_conv_desc* desc);
/* x, y: [tokens][channels], w: [channels][width], windows: [slots][width-1][channels], dense.
 * Errors: E_NULL, E_INVALID (as seqmix_attn_fwd), E_HIP. */
int seqmix_conv_fwd(const seqmix_conv_desc* desc, const void* x, const void* w, const float* bias,
                    const int64_t* offsets, const int32_t* slot_index, const void* window_in, void* window_out, void* y,
                    void* stream);

/* ------------------------------------------------------------------ norms around a block
 * Per row of `width` elements, in groups of `group`:
 *
 *   n = post(u) act(gate)          or, with gate_first,   n = post(u act(gate))
 *   y = residual + scale scale_vec n        h = pre(y)
 *
 * post norms each group, pre the whole row: RMS x / sqrt(mean(x^2) + eps) * w, or LAYER with
 * the mean taken off first, + b where there is a bias.  Leave out what is not wanted: post and
 * pre NONE, gate NONE (factor 1), no residual, no scale_vec.  y is rounded to its type after h
 * has been computed from it in fp32. */
enum { SEQMIX_NORM_NONE = 0, SEQMIX_NORM_RMS = 1, SEQMIX_NORM_LAYER = 2 };

#define SEQMIX_MAX_NORM_WIDTH 16384

typedef struct {
    int64_t rows, width;
    int64_t group;         /* divides width; with pre: width */
    int64_t gate_run;      /* rows that share a row of the gate: row r reads gate row r / gate_run */
    int32_t dtype;         /* u, gate, h */
    int32_t res_dtype;     /* residual, y: dtype, or CONV2D_F32 */
    int32_t post, post_bias;  /* SEQMIX_NORM_*; weight and bias fp32 [group], shared by the groups */
    int32_t gate;          /* SEQMIX_ACT_NONE (no gate), SILU, SIGMOID or LINEAR (gate itself) */
    int32_t gate_first;
    int32_t residual;
    int32_t scale_vec;     /* scale_vec fp32 [width] is given */
    int32_t pre, pre_bias; /* SEQMIX_NORM_*; weight and bias fp32 [width] */
    float scale;
    float post_eps, pre_eps;  /* >= 0 */
    int64_t u_row, gate_row, res_row, y_row, h_row;
} seqmix_norm_params;

typedef struct seqmix_norm_desc seqmix_norm_desc;

/* E_NULL, E_INVALID, E_UNSUPPORTED (group over SEQMIX_MAX_NORM_WIDTH, pre with group < width, unknown types,
 * norms or gates). */
int seqmix_norm_desc_create(const seqmix_norm_params* params, seqmix_norm_desc** out);
int seqmix_norm_desc_destroy(seqmix_norm_desc* desc);
/* Pointers that the descriptor does not ask for are ignored.  y may be NULL when pre is given (only h
 * is wanted).  y may be the residual itself (rows and strides the same).
 * Errors: E_NULL, E_INVALID (h is y), E_HIP. */
int seqmix_norm_fwd(const seqmix_norm_desc* desc, const void* u, const float* post_w, const float* post_b,
                    const void* gate, const void* residual, const float* scale_vec, const float* pre_w,
                    const float* pre_b, void* y, void* h, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* SEQMIX_H */
