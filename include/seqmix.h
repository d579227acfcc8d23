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
 * and where some of its layers keep keys and values instead of a state:
 *
 *   seqmix_softmax  softmax attention of prompts, of single tokens and of trees of drafted tokens
 *   seqmix_rotary   rotary positions of q and k, which writes k and v into the cache
 *   seqmix_pages    which pages of the cache each request has, and where its next tokens go
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
 *   - Any alignment of an element's size is accepted, at the same speed but for rows below 16 bytes (softmax attention: up
 *     to twice the time where k and v are not in whole 16 bytes).  Results are bitwise reproducible for the same
 *     descriptor parameters, at whatever addresses.
 *   - Every product is summed in fp32 and states are fp32; outputs are rounded once, to nearest even.  (Attention in bf16
 *     multiplies what it has computed in fp32, scores and states, as sums of bf16 parts: 2^-16 of each term is
 *     left out where outputs are bf16, 2^-24 where they are fp32.  seqmix_softmax says for itself.)
 *   - seqmix_conv, seqmix_norm, seqmix_rotary and seqmix_pages descriptors are never written by a call: any number of threads
 *     and streams may use one at a time.  A seqmix_attn or seqmix_softmax descriptor may own a workspace; like a conv2d
 *     descriptor it is used by one host thread at a time, and a call on another stream than the
 *     previous one makes its stream wait for that call (whose stream must still exist, and must not be
 *     under capture by then: E_HIP).
 *   - Under graph capture, calls of one capture wait for each other, on whatever streams of it, and not
 *     for calls outside it.  The library does not see when a graph is launched: launches of graphs that hold
 *     calls of one seqmix_attn or seqmix_softmax descriptor, and its other calls, are kept in order by the caller (on one
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

/* ------------------------------------------------------------------ softmax attention
 * Per row t of sequence i and head h, with the k/v head h / (heads / kv_heads):
 *
 *   o_t = sum_j p_tj v_j / sum_j p_tj        p_tj = exp(scale q_t . k_j), over the keys j that t sees
 *
 * A sequence of `len` rows has n keys, of which the last `len` are the rows' own (those of its new tokens) and the ones before
 * them what went before.  A row sees
 *   SEQMIX_MASK_FULL    all n keys
 *   SEQMIX_MASK_CAUSAL  keys 0 .. n - len + t
 *   SEQMIX_MASK_TREE    keys 0 .. n - len - 1, and of the own keys number j < 64 where bit j of tree[t] is set (drafted tokens
 *                       that continue the text in several ways: the bits of a token, its parent, ...)
 * Rows that see no key (n = 0, n < len, an empty mask) are zeros.  Keys that a row does not see never reach it, also where
 * they hold infinities or NaN.  Where it sees values that are not finite, its results there are NaN.  Scores are
 * compared as they are, times log2(e): one of +infinity makes the row NaN, ones of -infinity count nothing (a row of which all
 * are is zeros).
 *
 * Keys and values lie
 *   packed (page 0)  in key_tokens rows; sequence i holds rows [key_offsets[i], key_offsets[i+1]); key_offsets NULL: the rows
 *                    of q (key_tokens = tokens).
 *   in pages         of `page` tokens (a power of two): key j of the sequence in slot s lies in page
 *                    table[s][j / page], row j % page, and the slot holds lens[s] keys (the new ones among them).
 * Lengths and page numbers are clamped to what there is, so bad ones give wrong results but no access out of range.
 *
 * Precision: scores and sums are fp32 products and sums of what q, k and v hold.  Sums over v are of weights up to 2^8 (they are
 * divided at the end), so they are finite where 2^8 times the number of keys times the largest |v| is.  bf16: the step kernel
 * multiplies v by weights in two bf16 parts (2^-16 of each is left out), so results are rounded once; the prompt kernel by
 * weights rounded to bf16 (2^-8 of each at most, about the result's own rounding: 0.0020 to 0.0023 off in the 2-norm, one rounding 0.0016),
 * which halves its longest products.  Which kernel a call has, plan_query says: trees of more than a few drafts have the
 * prompt kernel, single tokens the other, so a token that is drafted in a tree and one that is decoded alone may differ by that. */
enum { SEQMIX_MASK_FULL = 0, SEQMIX_MASK_CAUSAL = 1, SEQMIX_MASK_TREE = 2 };

#define SEQMIX_MAX_PAGE 65536

typedef struct {
    int64_t tokens, seqs, slots;
    int64_t key_tokens;  /* packed: rows of k and v */
    int64_t pages;       /* in pages: of the cache, */
    int64_t max_pages;   /* columns of the table, */
    int32_t page;        /* tokens of a page; 0: packed */
    int32_t heads;       /* of q and o */
    int32_t kv_heads;    /* of k and v: divides heads */
    int32_t dk, dv;      /* 1 .. SEQMIX_MAX_HEAD_DIM */
    int32_t dtype;       /* q, k, v, o */
    int32_t mask;        /* SEQMIX_MASK_* */
    float scale;         /* times log2(e) finite */
    /* elements from a token to the next, from a head to the next, and from a page to the next (in pages) */
    int64_t q_row, q_head, o_row, o_head;
    int64_t k_row, k_head, k_page, v_row, v_head, v_page;
} seqmix_softmax_params;

/* Kernels of a call: 128 rows of a sequence per workgroup, or 32, whose keys its waves divide; chosen by the average number of
 * rows of a sequence (times the heads that share a k/v head).  Rows of a workgroup are of one sequence, and of `pack` heads of those
 * that share a k/v head, a divisor of their number: as many as fill it by that average.  What this serves badly (16 heads of
 * 128 over 4 k/v heads where nothing else is said):
 *   - a prompt and single tokens in one call, as each single token's keys are read for every head: 2048 tokens and 32 single
 *     ones over up to 8000 keys take 333 us, the two as calls of their own 64 and 64;
 *   - few heads to pack, where those of a k/v head have few divisors: 16 trees of 24 drafts over up to 5000 keys take 49 us,
 *     with 28 heads (7 of a k/v head) 201; 16 of 2 drafts with 64 heads over one 35, with 71 over one 306. */
enum { SEQMIX_KERNEL_PROMPT = 0, SEQMIX_KERNEL_STEP = 1 };

typedef struct {
    int32_t kernel;           /* SEQMIX_KERNEL_* */
    int32_t pack;             /* heads that share a workgroup, a divisor of heads / kv_heads */
    int64_t shares;           /* 0: a workgroup takes all keys of its rows; else the keys of all rows are divided in so many shares */
    int64_t workspace_bytes;  /* results of rows whose keys are in several shares */
} seqmix_softmax_plan_info;

typedef struct seqmix_softmax_desc seqmix_softmax_desc;

/* E_NULL, E_INVALID (sizes out of range, a stride below the dimension inside it, a page that is no power of two),
 * E_UNSUPPORTED (dims over SEQMIX_MAX_HEAD_DIM, pages over SEQMIX_MAX_PAGE, unknown types or masks, 2^31 tokens or cached rows or
 * more; keys of a sequence, or tokens and sequences together times heads, beyond 2^31 - 1024).  Workspaces, streams and captures are as those of
 * seqmix_attn. */
int seqmix_softmax_desc_create(const seqmix_softmax_params* params, seqmix_softmax_desc** out);
int seqmix_softmax_desc_destroy(seqmix_softmax_desc* desc);
int seqmix_softmax_plan_query(const seqmix_softmax_desc* desc, seqmix_softmax_plan_info* out);
/* As seqmix_attn_reserve, but it waits for work queued on the device (counts in the workspace are cleared), and is not to be
 * done under capture.  A first call without it clears them on its stream and does not wait; a captured one does so whenever its
 * graph runs. */
int seqmix_softmax_reserve(seqmix_softmax_desc* desc);
/* q: [tokens][heads][dk], o: [tokens][heads][dv], k: [key_tokens][kv_heads][dk] or [pages][page][kv_heads][dk], v alike, by the
 * strides given; key_offsets int64 [seqs + 1] (packed; else ignored); lens int32 [slots], table int32
 * [slots][max_pages] (in pages; else ignored); tree int64 [tokens] (SEQMIX_MASK_TREE; else ignored).
 * Rows of skipped sequences, and rows of no sequence, are left as they were.
 * Errors: E_NULL, E_INVALID (as seqmix_attn_fwd; key_offsets NULL and key_tokens not tokens), E_ALLOC, E_HIP, E_UNSUPPORTED
 * (workspace on another device). */
int seqmix_softmax_fwd(seqmix_softmax_desc* desc, const void* q, const void* k, const void* v, const int64_t* offsets,
                       const int64_t* key_offsets, const int32_t* slot_index, const int32_t* lens, const int32_t* table,
                       const int64_t* tree, void* o, void* stream);

/* ------------------------------------------------------------------ rotary positions
 * The first `rot` elements of each head of q and k turn in pairs (a, b) by the angle w = position[t] freqs[i] of pair i:
 *
 *   a' = amplitude (a cos w - b sin w)        b' = amplitude (b cos w + a sin w)
 *
 * Pair i is elements i and i + rot / 2 (SEQMIX_ROTARY_HALF) or 2 i and 2 i + 1 (SEQMIX_ROTARY_INTERLEAVED); the elements from
 * rot on are copied.  Angles are computed in 64 bits, whatever the type.  Frequencies that are scaled for long
 * contexts are other freqs (and amplitude).
 * With a cache (page > 0), turned k and v as it is go to row place[t] of it: page place[t] / page, row
 * place[t] % page.  Tokens with a place outside the cache are not stored; no two tokens of a call may have the same place. */
enum { SEQMIX_ROTARY_HALF = 0, SEQMIX_ROTARY_INTERLEAVED = 1 };

typedef struct {
    int64_t tokens;
    int64_t pages;     /* of the cache */
    int32_t page;      /* tokens of a page, a power of two; 0: no cache */
    int32_t heads;     /* of q; 0: no q */
    int32_t kv_heads;  /* of k and v; 0: none */
    int32_t dk, dv;    /* 1 .. SEQMIX_MAX_HEAD_DIM (dv: with a cache) */
    int32_t rot;       /* even, 0 .. dk */
    int32_t layout;    /* SEQMIX_ROTARY_* */
    int32_t dtype;
    float amplitude;
    int64_t q_row, q_head, k_row, k_head, v_row, v_head, qo_row, qo_head, ko_row, ko_head;
    int64_t kc_row, kc_head, kc_page, vc_row, vc_head, vc_page;
} seqmix_rotary_params;

typedef struct seqmix_rotary_desc seqmix_rotary_desc;

/* E_NULL, E_INVALID, E_UNSUPPORTED (as seqmix_softmax_desc_create).  Descriptors are never written by a call. */
int seqmix_rotary_desc_create(const seqmix_rotary_params* params, seqmix_rotary_desc** out);
int seqmix_rotary_desc_destroy(seqmix_rotary_desc* desc);
/* q, q_out: [tokens][heads][dk], k, k_out: [tokens][kv_heads][dk], v: [tokens][kv_heads][dv], by the strides given; position, place:
 * int32 [tokens]; freqs: float64 [rot / 2], in radians per position.  q_out may be q and k_out k (same strides).  What
 * is not wanted is NULL: k_out with a cache, or both it and the caches (then k and v are ignored).
 * Errors: E_NULL, E_HIP. */
int seqmix_rotary_fwd(const seqmix_rotary_desc* desc, const void* q, const void* k, const void* v, const int32_t* position,
                      const double* freqs, void* q_out, void* k_out, void* k_cache, void* v_cache, const int32_t* place,
                      void* stream);

/* ------------------------------------------------------------------ pages of the cache
 * Moves the requests of a call on to their next tokens.  Slot s of the pool holds a request of lens[s] tokens, in pages
 * table[s][0 .. ceil(lens[s] / page) - 1].  free_pages holds each page of the cache once; the first *taken of them
 * are in use (a new pool: free_pages 0, 1, 2, ..., *taken 0, lens 0).  In this order:
 *
 *   1. Each sequence goes back to its first kept[i] tokens (at least 0, at most what it has; kept NULL: none goes back: refused
 *      drafts are taken off so, and requests that have ended, with no new rows).  Pages that it no longer needs
 *      become the last *taken entries of free_pages that were in use, in the order of the sequences and of
 *      their pages, and *taken falls.
 *   2. Its new rows [offsets[i], offsets[i+1]) are added, in pages from free_pages[*taken] on, in the same order; *taken rises.
 *      A sequence that would need more than max_pages is refused, and so is every one that needs pages from the first on
 *      that the pool has too few for: it gets none, and keeps its kept[i] tokens.
 *   3. position[t] and place[t] are the number of each new row in its request and its row of the cache.
 *      admitted[i] is the sequence's slot, or -1 where it was refused or skipped: the slot_index for the
 *      operators that follow.  Rows of refused and skipped sequences, and of none, have place -1 and position 0.
 *
 * Entries of the table behind a request's pages are left as they were.  One workgroup does 1. and 2. */
typedef struct {
    int64_t tokens, seqs, slots;
    int64_t pages, max_pages;
    int32_t page;  /* tokens of a page, a power of two */
} seqmix_pages_params;

typedef struct seqmix_pages_desc seqmix_pages_desc;

/* E_NULL, E_INVALID, E_UNSUPPORTED (as seqmix_softmax_desc_create).  Descriptors are never written by a call. */
int seqmix_pages_desc_create(const seqmix_pages_params* params, seqmix_pages_desc** out);
int seqmix_pages_desc_destroy(seqmix_pages_desc* desc);
/* kept, slot_index, admitted: int32 [seqs]; lens: int32 [slots], table: int32 [slots][max_pages], free_pages: int32 [pages],
 * taken: int32 [1], all four updated; place, position: int32 [tokens].
 * Errors: E_NULL, E_INVALID (as seqmix_attn_fwd), E_HIP. */
int seqmix_pages_fwd(const seqmix_pages_desc* desc, const int32_t* kept, const int64_t* offsets, const int32_t* slot_index,
                     int32_t* lens, int32_t* table, int32_t* free_pages, int32_t* taken, int32_t* place, int32_t* position,
                     int32_t* admitted, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* SEQMIX_H */
