// seqmix_api.hip -- C ABI of the token-mixing operators: validation, plans, workspaces, launches.
#include <algorithm>
#include <new>

#include "seqmix_workspace.h"

using namespace cv;

struct seqmix_attn_desc {
    seqmix_attn_params p;
    seqmix_attn_plan_info plan;
    int32_t block = 0, block_uncut = 0;  // state columns per workgroup; of chunk kernels where no sequence is cut
    int64_t alone = 0, alone_packed = 0;  // sequences of up to this many tokens are not cut: of one length; packed
    Workspace ws;  // of plan.workspace_bytes
};
struct seqmix_conv_desc {
    seqmix_conv_params p;
};
struct seqmix_norm_desc {
    seqmix_norm_params p;
};

namespace {

// The chunk kernels address the rows of a chunk by 32-bit byte offsets from its first: rows further apart go
// token by token.
bool chunk_rows_near(const seqmix_attn_params& p) {
    return std::max({p.q_row, p.k_row, p.v_row, p.o_row, (int64_t)p.heads}) <= (1LL << 31) / (kChunk * 4) - SEQMIX_MAX_HEAD_DIM;
}

// Sequences of one length up to this are not cut: the chain of their chunks would be shortened by less than cutting
// costs, which is 0.6 of the chunks of a segment and 3 chunks (dk up to 64), 2.75 (128) or 1.5 (256; fp32 2.75, 1.75, 1).
// Both sides measured: 2 heads, 320 tokens of 64 x 64 15.4 us, cut 13.7; 256 of 256 x 128 24.7, 19.4 (fp32 59.5, 23.0).  At dk
// 128 the limit is that of 16 heads (300 tokens of 128 x 128 20.1, 19.6); fewer heads gain by cutting from 5 chunks on, and
// some lengths of theirs stay uncut that need not (8 heads: 256 tokens 16.8, 16.6; 300 20.0, 17.1).  `groups` workgroups
// of 64 columns are busy uncut; 1.25 times their share of the CUs is what cutting costs in throughput (16 heads of
// 128 x 128, 4 sequences: 1000 tokens 57 us, cut 56, and 4000 224, 133; 6 of 700 43, 56; 8 of 2000 120, 136).
int64_t alone(const seqmix_attn_params& p, int64_t segment, int64_t chunk, int64_t groups) {
    const int quarters[2][3] = {{12, 11, 6}, {11, 7, 4}};  // of a chunk
    const int64_t least = segment * 8 / 5 + chunk * quarters[p.dtype == CONV2D_F32][p.dk <= 64 ? 0 : p.dk <= 128 ? 1 : 2] / 4;
    const int64_t left = 4 * kSeqmixCUs - 5 * groups;  // of 4 per CU
    return left > 0 ? least * 4 * kSeqmixCUs / left : INT64_MAX;
}

// ... of packed sequences, where a longer one may make the other launches necessary in any case.  16 of 62 to 1000 tokens,
// 8 heads of 64 x 128, segments of 192: 41 us, up to 531 uncut 49; 8 of 500, 16 heads of 128 x 128, whose ends would have met
// uncut: 58 us, 44; 8 of 200, segments of 128, 29 us, cut 41.
int64_t alone_packed(int64_t segment, int64_t chunk) { return std::max(segment + chunk, segment * 8 / 5); }

// State columns of a workgroup of the chunk kernels, of which there are `groups` with the wider blocks.  Where the last
// 128 would be half empty 64 are better in fp32 (4096 tokens, 16 heads of 128 x 192: 129 us, 147) and for keys of up to 64
// (8192 tokens of 64 x 192 73.6, 74.6; 7 sequences, 3408 tokens of 64 x 189 59.8, 62.6), not for wider bf16 keys, whose
// scores each block computes (8192 tokens of 128 x 192 110, 103; of 256 x 192 215, 189).
int64_t chunk_columns(const seqmix_attn_params& p) {
    const bool narrow = p.dv <= 64 || p.dk <= 64 || p.dtype == CONV2D_F32;
    return narrow && (p.dv - 1) % 128 < 64 ? 64 : 128;
}
int32_t chunk_block(const seqmix_attn_params& p, int64_t groups) {
    return (int32_t)(groups * 2 <= kSeqmixCUs ? 64 : chunk_columns(p));
}

// Places for segments' states in the workspace.
int64_t ws_places(const seqmix_attn_params& p, int64_t segment) {
    return p.seqs == 1 ? (p.tokens + segment - 1) / segment : 2 * p.tokens / segment;
}

// Kernel, state columns per workgroup (block) and where sequences are cut.
//
// Up to 2 tokens per sequence (fp32: 4) go token by token.  A chunk costs the same for 1 token as for 64, the token
// kernel more with each: 8 sequences, 16 heads of 128 x 128 bf16: 4.9, 5.8 and 6.7 us for 1, 2 and 3 tokens, a chunk
// 8.2; 256 sequences: 105, 113 and 120 us, a chunk 117; fp32, 128 sequences: 55 to 68 us for 1 to 4 tokens, a chunk 74.
// Its blocks have 32 columns (more workgroups; 64 sequences of 16 heads of 64 x 64: 8.6 us, with 128 columns 8.8)
// until there are 8 such per CU, then 128 (256 sequences as above: 105 us, with 32 columns 106).  Where dv is no
// multiple of 32, blocks share cache lines at their ends, and 128 are better from one per CU on (16 heads of 127 x 127,
// 4, 8 and 64 sequences: 7.6, 11.7 and 43 us with 32 columns, 8.1, 8.6 and 24 with 128).
//
// A workgroup takes its chunks one after the other, about 5 us each (dk = dv = 128) with one workgroup per CU and 8
// with two. Cutting adds a pass over k and v, two more launches and 16 dk dv bytes per segment and head, so the
// segments are as long as 256 workgroups allow, or 512 where those still have 8 chunks each: 8192 tokens, 16 heads of
// 128 x 128 bf16: 74 us in segments of 512, 79 of 256, 87 of 384 (a part of the CUs has two), 94 of 1024; 65536
// tokens, 8 heads: 224 us in segments of 1024, 235 of 2048, 250 of 512.  In fp32 segments may be one chunk of 32 tokens
// while they leave half of the CUs empty (512 tokens, 2 heads: 18.6 us, of 64 tokens 22.1; 16 heads: 31, 29).
// Packed sequences, whose lengths the host does not know, take 512 (5664 tokens in 10 sequences, 12 heads of 64 x 128:
// 43 us in segments of 192, 45 of 256, 49 of 512); the kernels cut the longer ones (alone_packed).  They may be one
// long prompt among single tokens (1, 570, 3, 1 tokens, 1 head of 191 x 128: 23 us, uncut 70; 64 of 1 and one of 1000,
// 16 heads of 128 x 128: 60, uncut 100) or of one length, where the other launches are wasted (4 of 150, 4 heads: 18 us,
// uncut 13.6). Where 128-column blocks leave half of the CUs empty, blocks of 64 (8 heads, 1024 tokens: 24.5 us, 25.8;
// 300 tokens: 20.0, 23.4).
//
// The rules look at averages, so packs of many sequences with a long one among them are far from what they could be: with 512
// workgroups or more and 64 tokens on average nothing is cut (39 of 100 tokens and one of 16384, 16 heads of 128 x 128: 1072 us,
// of which the long one's bytes are 66), and at 2 tokens on average all go token by token (255 of 1 token and one of 257:
// 499 us, in chunks 151; 255 empty places and one of 512: 896, 141; but 256 of 2: 114, 138).
void plan_attn(seqmix_attn_desc* d) {
    const seqmix_attn_params& p = d->p;
    d->plan = seqmix_attn_plan_info{SEQMIX_KERNEL_TOKENS, 0, 0, 0};
    const int64_t narrow = p.seqs * p.heads * ((p.dv + kTokensBlock - 1) / kTokensBlock);
    d->block = narrow > (p.dv % kTokensBlock ? 1 : 8) * kSeqmixCUs ? kTokensWide : kTokensBlock;
    if (p.tokens <= (p.dtype == CONV2D_BF16 ? 2 : 4) * p.seqs || !chunk_rows_near(p)) return;
    const int64_t chunk = p.dtype == CONV2D_BF16 ? kChunk : kChunkF32;
    d->plan.kernel = SEQMIX_KERNEL_CHUNKS;
    d->plan.chunk = (int32_t)chunk;
    const int64_t across = p.heads * ((p.dv + 127) / 128);
    const int64_t groups = p.seqs * across;  // workgroups, uncut
    d->block = d->block_uncut = chunk_block(p, groups);
    if (groups < 2 * kSeqmixCUs || p.tokens < chunk * p.seqs) {
        auto length = [&](int64_t want) {  // of segments, such that there are about `want` workgroups
            const int64_t all = want / across, parts = std::max<int64_t>(p.seqs > 1 ? std::max(all - p.seqs, all / 2) : all, 1);
            const int64_t unit = (p.tokens / chunk + (p.seqs > 1 ? p.seqs : 0)) * across * 2 <= kSeqmixCUs ? chunk : kChunk;
            return ((p.tokens + parts - 1) / parts + unit - 1) / unit * unit;
        };
        int64_t seg = length(2 * kSeqmixCUs);
        if (p.seqs == 1 && seg < 8 * chunk) seg = length(kSeqmixCUs);
        d->alone = alone(p, seg, chunk, p.seqs * p.heads * ((p.dv + 63) / 64));
        if (p.tokens > (p.seqs == 1 ? d->alone : alone(p, seg, chunk, 0) + 2 * chunk)) {
            d->plan.segment = seg;
            d->alone_packed = alone_packed(seg, chunk);
            d->plan.workspace_bytes = ws_places(p, seg) * p.heads * ((int64_t)p.dk * p.dv * 4 + 4);
            d->block = chunk_block(p, std::max<int64_t>((p.tokens + seg - 1) / seg, p.seqs) * across);
        }
    }
}

}  // namespace

extern "C" {

// ------------------------------------------------------------------ attention
int seqmix_attn_desc_create(const seqmix_attn_params* params, seqmix_attn_desc** out) {
    if (!params || !out) return CONV2D_E_NULL;
    const seqmix_attn_params& p = *params;
    SM_TRY(check_seqs(p.tokens, p.seqs, p.slots));
    if (p.heads < 1 || p.qk_heads < 1 || p.heads % p.qk_heads != 0 || p.dk < 1 || p.dv < 1) return CONV2D_E_INVALID;
    if (!strides_ok(p.tokens, p.q_row, p.qk_heads, p.q_head, p.dk) ||
        !strides_ok(p.tokens, p.k_row, p.qk_heads, p.k_head, p.dk) ||
        !strides_ok(p.tokens, p.v_row, p.heads, p.v_head, p.dv) ||
        !strides_ok(p.tokens, p.o_row, p.heads, p.o_head, p.dv))
        return CONV2D_E_INVALID;
    if (!known_dtype(p.dtype) || !known_dtype(p.o_dtype) || (p.dtype == CONV2D_F32 && p.o_dtype != CONV2D_F32))
        return CONV2D_E_UNSUPPORTED;
    if (p.decay != SEQMIX_DECAY_NONE && p.decay != SEQMIX_DECAY_HEAD && p.decay != SEQMIX_DECAY_TOKEN)
        return CONV2D_E_INVALID;
    if (p.dk > SEQMIX_MAX_HEAD_DIM || p.dv > SEQMIX_MAX_HEAD_DIM) return CONV2D_E_UNSUPPORTED;
    seqmix_attn_desc* d = new (std::nothrow) seqmix_attn_desc;
    if (!d) return CONV2D_E_ALLOC;
    d->p = p;
    plan_attn(d);
    *out = d;
    return CONV2D_OK;
}

int seqmix_attn_desc_destroy(seqmix_attn_desc* d) {
    if (!d) return CONV2D_OK;
    d->ws.release();
    delete d;
    return CONV2D_OK;
}

int seqmix_attn_plan_query(const seqmix_attn_desc* d, seqmix_attn_plan_info* out) {
    if (!d || !out) return CONV2D_E_NULL;
    *out = d->plan;
    return CONV2D_OK;
}

int seqmix_attn_reserve(seqmix_attn_desc* d) {
    if (!d) return CONV2D_E_NULL;
    return d->ws.ensure(d->plan.workspace_bytes);
}

int seqmix_attn_fwd(seqmix_attn_desc* d, const void* q, const void* k, const void* v, const float* decay,
                    const int64_t* offsets, const int32_t* slot_index, const float* state_in, float* state_out, void* o,
                    void* stream) {
    if (!d) return CONV2D_E_NULL;
    const seqmix_attn_params& p = d->p;
    if (p.tokens > 0 && (!q || !k || !v || !o || (p.decay != SEQMIX_DECAY_NONE && !decay))) return CONV2D_E_NULL;
    AttnArgs a{};
    SM_TRY(seq_args(p.tokens, p.seqs, p.slots, offsets, slot_index, &a.sq));
    hipStream_t s = static_cast<hipStream_t>(stream);
    a.q = q;
    a.k = k;
    a.v = v;
    a.g = p.decay == SEQMIX_DECAY_NONE ? nullptr : decay;
    a.s_in = state_in;
    a.s_out = state_out;
    a.o = o;
    a.q_row = p.q_row, a.q_head = p.q_head, a.k_row = p.k_row, a.k_head = p.k_head;
    a.v_row = p.v_row, a.v_head = p.v_head, a.o_row = p.o_row, a.o_head = p.o_head;
    a.g_row = p.decay == SEQMIX_DECAY_TOKEN ? p.heads : 0;
    a.heads = p.heads;
    a.rep = p.heads / p.qk_heads;
    a.dk = p.dk;
    a.dv = p.dv;
    a.scale = p.scale;
    const int64_t unit = 16 / esize(p.dtype);
    a.vec = p.dk % unit == 0 && p.dv % unit == 0;
    const bool chunked = d->plan.kernel == SEQMIX_KERNEL_CHUNKS;
    const bool cut = d->plan.segment > 0 && (offsets || a.sq.seq_len > d->alone);
    a.block = chunked && !cut ? d->block_uncut : d->block;
    a.ndvb = (p.dv + a.block - 1) / a.block;
    if (!chunked) {
        return launch_attn_tokens(a, p.dtype, p.o_dtype, s) == hipSuccess ? CONV2D_OK : CONV2D_E_HIP;
    }
    auto chunks = [&](bool state_only) {
        a.places = state_only && offsets && a.nws < a.nseg;
        a.ids = !cut ? p.seqs : a.places ? a.nws : a.nseg;
        // heads that share q and k, and their column blocks, stay together where there are units for all XCDs
        a.unit = a.ids * p.qk_heads >= 16 ? a.rep * a.ndvb : 1;
        a.units = p.heads * a.ndvb / a.unit;
        return p.dtype == CONV2D_BF16 ? launch_attn_chunks_bf16(a, p.o_dtype, state_only, s)
                                      : launch_attn_chunks_f32(a, state_only, s);
    };
    if (!cut) return chunks(false) == hipSuccess ? CONV2D_OK : CONV2D_E_HIP;
    SM_TRY(d->ws.ensure(d->plan.workspace_bytes));
    SM_TRY(d->ws.order_after_last(s));
    a.segment = d->plan.segment;
    a.alone = offsets ? d->alone_packed : a.segment;
    a.nseg = seq_part_ids(a.sq, a.segment);
    a.ws_mul = p.seqs == 1 ? 1 : 2;
    a.nws = ws_places(p, a.segment);
    a.ws_state = static_cast<float*>(d->ws.data);
    a.ws_decay = a.ws_state + a.nws * p.heads * p.dk * p.dv;
    if (chunks(true) != hipSuccess || launch_attn_join(a, s) != hipSuccess || chunks(false) != hipSuccess)
        return CONV2D_E_HIP;
    return CONV2D_OK;
}

// ------------------------------------------------------------------ causal convolution
int seqmix_conv_desc_create(const seqmix_conv_params* params, seqmix_conv_desc** out) {
    if (!params || !out) return CONV2D_E_NULL;
    const seqmix_conv_params& p = *params;
    SM_TRY(check_seqs(p.tokens, p.seqs, p.slots));
    if (p.channels < 1 || p.width < 1) return CONV2D_E_INVALID;
    if (p.tokens > 1 && (p.x_row < p.channels || p.y_row < p.channels)) return CONV2D_E_INVALID;
    if (!known_dtype(p.dtype) || (p.act != SEQMIX_ACT_NONE && p.act != SEQMIX_ACT_SILU) ||
        p.width > SEQMIX_MAX_CONV_WIDTH || p.channels > kMaxRows - 4096)
        return CONV2D_E_UNSUPPORTED;
    seqmix_conv_desc* d = new (std::nothrow) seqmix_conv_desc{p};
    if (!d) return CONV2D_E_ALLOC;
    *out = d;
    return CONV2D_OK;
}

int seqmix_conv_desc_destroy(seqmix_conv_desc* d) {
    delete d;
    return CONV2D_OK;
}

int seqmix_conv_fwd(const seqmix_conv_desc* d, const void* x, const void* w, const float* bias, const int64_t* offsets,
                    const int32_t* slot_index, const void* window_in, void* window_out, void* y, void* stream) {
    if (!d) return CONV2D_E_NULL;
    const seqmix_conv_params& p = d->p;
    if (!w || (p.has_bias && !bias) || (p.tokens > 0 && (!x || !y))) return CONV2D_E_NULL;
    ConvArgs a{};
    SM_TRY(seq_args(p.tokens, p.seqs, p.slots, offsets, slot_index, &a.sq));
    a.x = x;
    a.w = w;
    a.bias = p.has_bias ? bias : nullptr;
    a.win_in = p.width > 1 ? window_in : nullptr;
    a.win_out = p.width > 1 ? window_out : nullptr;
    a.y = y;
    a.x_row = p.x_row;
    a.y_row = p.y_row;
    a.channels = (int32_t)p.channels;
    a.width = p.width;
    a.silu = p.act == SEQMIX_ACT_SILU;
    a.past = p.tokens * p.channels * esize(p.dtype) >= kPastBytes;
    return launch_token_conv(a, p.dtype, static_cast<hipStream_t>(stream)) == hipSuccess ? CONV2D_OK : CONV2D_E_HIP;
}

// ------------------------------------------------------------------ norms
int seqmix_norm_desc_create(const seqmix_norm_params* params, seqmix_norm_desc** out) {
    if (!params || !out) return CONV2D_E_NULL;
    const seqmix_norm_params& p = *params;
    if (p.rows < 0 || p.width < 1 || p.group < 1 || p.width % p.group != 0 || p.gate_run < 1) return CONV2D_E_INVALID;
    if (!(p.post_eps >= 0.0f) || !(p.pre_eps >= 0.0f)) return CONV2D_E_INVALID;
    if (p.u_row < p.width || (p.gate != SEQMIX_ACT_NONE && p.gate_row < p.width) ||
        (p.residual && p.res_row < p.width) || p.y_row < p.width ||
        (p.pre != SEQMIX_NORM_NONE && p.h_row < p.width))
        return CONV2D_E_INVALID;
    if (!known_dtype(p.dtype) || !known_dtype(p.res_dtype) || (p.dtype == CONV2D_F32 && p.res_dtype != CONV2D_F32) ||
        p.post < SEQMIX_NORM_NONE || p.post > SEQMIX_NORM_LAYER || p.pre < SEQMIX_NORM_NONE ||
        p.pre > SEQMIX_NORM_LAYER || p.gate < SEQMIX_ACT_NONE || p.gate > SEQMIX_ACT_LINEAR)
        return CONV2D_E_UNSUPPORTED;
    if (p.group > SEQMIX_MAX_NORM_WIDTH || p.rows > kMaxRows || p.width > kMaxRows ||
        (p.pre != SEQMIX_NORM_NONE && p.group != p.width))
        return CONV2D_E_UNSUPPORTED;
    seqmix_norm_desc* d = new (std::nothrow) seqmix_norm_desc{p};
    if (!d) return CONV2D_E_ALLOC;
    *out = d;
    return CONV2D_OK;
}

int seqmix_norm_desc_destroy(seqmix_norm_desc* d) {
    delete d;
    return CONV2D_OK;
}

int seqmix_norm_fwd(const seqmix_norm_desc* d, const void* u, const float* post_w, const float* post_b, const void* gate,
                    const void* residual, const float* scale_vec, const float* pre_w, const float* pre_b, void* y,
                    void* h, void* stream) {
    if (!d) return CONV2D_E_NULL;
    const seqmix_norm_params& p = d->p;
    const bool post = p.post != SEQMIX_NORM_NONE, pre = p.pre != SEQMIX_NORM_NONE;
    if ((post && (!post_w || (p.post_bias && !post_b))) || (p.scale_vec && !scale_vec) ||
        (pre && (!pre_w || (p.pre_bias && !pre_b))))
        return CONV2D_E_NULL;
    if (p.rows > 0 && (!u || (p.gate != SEQMIX_ACT_NONE && !gate) || (p.residual && !residual) || (pre && !h) ||
                       (!pre && !y)))
        return CONV2D_E_NULL;
    if (pre && h == y && p.rows > 0) return CONV2D_E_INVALID;
    NormArgs a{};
    a.u = u;
    a.post_w = post ? post_w : nullptr;
    a.post_b = post && p.post_bias ? post_b : nullptr;
    a.gate = p.gate != SEQMIX_ACT_NONE ? gate : nullptr;
    a.res = p.residual ? residual : nullptr;
    a.scale_vec = p.scale_vec ? scale_vec : nullptr;
    a.pre_w = pre ? pre_w : nullptr;
    a.pre_b = pre && p.pre_bias ? pre_b : nullptr;
    a.y = y;
    a.h = pre ? h : nullptr;
    a.ngroups = (int32_t)(p.width / p.group);
    a.rows = p.rows * a.ngroups;
    a.group = (int32_t)p.group;
    a.by_groups = make_fastdiv((uint32_t)a.ngroups);
    a.by_run = make_fastdiv((uint32_t)std::min(p.gate_run, kMaxRows));
    a.u_row = p.u_row, a.gate_row = p.gate_row, a.res_row = p.res_row, a.y_row = p.y_row, a.h_row = p.h_row;
    a.post = p.post;
    a.gate_act = p.gate;
    a.gate_first = p.gate_first;
    a.pre = p.pre;
    a.scale = p.scale;
    a.post_eps = p.post_eps;
    a.pre_eps = p.pre_eps;
    a.past = p.rows * p.width * ((y ? esize(p.res_dtype) : 0) + (pre ? esize(p.dtype) : 0)) >= kPastBytes;
    return launch_norm(a, p.dtype, p.res_dtype, static_cast<hipStream_t>(stream)) == hipSuccess ? CONV2D_OK
                                                                                               : CONV2D_E_HIP;
}

}  // extern "C"
