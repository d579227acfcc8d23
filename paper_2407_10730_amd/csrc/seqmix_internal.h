// seqmix_internal.h -- shared declarations of the token-mixing operators (seqmix.h).
#pragma once

#include "conv2d_internal.h"
#include "seqmix.h"

namespace cv {

// Results of this many bytes or more are written past the caches: 8192 x 4096 bf16 convolution 31.8 -> 26.3 us, 8192 x 2048 norm
// with residual 34.0 -> 26.4 us, 2048 rows of the two 12.4 -> 10.6 and 11.3 -> 9.6 us.  The operators after them do
// not miss it (a layer over 8496 tokens 297 us, 296 with it): the XCDs' L2s hold little of what others wrote.
constexpr int64_t kPastBytes = 4LL << 20;
constexpr int kSeqmixCUs = 256;  // plans are made without a GPU: MI355X has 256 CUs

// How the rows of a call divide into sequences, and which pool entry each has.
struct SeqArgs {
    const int64_t* off;   // [seqs + 1] or NULL: seq_len rows each
    const int32_t* slot;  // [seqs] or NULL: slot i
    int64_t tokens, seq_len, slots;
    int32_t seqs;
};

// Parts of `size` tokens of a sequence (an empty one has one), and the ids that number the parts of all sequences.
inline int64_t seq_parts(int64_t len, int64_t size) {
    return len > size ? (len + size - 1) / size : 1;
}
inline int64_t seq_part_ids(const SeqArgs& a, int64_t size) {
    return a.off ? a.tokens / size + a.seqs : (int64_t)a.seqs * seq_parts(a.seq_len, size);
}

struct AttnArgs {
    SeqArgs sq;
    const void *q, *k, *v;
    const float* g;
    const float* s_in;
    float* s_out;
    void* o;
    int64_t q_row, q_head, k_row, k_head, v_row, v_head, o_row, o_head;
    int64_t g_row;        // heads (a decay for each token) or 0
    int32_t heads, rep;   // rep heads share a q/k head
    int32_t dk, dv;
    int32_t block, ndvb;  // state columns per workgroup, such blocks per head
    float scale;
    int32_t vec;          // dk and dv are multiples of 16 bytes of q, k and v
    // Sequences of more than `alone` tokens (more than `segment`) are cut in segments: ids offsets[i] / segment + i +
    // (segment of sequence i), of which only the first has work where a sequence is not cut.  Only cut ones have a place
    // in the workspace, ws_mul * offsets[i] / segment + (segment of sequence i): with ws_mul 2 the ranges of two cut
    // sequences are apart, as 2 len / segment, rounded down, is at least len / segment, rounded up.
    int64_t segment, alone, nseg, nws;
    int32_t ws_mul;
    int32_t places;       // the ids of this pass number places of the workspace
    int64_t ids;          // of this pass: sequences, segments or places
    int32_t unit, units;  // workgroups of an id that stay on one XCD, such units per id
    float* ws_state;      // [nws][heads][dk][dv]
    float* ws_decay;      // [nws][heads]: log of a segment's whole decay, times log2(e)
};

constexpr int kTokensBlock = 32, kTokensWide = 128;  // state columns of a workgroup of the token kernel
hipError_t launch_attn_tokens(const AttnArgs& a, int dt, int odt, hipStream_t s);

// Chunk kernels: 64 or 128 state columns per workgroup.  state_only: the states that segments add from zero
// (all but the last of each sequence) into ws_state / ws_decay; launch_attn_join turns them into
// the states that the segments start from, which the full pass reads.
constexpr int kChunk = 64, kChunkF32 = 32;
hipError_t launch_attn_chunks_bf16(const AttnArgs& a, int odt, bool state_only, hipStream_t s);
hipError_t launch_attn_chunks_f32(const AttnArgs& a, bool state_only, hipStream_t s);
hipError_t launch_attn_join(const AttnArgs& a, hipStream_t s);

struct ConvArgs {
    SeqArgs sq;
    const void *x, *w;
    const float* bias;
    const void* win_in;
    void* win_out;
    void* y;
    int64_t x_row, y_row;
    int32_t channels, width, silu;
    int32_t past;         // y is written past the caches
};
hipError_t launch_token_conv(const ConvArgs& a, int dt, hipStream_t s);

struct NormArgs {
    const void* u;
    const float *post_w, *post_b;
    const void* gate;
    const void* res;
    const float *scale_vec, *pre_w, *pre_b;
    void *y, *h;
    int64_t rows;         // rows * groups of the call
    int32_t group, ngroups;
    FastDiv by_groups, by_run;  // rows below 2^31
    int64_t u_row, gate_row, res_row, y_row, h_row;
    int32_t post, gate_act, gate_first, pre;
    float scale, post_eps, pre_eps;
    int32_t past;
};
hipError_t launch_norm(const NormArgs& a, int dt, int rdt, hipStream_t s);

}  // namespace cv
