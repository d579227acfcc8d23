// linattn_device.h -- what the chunk kernels of linear attention share.
#pragma once

#include "seqmix_device.h"

namespace cv {

// What a workgroup of a chunk kernel runs: tokens [row0, row0 + len) for one head and block of columns.
struct AttnPlace {
    int head, blk;
    int64_t id, slot, row0, len;
    bool last;  // the end of its sequence
};
// False: nothing (in all threads of the workgroup).  Consecutive ids (column blocks, then heads, of the same tokens)
// go to the same XCD, where they share q and k in its L2.
__device__ __forceinline__ bool attn_place(const AttnArgs& A, bool state_only, AttnPlace* out) {
    const int bid = xcd_remap(blockIdx.x, gridDim.x);
    const int hid = bid / A.ndvb;
    out->blk = bid - hid * A.ndvb;
    out->id = hid / A.heads;
    out->head = hid - (int)out->id * A.heads;
    SeqPart sp{(int)out->id, 0, out->id};
    if (A.segment) sp = seq_part(A.sq, out->id, A.segment);
    if (sp.seq >= A.sq.seqs || sp.part < 0) return false;
    const SeqRange r = seq_range(A.sq, sp.seq);
    const int64_t start = sp.part * A.segment;
    if (sp.part > 0 && start >= r.len) return false;
    out->last = !A.segment || r.len - start <= A.segment;
    if (state_only && out->last) return false;
    out->slot = seq_slot(A.sq, sp.seq);
    out->len = out->last ? r.len - start : A.segment;
    out->row0 = r.first + start;
    return out->slot >= 0;
}
__device__ __forceinline__ const float* attn_first_state(const AttnArgs& A, const AttnPlace& p) {
    const int64_t size = (int64_t)A.dk * A.dv;
    if (A.segment) return A.ws_state + (p.id * A.heads + p.head) * size;
    return A.s_in ? A.s_in + (p.slot * A.heads + p.head) * size : nullptr;
}
__device__ __forceinline__ float* attn_last_state(const AttnArgs& A, const AttnPlace& p, bool state_only) {
    const int64_t size = (int64_t)A.dk * A.dv;
    if (state_only) return A.ws_state + (p.id * A.heads + p.head) * size;
    return p.last && A.s_out ? A.s_out + (p.slot * A.heads + p.head) * size : nullptr;
}

// One wave: the decays of a chunk of up to 64 tokens (g of this lane's token, 0 past the chunk).  sB: running sums in
// log2, in 64 bits, so that differences of sums stay exact after decays that clear the state; sD their
// exponentials; sE the exponentials of what is left to the chunk's end.  Returns the whole chunk's.
__device__ __forceinline__ double chunk_decays(float g, double* sB, float* sD, float* sE, int size) {
    const int lane = threadIdx.x & 63;
    double b = decay_log2(g);
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const double up = __shfl_up(b, d);
        if (lane >= d) b += up;
    }
    const double tot = __shfl(b, 63);
    if (lane < size) {
        sB[lane] = b;
        sD[lane] = __builtin_amdgcn_exp2f((float)b);
        sE[lane] = __builtin_amdgcn_exp2f((float)(tot - b));
    }
    return tot;
}

__device__ __forceinline__ bool finite(float x) { return fabsf(x) < __builtin_inff(); }

// N results of one token, scaled and rounded, to columns c .. c + N - 1 (those at or past dv are none).
template <int N>
__device__ __forceinline__ void attn_store(const AttnArgs& A, int o_f32, int64_t row, int head, int c, float (&e)[N]) {
    const int64_t at = row * A.o_row + head * A.o_head + c;
#pragma unroll
    for (int x = 0; x < N; ++x) e[x] *= A.scale;
    if (o_f32) {
        float* o = static_cast<float*>(A.o) + at;
        if (A.vec) {
            store_pack<float, N>(o, e);
        } else {
#pragma unroll
            for (int x = 0; x < N; ++x)
                if (c + x < A.dv) o[x] = e[x];
        }
    } else {
        uint16_t* o = static_cast<uint16_t*>(A.o) + at;
        if (A.vec) {
            store_pack<uint16_t, N>(o, e);
        } else {
#pragma unroll
            for (int x = 0; x < N; ++x)
                if (c + x < A.dv) o[x] = from_f32<uint16_t>(e[x]);
        }
    }
}

}  // namespace cv
