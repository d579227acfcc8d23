// linattn_device.h -- what the chunk kernels of linear attention share.
#pragma once

#include "seqmix_device.h"

namespace cv {

typedef double f64x2 __attribute__((ext_vector_type(2)));

// What a workgroup of a chunk kernel runs: tokens [row0, row0 + len) for one head and block of columns.
struct AttnPlace {
    int head, blk;
    int64_t ws;  // place in the workspace (of a cut sequence)
    int64_t slot, row0, len;
    bool cut, last;  // a segment; the end of its sequence
};
// False: nothing (in all threads of the workgroup).  Heads that share q and k, and their column blocks, go to the same
// XCD, where they share them in its L2; these units go to the XCDs in turn, as ids without work may lie side by side (8
// sequences of 200 tokens, 16 heads of 128 x 128: 29 us, with neighbouring ids on one XCD 39).
__device__ __forceinline__ bool attn_place(const AttnArgs& A, bool state_only, AttnPlace* out) {
    const uint32_t j = blockIdx.x / 8, round = j / (uint32_t)A.unit, u = blockIdx.x % 8 + 8 * round;
    const int id = u / (uint32_t)A.units;
    if (id >= A.ids) return false;
    const uint32_t at = (u - id * A.units) * A.unit + (j - round * A.unit);
    out->head = at / (uint32_t)A.ndvb;
    out->blk = at - out->head * A.ndvb;
    SeqPart sp{id, 0};
    if (A.segment) sp = seq_part(A.sq, id, (uint32_t)A.segment, A.places, A.ws_mul);
    if (sp.seq >= A.sq.seqs || sp.part < 0) return false;
    const SeqRange r = seq_range(A.sq, sp.seq);
    const int64_t start = sp.part * A.segment;
    out->cut = A.segment && r.len > A.alone;
    if (sp.part > 0 && (!out->cut || start >= r.len)) return false;  // (the first of these where none is left)
    out->last = !out->cut || r.len - start <= A.segment;
    out->ws = out->cut ? (uint32_t)A.ws_mul * (uint32_t)r.first / (uint32_t)A.segment + sp.part : 0;
    if (state_only && out->last) return false;
    out->slot = seq_slot(A.sq, sp.seq);
    out->len = out->last ? r.len - start : A.segment;
    out->row0 = r.first + start;
    return out->slot >= 0;
}
__device__ __forceinline__ const float* attn_first_state(const AttnArgs& A, const AttnPlace& p) {
    const int64_t size = (int64_t)A.dk * A.dv;
    if (p.cut) return A.ws_state + (p.ws * A.heads + p.head) * size;
    return A.s_in ? A.s_in + (p.slot * A.heads + p.head) * size : nullptr;
}
__device__ __forceinline__ float* attn_last_state(const AttnArgs& A, const AttnPlace& p, bool state_only) {
    const int64_t size = (int64_t)A.dk * A.dv;
    if (state_only) return A.ws_state + (p.ws * A.heads + p.head) * size;
    return p.last && A.s_out ? A.s_out + (p.slot * A.heads + p.head) * size : nullptr;
}

// Log decay of the lane's token in a chunk of n tokens that starts at g; 0 past its end and without decays.
__device__ __forceinline__ float load_decay(const AttnArgs& A, const float* g, int64_t c, int lane, int n) {
    const __amdgpu_buffer_rsrc_t r = make_rsrc(g + c * A.g_row, g ? OOB_OFF - 1 : 0u);
    return ld_f32(r, lane < n ? (uint32_t)lane * (uint32_t)A.g_row * 4u : OOB_OFF);
}

// One wave: the decays of a chunk of up to 64 tokens (g of this lane's token, 0 past the chunk).  sB: running sums in
// log2, in 64 bits, so that differences of sums stay exact after decays that clear the state; sD their
// exponentials; sE the exponentials of what is left to the chunk's end.  Returns the whole chunk's.
__device__ __forceinline__ double chunk_decays(float g, int lane, double* sB, float* sD, float* sE, int size) {
    double b = decay_log2(g);
    // inclusive scan by lane moves: 1, 2, 4 and 8 lanes up within rows of 16, then the rows' sums
#define SCAN_STEP(ctrl, rows)                                                                            \
    {                                                                                                    \
        const u32x2 w = __builtin_bit_cast(u32x2, b);                                                    \
        b += __builtin_bit_cast(double, u32x2{(uint32_t)__builtin_amdgcn_update_dpp(0, w[0], ctrl, rows, 0xf, false),  \
                                              (uint32_t)__builtin_amdgcn_update_dpp(0, w[1], ctrl, rows, 0xf, false)}); \
    }
    SCAN_STEP(0x111, 0xf)
    SCAN_STEP(0x112, 0xf)
    SCAN_STEP(0x114, 0xf)
    SCAN_STEP(0x118, 0xf)
    SCAN_STEP(0x142, 0xa)
    SCAN_STEP(0x143, 0xc)
#undef SCAN_STEP
    const u32x2 w = __builtin_bit_cast(u32x2, b);
    const double tot = __builtin_bit_cast(double, u32x2{(uint32_t)__builtin_amdgcn_readlane(w[0], 63),
                                                        (uint32_t)__builtin_amdgcn_readlane(w[1], 63)});
    if (lane < size) {
        sB[lane] = b;
        sD[lane] = __builtin_amdgcn_exp2f((float)b);
        sE[lane] = __builtin_amdgcn_exp2f((float)(tot - b));
    }
    return tot;
}

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
}

// Rows of a chunk are loaded through range-checked buffers, which read zero outside their range: the range ends with
// the chunk's last row, and columns past the end go to OOB_OFF, so no load needs a branch or a mask and all
// loads of a chunk are in flight together.  `n` rows of `dim` elements, `row` elements apart (row >= dim).
template <typename T>
__device__ __forceinline__ __amdgpu_buffer_rsrc_t chunk_rsrc(const T* p, int n, uint32_t row, int dim) {
    return make_rsrc(p, ((uint32_t)(n - 1) * row + (uint32_t)dim) * (uint32_t)sizeof(T));
}

// A thread's 16 bytes of a row of `dim` elements, from column `col` on; loads at any address of the element's alignment are
// whole.  VEC: dim is a multiple of 16 bytes.  Otherwise the last part is read where it ends with the row, and moved down by
// `shift` bits, which brings in zeros, when it is used (row_part_of); rows below 16 bytes are read by elements.
// 5664 tokens in 10 sequences, 12 heads of 84 x 100 bf16: 56 us, all by elements 93; 8192 tokens, 16 heads of
// 127 x 127: 94 us, 151.
template <typename T, bool VEC>
__device__ __forceinline__ uint32_t row_part(uint32_t first, int col, int dim, uint32_t* shift) {
    constexpr int U = 16 / sizeof(T);
    const int live = dim - col;
    const bool cut = !VEC && live > 0 && live < U && dim >= U;
    *shift = cut ? (U - live) * (8 * sizeof(T)) : 0;
    return live > 0 ? (first + (cut ? dim - U : col)) * (uint32_t)sizeof(T) : OOB_OFF;
}
template <typename T, bool VEC>
__device__ __forceinline__ u32x4 load_row(__amdgpu_buffer_rsrc_t r, uint32_t off, int dim) {
    if (VEC || dim >= (int)(16 / sizeof(T))) return __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, 0);
    u32x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4)
            v[i] = __builtin_amdgcn_raw_buffer_load_b32(r, i < dim ? off + 4 * i : OOB_OFF, 0, 0);
        else
            v[i] = (uint32_t)ld_u16(r, 2 * i < dim ? off + 4 * i : OOB_OFF) |
                   (uint32_t)ld_u16(r, 2 * i + 1 < dim ? off + 4 * i + 2 : OOB_OFF) << 16;
    }
    return v;
}
template <typename T, bool VEC>
__device__ __forceinline__ u32x4 row_part_of(u32x4 v, uint32_t shift) {
    if constexpr (!VEC) {
        if (shift & 64) v = u32x4{v[2], v[3], 0, 0};
        if (shift & 32) v = u32x4{v[1], v[2], v[3], 0};
        if constexpr (sizeof(T) == 2)
            v = u32x4{__builtin_amdgcn_alignbit(v[1], v[0], shift & 16), __builtin_amdgcn_alignbit(v[2], v[1], shift & 16),
                      __builtin_amdgcn_alignbit(v[3], v[2], shift & 16), v[3] >> (shift & 16)};
    }
    return v;
}

// Column c of a state as MFMA results hold it: tile m has rows QS quad + i from its first row on; odd tiles begin TS rows
// after even ones, pairs 32 rows apart.  Rows past dk lie past the buffer's range.
template <int QS, int TS, int MT>
__device__ __forceinline__ void load_state(const AttnArgs& A, const float* p, int c, int quad, f32x4 (&S)[MT]) {
    const __amdgpu_buffer_rsrc_t r = make_rsrc(p, p ? (uint32_t)(A.dk * A.dv * 4) : 0u);
    const uint32_t row = (uint32_t)A.dv * 4;
    const uint32_t at = c < A.dv ? QS * quad * row + c * 4 : OOB_OFF;
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i) S[m][i] = ld_f32(r, at + (m / 2 * 32 + m % 2 * TS + i) * row);
}
template <int QS, int TS, int MT>
__device__ __forceinline__ void store_state(const AttnArgs& A, float* p, int c, int quad, const f32x4 (&S)[MT]) {
    const __amdgpu_buffer_rsrc_t r = make_rsrc(p, (uint32_t)(A.dk * A.dv * 4));
    uint32_t row = (uint32_t)A.dv * 4;
    asm volatile("" : "+s"(row));  // or the addresses of the load would be kept in registers until here
    const uint32_t at = c < A.dv ? QS * quad * row + c * 4 : OOB_OFF;
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i) st_f32(r, at + (m / 2 * 32 + m % 2 * TS + i) * row, S[m][i]);
}

// Results of a chunk of n tokens that starts at token c of the segment, scaled and rounded: tile it holds tokens 16 it + l16,
// columns col .. col + 3 (those at or past dv are none).
template <int IT, bool VEC, bool F32>
__device__ __forceinline__ void attn_store(const AttnArgs& A, const AttnPlace& pl, int64_t c, int n, int col, int l16,
                                           const f32x4 (&O)[IT]) {
    const int64_t first = (pl.row0 + c) * A.o_row + pl.head * A.o_head;
    const uint32_t row = (uint32_t)A.o_row, at = (uint32_t)l16 * row + col;
    const int live = A.dv - col;
    if constexpr (F32) {
        const __amdgpu_buffer_rsrc_t r = chunk_rsrc(static_cast<float*>(A.o) + first, n, row, A.dv);
#pragma unroll
        for (int it = 0; it < IT; ++it) {
            const f32x4 v = O[it] * A.scale;
            if (VEC || live <= 0 || live >= 4) {
                __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v), r,
                                                       live > 0 ? (at + it * 16 * row) * 4 : OOB_OFF, 0, 0);
            } else {
#pragma unroll
                for (int x = 0; x < 3; ++x) st_f32(r, x < live ? (at + it * 16 * row + x) * 4 : OOB_OFF, v[x]);
            }
        }
    } else {
        const __amdgpu_buffer_rsrc_t r = chunk_rsrc(static_cast<uint16_t*>(A.o) + first, n, row, A.dv);
#pragma unroll
        for (int it = 0; it < IT; ++it) {
            const f32x4 v = O[it] * A.scale;
            const u32x2 w{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
            if (VEC || live <= 0 || live >= 4) {
                __builtin_amdgcn_raw_buffer_store_b64(w, r, live > 0 ? (at + it * 16 * row) * 2 : OOB_OFF, 0, 0);
            } else {
#pragma unroll
                for (int x = 0; x < 3; ++x)
                    st_u16(r, x < live ? (at + it * 16 * row + x) * 2 : OOB_OFF, (uint16_t)(w[x / 2] >> (16 * (x & 1))));
            }
        }
    }
}

}  // namespace cv
