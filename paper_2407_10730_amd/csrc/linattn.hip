// linattn.hip -- linear attention with a decay per head, token by token, and the joining of segments.
//
//   S_t = exp(g_t) S_{t-1} + k_t v_t^T        o_t = scale q_t S_t
#include "seqmix_device.h"

namespace cv {

// One workgroup runs one sequence, head and block of DVB columns of the state through all tokens, the state in
// registers: thread (rg, cg) holds RPT neighbouring rows of 4 columns.  Bound by reading and writing the state (8 dk dv
// bytes per head against 4 dk dv operations per token), so it is the kernel of one or two tokens: 256 sequences, 16
// heads of 128 x 128 in 105 us (537 MB of states, 5.1 TB/s); 8 sequences in 4.9, a launch and one chain of loads. All
// loads are wide at any alignment: a thread whose columns pass the last one moves down to the last four, and owns those
// from `skip` on only; what it computes of the others is not used (128 sequences, 16 heads of 128 x 189: 101 us, with
// such rows read by elements 170; of 131 x 130: 86, 262).
template <typename T, typename TO, int DVB, int RPT>
__global__ __launch_bounds__(256) void attn_tokens_kernel(AttnArgs A) {
    constexpr int LR = DVB / 4;  // threads across the columns
    __shared__ float red[2][4][DVB];
    const int t = threadIdx.x, cg = t % LR, rg = t / LR;
    const uint32_t bh = blockIdx.x / (uint32_t)A.ndvb;
    const int blk = (int)(blockIdx.x - bh * A.ndvb);
    const int seq = (int)(bh / (uint32_t)A.heads), head = (int)(bh - (uint32_t)seq * A.heads);
    const SeqRange r = seq_range(A.sq, seq);
    const int r0 = rg * RPT, nc = min(4, A.dv - blk * DVB - cg * 4);  // owned columns (none: below 1)
    const int skip = A.dv >= 4 && nc > 0 ? 4 - nc : 0, jend = skip + nc;
    const int c0 = blk * DVB + cg * 4 - skip;
    const int nr = nc > 0 ? max(0, min(RPT, A.dk - r0)) : 0;  // owned rows

    const int qh = head / A.rep;
    const T* q = static_cast<const T*>(A.q) + r.first * A.q_row + qh * A.q_head + r0;
    const T* k = static_cast<const T*>(A.k) + r.first * A.k_row + qh * A.k_head + r0;
    const T* v = static_cast<const T*>(A.v) + r.first * A.v_row + head * A.v_head + c0;
    const float* g = A.g ? A.g + r.first * A.g_row + head : nullptr;
    TO* o = static_cast<TO*>(A.o) + r.first * A.o_row + head * A.o_head + blk * DVB;
    float kk[RPT], qq[RPT], vv[4], gg = 0.0f;
    auto load = [&] {  // the token at the pointers
        if (nr == RPT) {
            load_pack<T, RPT>(k, kk);
            load_pack<T, RPT>(q, qq);
        } else {
#pragma unroll
            for (int i = 0; i < RPT; ++i) {
                kk[i] = i < nr ? to_f32(k[i]) : 0.0f;
                qq[i] = i < nr ? to_f32(q[i]) : 0.0f;
            }
        }
        if (jend == 4) {
            load_pack<T, 4>(v, vv);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) vv[j] = j < jend ? to_f32(v[j]) : 0.0f;
        }
        if (g) gg = *g;
    };
    if (r.len > 0) load();  // under way while the slot, and then the state, are looked up

    const int64_t slot = seq_slot(A.sq, seq);
    if (slot < 0) return;
    const int64_t soff = (slot * A.heads + head) * A.dk * A.dv;
    const uint32_t row = (uint32_t)A.dv * 4, size = (uint32_t)A.dk * row;  // bytes; rows past dk are out of range
    const uint32_t at = nc > 0 ? (uint32_t)r0 * row + c0 * 4 : OOB_OFF;
    const __amdgpu_buffer_rsrc_t rin = make_rsrc(A.s_in ? A.s_in + soff : nullptr, A.s_in ? size : 0u);
    f32x4 S[RPT];
    if (A.dv >= 4) {
#pragma unroll
        for (int i = 0; i < RPT; ++i)
            S[i] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(rin, at + i * row, 0, 0));
    } else {
#pragma unroll
        for (int i = 0; i < RPT; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) S[i][j] = ld_f32(rin, j < jend ? at + i * row + j * 4 : OOB_OFF);
    }

#pragma unroll 1
    for (int64_t n = 0; n < r.len; ++n) {
        const float d = g ? __builtin_amdgcn_exp2f((float)decay_log2(gg)) : 1.0f;
        float acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        auto update = [&](int rows) {
#pragma unroll
            for (int i = 0; i < RPT; ++i)
                if (i < rows) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        S[i][j] = fmaf(kk[i], vv[j], S[i][j] * d);
                        acc[j] = fmaf(qq[i], S[i][j], acc[j]);
                    }
                }
        };
        if (nr == RPT)
            update(RPT);
        else  // rows past dk stay out of the sums: 0 * infinity is no zero
            update(nr);
        if (n + 1 < r.len) {
            q += A.q_row;
            k += A.k_row;
            v += A.v_row;
            if (g) g += A.g_row;
            load();
        }
#pragma unroll
        for (int m = LR; m < 64; m <<= 1)
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[j] += __shfl_xor(acc[j], m);
        float(*rd)[DVB] = red[n & 1];  // two buffers: one barrier per token
        if ((t & 63) < LR) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (j >= skip) rd[t >> 6][cg * 4 + j - skip] = acc[j];
        }
        __syncthreads();
        if (t < DVB && blk * DVB + t < A.dv)
            o[t] = from_f32<TO>(A.scale * ((rd[0][t] + rd[1][t]) + (rd[2][t] + rd[3][t])));
        o += A.o_row;
    }
    if (!A.s_out) return;
    const __amdgpu_buffer_rsrc_t rout = make_rsrc(A.s_out + soff, size);
    if (nc >= 4) {
#pragma unroll
        for (int i = 0; i < RPT; ++i)
            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, S[i]), rout, at + i * row, 0, 0);
    } else if (nc > 0) {
#pragma unroll
        for (int i = 0; i < RPT; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) st_f32(rout, j >= skip && j < jend ? at + i * row + j * 4 : OOB_OFF, S[i][j]);
    }
}

template <typename T, typename TO, int DVB, int DK>
static void launch_tokens_r(const AttnArgs& a, dim3 grid, hipStream_t s) {
    constexpr int RPT = DK * DVB / 1024;
    hipLaunchKernelGGL((attn_tokens_kernel<T, TO, DVB, RPT>), grid, dim3(256), 0, s, a);
}

template <typename T, typename TO, int DVB>
static hipError_t launch_tokens_b(const AttnArgs& a, hipStream_t s) {
    const int64_t blocks = (int64_t)a.sq.seqs * a.heads * a.ndvb;
    if (blocks > 0x7fffffffLL) return hipErrorInvalidValue;
    const dim3 grid((unsigned)blocks);
    if (a.dk <= 32)
        launch_tokens_r<T, TO, DVB, 32>(a, grid, s);
    else if (a.dk <= 64)
        launch_tokens_r<T, TO, DVB, 64>(a, grid, s);
    else if (a.dk <= 128)
        launch_tokens_r<T, TO, DVB, 128>(a, grid, s);
    else
        launch_tokens_r<T, TO, DVB, 256>(a, grid, s);
    return hipGetLastError();
}

template <typename T, typename TO>
static hipError_t launch_tokens_t(const AttnArgs& a, hipStream_t s) {
    return a.block == kTokensBlock ? launch_tokens_b<T, TO, kTokensBlock>(a, s)
                                   : launch_tokens_b<T, TO, kTokensWide>(a, s);
}

hipError_t launch_attn_tokens(const AttnArgs& a, int dt, int odt, hipStream_t s) {
    if (dt == CONV2D_F32) return launch_tokens_t<float, float>(a, s);
    return odt == CONV2D_F32 ? launch_tokens_t<uint16_t, float>(a, s) : launch_tokens_t<uint16_t, uint16_t>(a, s);
}

// Joins the segments of each sequence: ws_state holds the state that each segment but the last adds from
// zero; afterwards it holds the state that each segment starts from.  One thread owns V neighbouring elements of a state (from
// e on) and walks along the segments, AHEAD loads ahead of the sum.  Bound by its bytes, 8 dk dv per segment and head (16
// segments, 16 heads of 128 x 128: 8.1 us, 33 MB from the caches).
template <int V>
__device__ __forceinline__ void join_elements(const AttnArgs& A, int seq, int64_t e) {
    constexpr int AHEAD = 8;
    const int64_t size = (int64_t)A.dk * A.dv;
    const int head = blockIdx.y;
    const SeqRange r = seq_range(A.sq, seq);
    const uint32_t seg = (uint32_t)A.segment;
    if (r.len <= A.alone) return;  // starts from its own state
    const int64_t slot = seq_slot(A.sq, seq);
    if (slot < 0) return;
    const int64_t first = (uint32_t)A.ws_mul * (uint32_t)r.first / seg;
    const int parts = (int)min<int64_t>(((uint32_t)r.len + seg - 1) / seg, A.nws - first);
    float S[V];
#pragma unroll
    for (int v = 0; v < V; ++v) S[v] = 0.0f;
    if (A.s_in) load_pack<float, V>(A.s_in + (slot * A.heads + head) * size + e, S);
    const int64_t pitch = (int64_t)A.heads * size;
    float* ws = A.ws_state + (first * A.heads + head) * size + e;
    const float* wd = A.ws_decay + first * A.heads + head;
    for (int p = 0; p < parts; p += AHEAD) {
        float add[AHEAD][V], d[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {  // (past the last that counts: that one again)
            const int from = max(min(p + u, parts - 2), 0);
            load_pack<float, V>(ws + from * pitch, add[u]);
            d[u] = wd[(int64_t)from * A.heads];
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
            if (p + u < parts) {
                store_pack<float, V>(ws + (p + u) * pitch, S);
                if (fabsf(d[u]) <= 100.0f) {
                    const float f = __builtin_amdgcn_exp2f(d[u]);
#pragma unroll
                    for (int v = 0; v < V; ++v) S[v] = fmaf(f, S[v], add[u][v]);
                } else {
                    // exp2(d) in three factors within 2^+-100: together they take every float but zero out of the range, so the
                    // rest of d is not missed, and a state of zeros stays one under any growth
                    float f[3], rest = d[u];
#pragma unroll
                    for (int x = 0; x < 3; ++x) {
                        const float part = rest > 100.0f ? 100.0f : rest < -100.0f ? -100.0f : rest;
                        f[x] = __builtin_amdgcn_exp2f(part);
                        rest -= part;
                    }
#pragma unroll
                    for (int v = 0; v < V; ++v) S[v] = fmaf(S[v] * f[0] * f[1], f[2], add[u][v]);
                }
            }
    }
}

// Four elements per thread, and one in the threads of the last three.
__global__ __launch_bounds__(256) void attn_join_kernel(AttnArgs A) {
    const int size = A.dk * A.dv, i = blockIdx.x * 256 + threadIdx.x, packs = size / 4;
    for (int seq = blockIdx.z; seq < A.sq.seqs; seq += gridDim.z) {
        if (i < packs)
            join_elements<4>(A, seq, 4 * i);
        else if (i < packs + size % 4)
            join_elements<1>(A, seq, 3 * packs + i);
    }
}

hipError_t launch_attn_join(const AttnArgs& a, hipStream_t s) {
    const int size = a.dk * a.dv;
    if (a.heads > 65535) return hipErrorInvalidValue;
    // (most sequences of a large batch are not cut: 16 workgroups per CU share them)
    const int blocks = (size / 4 + size % 4 + 255) / 256;
    const int64_t across = std::max<int64_t>(16 * kSeqmixCUs / ((int64_t)blocks * a.heads), 1);
    const dim3 grid((unsigned)blocks, (unsigned)a.heads, (unsigned)std::min<int64_t>(across, a.sq.seqs));
    hipLaunchKernelGGL(attn_join_kernel, grid, dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace cv
