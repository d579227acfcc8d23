// linattn_chunks_f32.hip -- linear attention with a decay per head in chunks of 32 tokens, fp32 operands.
//
// The same four products per chunk and the same division of work as the bf16 kernel (linattn_chunks.hip), on the
// fp32 matrix instruction: nothing is rounded below fp32.  It multiplies at a sixteenth of the bf16 rate, which makes
// this kernel bound by it; 32 tokens per chunk halve the products within a chunk.  8192 tokens of 16 heads of 128 x 128: 161 us
// for all passes; 512 tokens of 2 heads: 19.
// Operand order: in step (m, u) of a reduction the lanes of quad q multiply index 16 m + 4 q + u, so that a lane's four
// steps are one 16-byte LDS read, and the state's registers are operands as they are.
#include "linattn_device.h"

namespace cv {

__device__ __forceinline__ f32x4 mfma_f32(float a, float b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}

// dk up to 64 DKT, 16 WAVES columns of v per workgroup; waves per SIMD that LDS leaves room for
constexpr int chunk_f32_occupancy(int dkt, int waves) { return waves == 8 ? (dkt <= 2 ? 4 : 2) : dkt <= 2 ? 3 : 2; }

template <int DKT, int WAVES, bool STATE_ONLY, bool VEC>
__global__ __launch_bounds__(64 * WAVES, chunk_f32_occupancy(DKT, WAVES)) void attn_chunks_f32_kernel(AttnArgs A) {
    constexpr int C = kChunkF32, DKP = 64 * DKT, DVB = 16 * WAVES, NTHR = 64 * WAVES;
    constexpr int QP = DKP + 4, VP = DVB + 4, PP = C + 4;  // LDS row pitches in floats
    constexpr int MT = DKP / 16;
    __shared__ __align__(16) float sQ[STATE_ONLY ? 1 : C * QP];
    __shared__ __align__(16) float sK[C * QP];
    __shared__ __align__(16) float sV[C * VP];
    __shared__ __align__(16) float sP[STATE_ONLY ? 1 : C * PP];
    __shared__ __align__(16) double sB[C];
    __shared__ __align__(16) float sE[C], sD[C];
    __shared__ float sTot;

    const int t = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    int lane = t & 63, l16 = lane & 15, quad = lane >> 4;
    AttnPlace pl;
    if (!attn_place(A, STATE_ONLY, &pl)) return;
    const int head = pl.head;
    const int64_t row0 = pl.row0, len = pl.len;
    const int c0 = pl.blk * DVB;      // first column of the workgroup
    const int wc = wave * 16;         // ... of the wave, within the workgroup's
    const int qh = head / A.rep;

    f32x4 S[MT];  // tile m: rows 16 m + 4 quad + i, column c0 + wc + l16
    load_state<4, 16>(A, STATE_ONLY ? nullptr : attn_first_state(A, pl), c0 + wc + l16, quad, S);

    constexpr int NQ = C * DKP / 4 / NTHR, NV = C * DVB / 4 / NTHR;  // 16-byte loads per thread
    constexpr int RS = NTHR / (DKP / 4), RSV = NTHR / (DVB / 4);
    const int lr = t / (DKP / 4), lc = t % (DKP / 4) * 4, lrv = t / (DVB / 4), lcv = t % (DVB / 4) * 4;
    const float* gq = static_cast<const float*>(A.q) + row0 * A.q_row + qh * A.q_head;
    const float* gk = static_cast<const float*>(A.k) + row0 * A.k_row + qh * A.k_head;
    const float* gv = static_cast<const float*>(A.v) + row0 * A.v_row + head * A.v_head;
    const float* gg = A.g ? A.g + row0 * A.g_row + head : nullptr;
    const uint32_t q_row = (uint32_t)A.q_row, k_row = (uint32_t)A.k_row, v_row = (uint32_t)A.v_row;
    uint32_t cut, cut_v;  // (of q, k and of v: row_part)
    uint32_t q_at = row_part<float, VEC>(lr * q_row, lc, A.dk, &cut);
    uint32_t k_at = row_part<float, VEC>(lr * k_row, lc, A.dk, &cut);
    uint32_t v_at = row_part<float, VEC>(lrv * v_row, c0 + lcv, A.dv, &cut_v);
    auto part_of = [](u32x4 v, uint32_t c) { return row_part_of<float, VEC>(v, c); };
    u32x4 rq[STATE_ONLY ? 1 : NQ], rk[NQ], rv[NV];
    float rg = 0.0f;
    auto load = [&](int64_t c) {
        const int n = (int)min<int64_t>(C, len - c);
        if constexpr (!STATE_ONLY) {
            const __amdgpu_buffer_rsrc_t r = chunk_rsrc(gq + c * A.q_row, n, q_row, A.dk);
#pragma unroll
            for (int i = 0; i < NQ; ++i) rq[i] = load_row<float, VEC>(r, q_at + i * (RS * 4) * q_row, A.dk);
        }
        const __amdgpu_buffer_rsrc_t r = chunk_rsrc(gk + c * A.k_row, n, k_row, A.dk);
        const __amdgpu_buffer_rsrc_t rr = chunk_rsrc(gv + c * A.v_row, n, v_row, A.dv);
#pragma unroll
        for (int i = 0; i < NQ; ++i) rk[i] = load_row<float, VEC>(r, k_at + i * (RS * 4) * k_row, A.dk);
#pragma unroll
        for (int i = 0; i < NV; ++i) rv[i] = load_row<float, VEC>(rr, v_at + i * (RSV * 4) * v_row, A.dv);
        if (wave == WAVES - 1) rg = load_decay(A, gg, c, lane, n);
    };

    double whole = 0.0;
    if (len > 0) load(0);
    for (int64_t c = 0; c < len; c += C) {
        const int n = (int)min<int64_t>(C, len - c);
        // what follows from these is cheaper computed again than kept in registers over the loop
        asm volatile("" : "+v"(q_at), "+v"(k_at), "+v"(v_at), "+v"(l16), "+v"(quad), "+v"(lane));
        if constexpr (!VEC) asm volatile("" : "+v"(cut), "+v"(cut_v));
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
            if constexpr (!STATE_ONLY) *reinterpret_cast<u32x4*>(&sQ[(lr + i * RS) * QP + lc]) = part_of(rq[i], cut);
            *reinterpret_cast<u32x4*>(&sK[(lr + i * RS) * QP + lc]) = part_of(rk[i], cut);
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) *reinterpret_cast<u32x4*>(&sV[(lrv + i * RSV) * VP + lcv]) = part_of(rv[i], cut_v);
        if (wave == WAVES - 1) {
            const double tot = chunk_decays(rg, lane, sB, sD, sE, C);
            if (lane == 0) sTot = __builtin_amdgcn_exp2f((float)tot);
            whole += tot;
        }
        __syncthreads();
        if (c + C < len) load(c + C);

        if constexpr (!STATE_ONLY) {
            // one 16x16 tile of scores per wave, transposed (a lane holds 4 neighbouring j of one i); the one above
            // the diagonal is never read
            const int it = (wave + 1) >> 1, jt = wave >> 1;  // (0,0) (1,0) (1,1), and a fourth wave without
            if (wave < 3) {
                f32x4 s{0, 0, 0, 0};
#pragma unroll
                for (int m = 0; m < MT; ++m) {
                    const f32x4 a = *reinterpret_cast<const f32x4*>(&sK[(16 * jt + l16) * QP + 16 * m + 4 * quad]);
                    const f32x4 b = *reinterpret_cast<const f32x4*>(&sQ[(16 * it + l16) * QP + 16 * m + 4 * quad]);
#pragma unroll
                    for (int u = 0; u < 4; ++u) s = mfma_f32(a[u], b[u], s);
                }
                const int i = 16 * it + l16;
                const double bi = sB[i];
                const int j = 16 * jt + 4 * quad;
                const f64x2 b01 = *reinterpret_cast<const f64x2*>(&sB[j]), b23 = *reinterpret_cast<const f64x2*>(&sB[j + 2]);
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const bool on = j + u <= i;
                    const float f = (float)(bi - (u < 2 ? b01[u] : b23[u - 2]));
                    s[u] = (on ? s[u] : 0.0f) * __builtin_amdgcn_exp2f(on ? f : 0.0f);
                }
                *reinterpret_cast<f32x4*>(&sP[i * PP + j]) = s;
            }
        }
        if constexpr (!STATE_ONLY) __syncthreads();
        float vf[2][4];  // v of token 16 h + 4 quad + u
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int u = 0; u < 4; ++u) vf[h][u] = sV[(16 * h + 4 * quad + u) * VP + wc + l16];
        if constexpr (!STATE_ONLY) {
            f32x4 O[2];  // transposed: rows are columns of v, columns the 16 tokens of a tile
            // exp(b_i) q_i S
#pragma unroll
            for (int it = 0; it < 2; ++it) O[it] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                f32x4 b[2];
#pragma unroll
                for (int it = 0; it < 2; ++it)
                    b[it] = *reinterpret_cast<const f32x4*>(&sQ[(16 * it + l16) * QP + 16 * m + 4 * quad]);
#pragma unroll
                for (int u = 0; u < 4; ++u)
#pragma unroll
                    for (int it = 0; it < 2; ++it) O[it] = mfma_f32(S[m][u], b[it][u], O[it]);
            }
#pragma unroll
            for (int it = 0; it < 2; ++it) O[it] *= sD[16 * it + l16];
            // zero scores above the diagonal times an infinite or NaN v are NaN: sum without those terms
            uint32_t top = 0;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int u = 0; u < 4; ++u) top = max(top, __builtin_bit_cast(uint32_t, vf[h][u]) & 0x7fffffffu);
            if (__any(top >= 0x7f800000u)) {
#pragma unroll
                for (int it = 0; it < 2; ++it) {
                    const int i = 16 * it + l16;
                    for (int j = 0; j <= i; ++j) {
                        const float p = sP[i * PP + j];
                        const float* v = &sV[j * VP + wc + 4 * quad];
#pragma unroll
                        for (int u = 0; u < 4; ++u) O[it][u] = fmaf(p, v[u], O[it][u]);
                    }
                }
            } else {
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int it = h; it < 2; ++it) {
                        const f32x4 p = *reinterpret_cast<const f32x4*>(&sP[(16 * it + l16) * PP + 16 * h + 4 * quad]);
#pragma unroll
                        for (int u = 0; u < 4; ++u) O[it] = mfma_f32(vf[h][u], p[u], O[it]);
                    }
            }
            attn_store<2, VEC, true>(A, pl, c, n, c0 + wc + 4 * quad, l16, O);
        }
        const float tot = sTot;
#pragma unroll
        for (int m = 0; m < MT; ++m) S[m] *= tot;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const f32x4 e = *reinterpret_cast<const f32x4*>(&sE[16 * h + 4 * quad]);
#pragma unroll
            for (int u = 0; u < 4; ++u) vf[h][u] *= e[u];
#pragma unroll
            for (int m = 0; m < MT; m += 4)  // four tiles side by side: a product does not wait for the one before
#pragma unroll
                for (int u = 0; u < 4; ++u)
#pragma unroll
                    for (int y = 0; y < 4; ++y)
                        S[m + y] = mfma_f32(sK[(16 * h + 4 * quad + u) * QP + 16 * (m + y) + l16], vf[h][u], S[m + y]);
        }
        __syncthreads();
    }

    float* s_left = attn_last_state(A, pl, STATE_ONLY);
    if (s_left) store_state<4, 16>(A, s_left, c0 + wc + l16, quad, S);
    if (STATE_ONLY && pl.blk == 0 && t == NTHR - 1) A.ws_decay[pl.ws * A.heads + head] = (float)whole;
}

template <int DKT, int WAVES>
static hipError_t launch_one(const AttnArgs& a, bool state_only, hipStream_t s) {
    const int64_t blocks = (a.ids * a.units + 7) / 8 * 8 * a.unit;
    if (blocks > 0x7fffffffLL) return hipErrorInvalidValue;
    const dim3 grid((unsigned)blocks), block(64 * WAVES);
    if (state_only) {
        if (a.vec)
            hipLaunchKernelGGL((attn_chunks_f32_kernel<DKT, WAVES, true, true>), grid, block, 0, s, a);
        else
            hipLaunchKernelGGL((attn_chunks_f32_kernel<DKT, WAVES, true, false>), grid, block, 0, s, a);
    } else {
        if (a.vec)
            hipLaunchKernelGGL((attn_chunks_f32_kernel<DKT, WAVES, false, true>), grid, block, 0, s, a);
        else
            hipLaunchKernelGGL((attn_chunks_f32_kernel<DKT, WAVES, false, false>), grid, block, 0, s, a);
    }
    return hipGetLastError();
}

hipError_t launch_attn_chunks_f32(const AttnArgs& a, bool state_only, hipStream_t s) {
    const int dkt = a.dk <= 64 ? 1 : a.dk <= 128 ? 2 : 4;
    if (a.block == 64)
        return dkt == 1 ? launch_one<1, 4>(a, state_only, s)
               : dkt == 2 ? launch_one<2, 4>(a, state_only, s)
                          : launch_one<4, 4>(a, state_only, s);
    return dkt == 1 ? launch_one<1, 8>(a, state_only, s)
           : dkt == 2 ? launch_one<2, 8>(a, state_only, s)
                      : launch_one<4, 8>(a, state_only, s);
}

}  // namespace cv
