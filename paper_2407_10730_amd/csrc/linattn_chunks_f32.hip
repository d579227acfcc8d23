// linattn_chunks_f32.hip -- linear attention with a decay per head in chunks of 32 tokens, fp32 operands.
//
// The same four products per chunk and the same division of work as the bf16 kernel (linattn_chunks.hip), on the
// fp32 matrix instruction: nothing is rounded below fp32.  It multiplies at a sixteenth of the bf16 rate, which makes
// this kernel bound by it; 32 tokens per chunk halve the products within a chunk.
// Operand order: in step (m, u) of a reduction the lanes of quad q multiply index 16 m + 4 q + u, so that a lane's four
// steps are one 16-byte LDS read, and the state's registers are operands as they are.
#include "linattn_device.h"

namespace cv {

__device__ __forceinline__ f32x4 mfma_f32(float a, float b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}

// 4 consecutive elements of a row, those at or past `n` zero.
__device__ __forceinline__ f32x4 load4(const float* p, int n, bool vec) {
    if (n <= 0) return f32x4{0, 0, 0, 0};
    if (vec) return *reinterpret_cast<const f32x4*>(p);
    f32x4 r{0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < n) r[i] = p[i];
    return r;
}

// dk up to 64 DKT, 64 NT columns of v per workgroup
template <int DKT, int NT, bool STATE_ONLY>
__global__ __launch_bounds__(256, 2) void attn_chunks_f32_kernel(AttnArgs A) {
    constexpr int C = kChunkF32, DKP = 64 * DKT, DVB = 64 * NT;
    constexpr int QP = DKP + 4, VP = DVB + 4, PP = C + 4;  // LDS row pitches in floats
    constexpr int MT = DKP / 16;
    __shared__ __align__(16) float sQ[STATE_ONLY ? 1 : C * QP];
    __shared__ __align__(16) float sK[C * QP];
    __shared__ __align__(16) float sV[C * VP];
    __shared__ __align__(16) float sP[STATE_ONLY ? 1 : C * PP];
    __shared__ __align__(16) double sB[C];
    __shared__ __align__(16) float sE[C], sD[C];
    __shared__ float sTot;

    const int t = threadIdx.x, wave = t >> 6, lane = t & 63, l16 = lane & 15, quad = lane >> 4;
    AttnPlace pl;
    if (!attn_place(A, STATE_ONLY, &pl)) return;
    const int head = pl.head;
    const int64_t row0 = pl.row0, len = pl.len;
    const int c0 = pl.blk * DVB;      // first column of the workgroup
    const int wc = wave * 16 * NT;    // ... of the wave, within the workgroup's
    const int qh = head / A.rep;
    const bool vec = A.vec;

    // tile (m, n): rows 16 m + 4 quad + i, column col(l16, n); a lane's results of all n tiles are 4 NT neighbours
    auto col = [&](int x, int n) { return wc + 4 * NT * (x >> 2) + 4 * n + (x & 3); };
    f32x4 S[MT][NT];
    const float* s_init = STATE_ONLY ? nullptr : attn_first_state(A, pl);
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int rr = 16 * m + 4 * quad + i, cc = c0 + col(l16, n);
                S[m][n][i] = s_init && rr < A.dk && cc < A.dv ? s_init[(int64_t)rr * A.dv + cc] : 0.0f;
            }

    constexpr int NQ = C * DKP / 4 / 256, NV = C * DVB / 4 / 256;  // 16-byte loads per thread
    constexpr int RS = 256 / (DKP / 4), RSV = 256 / (DVB / 4);
    const int lr = t / (DKP / 4), lc = t % (DKP / 4) * 4, lrv = t / (DVB / 4), lcv = t % (DVB / 4) * 4;
    const float* gq = static_cast<const float*>(A.q) + (row0 + lr) * A.q_row + qh * A.q_head + lc;
    const float* gk = static_cast<const float*>(A.k) + (row0 + lr) * A.k_row + qh * A.k_head + lc;
    const float* gv = static_cast<const float*>(A.v) + (row0 + lrv) * A.v_row + head * A.v_head + c0 + lcv;
    const float* gg = A.g ? A.g + row0 * A.g_row + head : nullptr;
    f32x4 rq[STATE_ONLY ? 1 : NQ], rk[NQ], rv[NV];
    float rg = 0.0f;
    auto load = [&](int64_t c) {
        const int n = (int)min<int64_t>(C, len - c);
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
            const bool ok = lr + i * RS < n;
            if constexpr (!STATE_ONLY) rq[i] = load4(gq + (c + i * RS) * A.q_row, ok ? A.dk - lc : 0, vec);
            rk[i] = load4(gk + (c + i * RS) * A.k_row, ok ? A.dk - lc : 0, vec);
        }
#pragma unroll
        for (int i = 0; i < NV; ++i)
            rv[i] = load4(gv + (c + i * RSV) * A.v_row, lrv + i * RSV < n ? A.dv - c0 - lcv : 0, vec);
        if (wave == 0) rg = gg && lane < n ? gg[(c + lane) * A.g_row] : 0.0f;
    };

    double whole = 0.0;
    if (len > 0) load(0);
    for (int64_t c = 0; c < len; c += C) {
        const int n = (int)min<int64_t>(C, len - c);
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
            if constexpr (!STATE_ONLY) *reinterpret_cast<f32x4*>(&sQ[(lr + i * RS) * QP + lc]) = rq[i];
            *reinterpret_cast<f32x4*>(&sK[(lr + i * RS) * QP + lc]) = rk[i];
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) *reinterpret_cast<f32x4*>(&sV[(lrv + i * RSV) * VP + lcv]) = rv[i];
        if (wave == 0) {
            const double tot = chunk_decays(rg, sB, sD, sE, C);
            if (lane == 0) sTot = __builtin_amdgcn_exp2f((float)tot);
            whole += tot;
        }
        __syncthreads();
        if (c + C < len) load(c + C);

        f32x4 O[2][NT];
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
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const int j = 16 * jt + 4 * quad + u;
                    const float f = __builtin_amdgcn_exp2f((float)(bi - sB[j]));
                    s[u] = j <= i ? s[u] * f : 0.0f;
                }
                *reinterpret_cast<f32x4*>(&sP[i * PP + 16 * jt + 4 * quad]) = s;
            }
        }
        auto inter = [&] {  // exp(b_i) q_i S, transposed
#pragma unroll
            for (int it = 0; it < 2; ++it)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) O[it][nt] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int it = 0; it < 2; ++it) {
                    const f32x4 b = *reinterpret_cast<const f32x4*>(&sQ[(16 * it + l16) * QP + 16 * m + 4 * quad]);
#pragma unroll
                    for (int u = 0; u < 4; ++u)
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) O[it][nt] = mfma_f32(S[m][nt][u], b[u], O[it][nt]);
                }
#pragma unroll
            for (int it = 0; it < 2; ++it) {
                const float d = sD[16 * it + l16];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) O[it][nt] *= d;
            }
        };
        if constexpr (!STATE_ONLY) {
            inter();
            __syncthreads();
        }
        float vf[2][4][NT];  // v of token 16 h + 4 quad + u
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) vf[h][u][nt] = sV[(16 * h + 4 * quad + u) * VP + col(l16, nt)];
        if constexpr (!STATE_ONLY) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int it = h; it < 2; ++it) {
                    const f32x4 p = *reinterpret_cast<const f32x4*>(&sP[(16 * it + l16) * PP + 16 * h + 4 * quad]);
#pragma unroll
                    for (int u = 0; u < 4; ++u)
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) O[it][nt] = mfma_f32(vf[h][u][nt], p[u], O[it][nt]);
                }
            // an infinite or NaN v of a later token has reached the first token of the 16: sum without the masked terms
            bool bad = false;
            if (l16 == 0) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int u = 0; u < 4; ++u) bad |= !finite(O[0][nt][u]) || !finite(O[1][nt][u]);
            }
            if (__any(bad)) {
                inter();
#pragma unroll
                for (int it = 0; it < 2; ++it) {
                    const int i = 16 * it + l16;
                    for (int j = 0; j <= i; ++j) {
                        const float p = sP[i * PP + j];
                        const float* v = &sV[j * VP + wc + 4 * NT * quad];
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int u = 0; u < 4; ++u) O[it][nt][u] = fmaf(p, v[4 * nt + u], O[it][nt][u]);
                    }
                }
            }
            const int oc = c0 + wc + 4 * NT * quad;
#pragma unroll
            for (int it = 0; it < 2; ++it) {
                const int i = 16 * it + l16;
                if (i < n && oc < A.dv) {
                    float e[4 * NT];
#pragma unroll
                    for (int x = 0; x < 4 * NT; ++x) e[x] = O[it][x / 4][x % 4];
                    attn_store<4 * NT>(A, 1, row0 + c + i, head, oc, e);
                }
            }
        }
        const float tot = sTot;
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) S[m][nt] *= tot;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const f32x4 e = *reinterpret_cast<const f32x4*>(&sE[16 * h + 4 * quad]);
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) vf[h][u][nt] *= e[u];
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const float k = sK[(16 * h + 4 * quad + u) * QP + 16 * m + l16];
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) S[m][nt] = mfma_f32(k, vf[h][u][nt], S[m][nt]);
                }
        }
        __syncthreads();
    }

    float* s_left = attn_last_state(A, pl, STATE_ONLY);
    if (s_left) {
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int rr = 16 * m + 4 * quad + i, cc = c0 + col(l16, n);
                    if (rr < A.dk && cc < A.dv) s_left[(int64_t)rr * A.dv + cc] = S[m][n][i];
                }
    }
    if (STATE_ONLY && pl.blk == 0 && t == 0) A.ws_decay[pl.id * A.heads + head] = (float)whole;
}

template <int DKT, int NT>
static hipError_t launch_one(const AttnArgs& a, bool state_only, hipStream_t s) {
    const int64_t blocks = (a.segment ? a.nseg : a.sq.seqs) * a.heads * a.ndvb;
    if (blocks > 0x7fffffffLL) return hipErrorInvalidValue;
    if (state_only)
        hipLaunchKernelGGL((attn_chunks_f32_kernel<DKT, NT, true>), dim3((unsigned)blocks), dim3(256), 0, s, a);
    else
        hipLaunchKernelGGL((attn_chunks_f32_kernel<DKT, NT, false>), dim3((unsigned)blocks), dim3(256), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_attn_chunks_f32(const AttnArgs& a, bool state_only, hipStream_t s) {
    if (a.dk > 128) return launch_one<4, 1>(a, state_only, s);
    if (chunk_block(a.dk, a.dv) == 64)
        return a.dk <= 64 ? launch_one<1, 1>(a, state_only, s) : launch_one<2, 1>(a, state_only, s);
    return a.dk <= 64 ? launch_one<1, 2>(a, state_only, s) : launch_one<2, 2>(a, state_only, s);
}

}  // namespace cv
