// linattn_chunks.hip -- linear attention with a decay per head in chunks of 64 tokens, bf16 operands.
//
// With b_i the sum of a chunk's first i log decays and S the state it starts from,
//
//   o_i = scale ( exp(b_i) q_i S + sum_{j <= i} exp(b_i - b_j) (q_i . k_j) v_j )
//   S'  = exp(b_C) S + sum_j exp(b_C - b_j) k_j v_j^T
//
// are four matrix products per chunk.  One workgroup (4 waves) runs a sequence's chunks in order, for one head and
// 64 NT columns of v.  Each wave owns 16 NT of the columns: its part of S stays in the accumulator
// registers from chunk to chunk and is itself an operand of q S (the rows that a lane holds as a result
// are the reduction indices that it feeds as an operand; q is read from LDS in the same order), so S never
// passes through LDS.  The scores are shared: each wave computes 16 rows of them into LDS.  Products over
// tokens read k and v from LDS through the transposing load.
//
// Rounding: the scores and, as an operand of q S, the state are rounded to bf16 once (o is bf16 itself, or
// as exact as bf16 operands make it); the state's own update multiplies exact k by exp(b_C - b_j) v_j
// as three bf16 planes, which hold all 24 bits, so states keep fp32 accuracy over any length.
#include "linattn_device.h"

namespace cv {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// Four rows of 16 columns transposed: lane l of each 16 gives the address of row l / 4, columns 4 (l % 4) .. + 3,
// and receives column l of the four rows.
__device__ __forceinline__ u32x2 lds_tr(const uint16_t* p) {
    typedef __attribute__((address_space(3))) s16x4* lds_ptr;
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(p)));
}
__device__ __forceinline__ bf16x8 join8(u32x2 a, u32x2 b) {
    return __builtin_bit_cast(bf16x8, u32x4{a[0], a[1], b[0], b[1]});
}
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
}

template <int DKT, int NT, bool STATE_ONLY, bool VEC>
__global__ __launch_bounds__(256, DKT <= 4 ? 2 : 1) void attn_chunks_bf16_kernel(AttnArgs A, int o_f32) {
    constexpr int C = kChunk, DKP = 32 * DKT, DVB = 64 * NT;
    // LDS row pitches.  Of the 64 banks, rows of q and k are 12 apart (or -12): 8 rows of 16 bytes, 16 of 8, and the 4
    // rows that a transposing load takes 8 banks of are free of conflicts; rows of v, of which it takes
    // every other 8 bytes with NT = 2, are 16 apart then.
    constexpr int QP = DKP + (DKP == 64 ? 40 : 24), VP = DVB + (NT == 1 ? 40 : 32), PP = C + 8;
    constexpr int MT = 2 * DKT;                            // 16-row tiles of the state
    __shared__ __align__(16) uint16_t sQ[STATE_ONLY ? 1 : C * QP];
    __shared__ __align__(16) uint16_t sK[C * QP];
    __shared__ __align__(16) uint16_t sV[C * VP];
    __shared__ __align__(16) uint16_t sP[STATE_ONLY ? 1 : C * PP];
    __shared__ __align__(16) double sB[C];
    __shared__ __align__(16) float sE[C], sD[C];
    __shared__ float sTot;

    const int t = threadIdx.x, wave = t >> 6, lane = t & 63, l16 = lane & 15, quad = lane >> 4;
    AttnPlace pl;
    if (!attn_place(A, STATE_ONLY, &pl)) return;
    const int head = pl.head;
    const int64_t row0 = pl.row0, len = pl.len;
    const int c0 = pl.blk * DVB;          // first column of the workgroup
    const int wc = wave * 16 * NT;        // ... of the wave, within the workgroup's
    const int qh = head / A.rep;

    // The state: tile (m, n) of the wave holds rows 16 m + 4 quad + i and column wc + col(l16, n).
    // Columns are dealt so that a lane's results of all n tiles are 4 NT neighbours.
    auto col = [&](int x, int n) { return wc + 4 * NT * (x >> 2) + 4 * n + (x & 3); };
    f32x4 S[MT][NT];
    auto scol = [&](int n) { return c0 + col(l16, n); };
    load_state<MT, NT>(A, STATE_ONLY ? nullptr : attn_first_state(A, pl), scol, quad, S);

    // Loads: thread t takes 8 elements of row t / (DKP / 8) + i * RS of q and k, likewise of v
    constexpr int RS = 256 / (DKP / 8), RSV = 256 / (DVB / 8);
    const int lr = t / (DKP / 8), lc = t % (DKP / 8) * 8, lrv = t / (DVB / 8), lcv = t % (DVB / 8) * 8;
    const uint16_t* gq = static_cast<const uint16_t*>(A.q) + row0 * A.q_row + qh * A.q_head;
    const uint16_t* gk = static_cast<const uint16_t*>(A.k) + row0 * A.k_row + qh * A.k_head;
    const uint16_t* gv = static_cast<const uint16_t*>(A.v) + row0 * A.v_row + head * A.v_head + c0;
    const float* gg = A.g ? A.g + row0 * A.g_row + head : nullptr;
    const uint32_t q_row = (uint32_t)A.q_row, k_row = (uint32_t)A.k_row, v_row = (uint32_t)A.v_row;
    const int live = A.dk - lc, live_v = A.dv - c0 - lcv;
    const uint32_t q_at = live > 0 ? (lr * q_row + lc) * 2 : OOB_OFF, k_at = live > 0 ? (lr * k_row + lc) * 2 : OOB_OFF;
    const uint32_t v_at = live_v > 0 ? (lrv * v_row + lcv) * 2 : OOB_OFF;
    u32x4 rq[STATE_ONLY ? 1 : DKT], rk[DKT], rv[2 * NT];
    float rg = 0.0f;
    auto load = [&](int64_t c) {  // chunk starting at token c of the segment into registers
        const int n = (int)min<int64_t>(C, len - c);
        if constexpr (!STATE_ONLY) {
            const __amdgpu_buffer_rsrc_t r = chunk_rsrc(gq + c * A.q_row, n, q_row, A.dk);
#pragma unroll
            for (int i = 0; i < DKT; ++i) rq[i] = load_row<uint16_t, VEC>(r, q_at + i * (RS * 2) * q_row, live);
        }
        const __amdgpu_buffer_rsrc_t r = chunk_rsrc(gk + c * A.k_row, n, k_row, A.dk);
        const __amdgpu_buffer_rsrc_t rr = chunk_rsrc(gv + c * A.v_row, n, v_row, A.dv - c0);
#pragma unroll
        for (int i = 0; i < DKT; ++i) rk[i] = load_row<uint16_t, VEC>(r, k_at + i * (RS * 2) * k_row, live);
#pragma unroll
        for (int i = 0; i < 2 * NT; ++i) rv[i] = load_row<uint16_t, VEC>(rr, v_at + i * (RSV * 2) * v_row, live_v);
        if (wave == 0) rg = gg && lane < n ? gg[(c + lane) * A.g_row] : 0.0f;
    };

    double whole = 0.0;  // log2 of the segment's decay (wave 0)
    if (len > 0) load(0);
    for (int64_t c = 0; c < len; c += C) {
        const int n = (int)min<int64_t>(C, len - c);
        // registers to LDS; decays
#pragma unroll
        for (int i = 0; i < DKT; ++i) {
            if constexpr (!STATE_ONLY) *reinterpret_cast<u32x4*>(&sQ[(lr + i * RS) * QP + lc]) = rq[i];
            *reinterpret_cast<u32x4*>(&sK[(lr + i * RS) * QP + lc]) = rk[i];
        }
#pragma unroll
        for (int i = 0; i < 2 * NT; ++i) *reinterpret_cast<u32x4*>(&sV[(lrv + i * RSV) * VP + lcv]) = rv[i];
        if (wave == 0) {
            const double tot = chunk_decays(rg, sB, sD, sE, C);
            if (lane == 0) sTot = __builtin_amdgcn_exp2f((float)tot);
            whole += tot;
        }
        __syncthreads();
        if (c + C < len) load(c + C);

        f32x4 O[4][NT];
        if constexpr (!STATE_ONLY) {
            // Scores, transposed (a lane holds 4 neighbouring j of one i).  10 of the 16 tiles are on or below the
            // diagonal and 2 above it are read as zeros: 3 per wave, (it, jt) =
            // (0,0) (3,0) (3,1) | (1,0) (1,1) (3,2) | (2,0) (2,1) (2,2) | (3,3) (0,1) (2,3)
            constexpr uint32_t kIt[3] = {0x3210, 0x0213, 0x2233}, kJt[3] = {0x3000, 0x1110, 0x3221};
            f32x4 sc[3];
            int row[3], krow[3];
#pragma unroll
            for (int x = 0; x < 3; ++x) {
                sc[x] = f32x4{0, 0, 0, 0};
                row[x] = 16 * ((kIt[x] >> (4 * wave)) & 15) + l16;
                krow[x] = 16 * ((kJt[x] >> (4 * wave)) & 15);
            }
#pragma unroll
            for (int k = 0; k < DKT; ++k)
#pragma unroll
                for (int x = 0; x < 3; ++x)
                    sc[x] = mfma16(*reinterpret_cast<const bf16x8*>(&sK[(krow[x] + l16) * QP + 32 * k + 8 * quad]),
                                   *reinterpret_cast<const bf16x8*>(&sQ[row[x] * QP + 32 * k + 8 * quad]), sc[x]);
#pragma unroll
            for (int x = 0; x < 3; ++x) {
                const int i = row[x], j = krow[x] + 4 * quad;
                const double bi = sB[i];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const bool on = j + u <= i;
                    const float f = __builtin_amdgcn_exp2f(on ? (float)(bi - sB[j + u]) : 0.0f);
                    sc[x][u] = (on ? sc[x][u] : 0.0f) * f;
                }
                *reinterpret_cast<u32x2*>(&sP[i * PP + j]) = u32x2{pack_bf16(sc[x][0], sc[x][1]), pack_bf16(sc[x][2], sc[x][3])};
            }
        }
        // exp(b_i) q_i S, transposed: rows are columns of v, columns the 16 tokens of a tile
        auto inter = [&] {
#pragma unroll
            for (int it = 0; it < 4; ++it)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) O[it][nt] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int k = 0; k < DKT; ++k) {
                bf16x8 sf[NT];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const f32x4 a = S[2 * k][nt], b = S[2 * k + 1][nt];
                    sf[nt] = __builtin_bit_cast(bf16x8, u32x4{pack_bf16(a[0], a[1]), pack_bf16(a[2], a[3]),
                                                              pack_bf16(b[0], b[1]), pack_bf16(b[2], b[3])});
                }
#pragma unroll
                for (int it = 0; it < 4; ++it) {
                    const uint16_t* p = &sQ[(16 * it + l16) * QP + 32 * k + 4 * quad];
                    const bf16x8 qf = join8(*reinterpret_cast<const u32x2*>(p), *reinterpret_cast<const u32x2*>(p + 16));
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) O[it][nt] = mfma16(sf[nt], qf, O[it][nt]);
                }
            }
#pragma unroll
            for (int it = 0; it < 4; ++it) {
                const float d = sD[16 * it + l16];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) O[it][nt] *= d;
            }
        };
        if constexpr (!STATE_ONLY) {
            inter();
            __syncthreads();
        }
        // v as an operand: 8 tokens of one column per lane
        u32x4 vf[2][NT];
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const uint16_t* p = &sV[(32 * s + 8 * quad + (l16 >> 2)) * VP + wc + 4 * NT * (l16 & 3) + 4 * nt];
                const u32x2 a = lds_tr(p), b = lds_tr(p + 4 * VP);
                vf[s][nt] = u32x4{a[0], a[1], b[0], b[1]};
            }
        if constexpr (!STATE_ONLY) {
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int it = 2 * s; it < 4; ++it) {
                    const bf16x8 pf =
                        *reinterpret_cast<const bf16x8*>(&sP[(16 * it + l16) * PP + 32 * s + 8 * quad]);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
                        O[it][nt] = mfma16(__builtin_bit_cast(bf16x8, vf[s][nt]), pf, O[it][nt]);
                }
            // A later token's infinite or NaN v times its score of zero has made every earlier token NaN too, the
            // first of the 32 that share a product step among them: such chunks are summed again
            // without the masked terms.
            bool bad = false;
            if (l16 == 0) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int u = 0; u < 4; ++u)
                        bad |= !finite(O[0][nt][u]) || !finite(O[2][nt][u]);
            }
            if (__any(bad)) {
                inter();
#pragma unroll
                for (int it = 0; it < 4; ++it) {
                    const int i = 16 * it + l16;
                    for (int j = 0; j <= i; ++j) {
                        const float p = to_f32(sP[i * PP + j]);
                        const uint16_t* v = &sV[j * VP + wc + 4 * NT * quad];
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int u = 0; u < 4; ++u) O[it][nt][u] = fmaf(p, to_f32(v[4 * nt + u]), O[it][nt][u]);
                    }
                }
            }
            const int oc = c0 + wc + 4 * NT * quad;
#pragma unroll
            for (int it = 0; it < 4; ++it) {
                const int i = 16 * it + l16;
                if (i < n && oc < A.dv) {
                    float e[4 * NT];
#pragma unroll
                    for (int x = 0; x < 4 * NT; ++x) e[x] = O[it][x / 4][x % 4];
                    attn_store<4 * NT, VEC>(A, o_f32, row0 + c + i, head, oc, e);
                }
            }
        }
        // the state moves on
        const float tot = sTot;
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) S[m][nt] *= tot;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            bf16x8 vp[NT][3];  // planes of exp(b_C - b_j) v_j
            const f32x4 e0 = *reinterpret_cast<const f32x4*>(&sE[32 * s + 8 * quad]);
            const f32x4 e1 = *reinterpret_cast<const f32x4*>(&sE[32 * s + 8 * quad + 4]);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                u32x4 pl[3];
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    float lo = __builtin_bit_cast(float, vf[s][nt][w] << 16) * (w < 2 ? e0[2 * w] : e1[2 * w - 4]);
                    float hi = __builtin_bit_cast(float, vf[s][nt][w] & 0xffff0000u) *
                               (w < 2 ? e0[2 * w + 1] : e1[2 * w - 3]);
#pragma unroll
                    for (int x = 0; x < 3; ++x) {
                        const uint32_t p = pack_bf16(lo, hi);
                        pl[x][w] = p;
                        lo -= __builtin_bit_cast(float, p << 16);
                        hi -= __builtin_bit_cast(float, p & 0xffff0000u);
                    }
                }
#pragma unroll
                for (int x = 0; x < 3; ++x) vp[nt][x] = __builtin_bit_cast(bf16x8, pl[x]);
            }
#pragma unroll
            for (int m = 0; m < MT; m += 2) {
                bf16x8 kf[2];
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const uint16_t* p = &sK[(32 * s + 8 * quad + (l16 >> 2)) * QP + 16 * (m + y) + 4 * (l16 & 3)];
                    kf[y] = join8(lds_tr(p), lds_tr(p + 4 * QP));
                }
#pragma unroll
                for (int x = 2; x >= 0; --x)
#pragma unroll
                    for (int y = 0; y < 2; ++y)
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) S[m + y][nt] = mfma16(kf[y], vp[nt][x], S[m + y][nt]);
            }
        }
        __syncthreads();
    }

    float* s_left = attn_last_state(A, pl, STATE_ONLY);
    if (s_left) store_state<MT, NT>(A, s_left, scol, quad, S);
    if (STATE_ONLY && pl.blk == 0 && t == 0) A.ws_decay[(int64_t)pl.id * A.heads + head] = (float)whole;
}

template <int DKT, int NT>
static hipError_t launch_one(const AttnArgs& a, int odt, bool state_only, hipStream_t s) {
    const int64_t blocks = (a.segment ? a.nseg : a.sq.seqs) * a.heads * a.ndvb;
    if (blocks > 0x7fffffffLL) return hipErrorInvalidValue;
    const dim3 grid((unsigned)blocks), block(256);
    const int f32 = odt == CONV2D_F32;
    if (state_only) {
        if (a.vec)
            hipLaunchKernelGGL((attn_chunks_bf16_kernel<DKT, NT, true, true>), grid, block, 0, s, a, f32);
        else
            hipLaunchKernelGGL((attn_chunks_bf16_kernel<DKT, NT, true, false>), grid, block, 0, s, a, f32);
    } else {
        if (a.vec)
            hipLaunchKernelGGL((attn_chunks_bf16_kernel<DKT, NT, false, true>), grid, block, 0, s, a, f32);
        else
            hipLaunchKernelGGL((attn_chunks_bf16_kernel<DKT, NT, false, false>), grid, block, 0, s, a, f32);
    }
    return hipGetLastError();
}

hipError_t launch_attn_chunks_bf16(const AttnArgs& a, int odt, bool state_only, hipStream_t s) {
    if (a.dk > 128) return launch_one<8, 1>(a, odt, state_only, s);  // two column tiles would not fit the registers
    if (chunk_block(a.dk, a.dv) == 64)
        return a.dk <= 64 ? launch_one<2, 1>(a, odt, state_only, s) : launch_one<4, 1>(a, odt, state_only, s);
    return a.dk <= 64 ? launch_one<2, 2>(a, odt, state_only, s) : launch_one<4, 2>(a, odt, state_only, s);
}

}  // namespace cv
