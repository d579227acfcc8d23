// linattn_chunks.hip -- linear attention with a decay per head in chunks of 64 tokens, bf16 operands.
//
// With b_i the sum of a chunk's first i log decays and S the state it starts from,
//
//   o_i = scale ( exp(b_i) q_i S + sum_{j <= i} exp(b_i - b_j) (q_i . k_j) v_j )
//   S'  = exp(b_C) S + sum_j exp(b_C - b_j) k_j v_j^T
//
// are four matrix products per chunk.  One workgroup runs a sequence's chunks in order, for one head and 64 or 128 columns
// of v, 16 per wave.  A wave's part of S stays in its accumulator registers from chunk to chunk and is itself an
// operand of q S (the rows that a lane holds as a result are the reduction indices that it feeds as an
// operand; q is read from LDS in the same order), so S never passes through LDS.  The scores are shared: the waves
// divide their 16x16 tiles and exchange them through LDS.  Products over tokens read k and v from LDS through the
// transposing load.
// Rounding: q, k and v are exact; what is computed in fp32 enters a product as bf16 planes, each the rounding of
// what the ones before left.  The update of the state multiplies k by exp(b_C - b_j) v_j in three planes, which hold all
// 24 bits, so states keep fp32 accuracy over any length.  The scores and, as an operand of q S, the state take two planes
// for bf16 results, which leave 2^-16 of each term where the result's own rounding is 2^-8, and three for fp32 results.
// (8192 tokens, 16 heads of 128 x 128, with one plane, whose roundings are of the result's size: 66 us; with two 71, with three
// and fp32 results 83.)
//
// Bound, at 65536 tokens of 8 heads of 128 x 128 in segments of 1024: the full pass moves q, k, v and o, 537 MB, in 140 us
// warm (3.8 TB/s; with one plane 120, by memory); its vector unit is busy 0.56 of the cycles, its matrix unit 0.37, LDS 0.39,
// and two workgroups per CU do not hide all of each other's waits.  The state pass by memory (268 MB in 65 us).  At 8192
// tokens of 16 heads, one workgroup per CU, by the waves' own chains: 46 and 21 us for 134 and 67 MB.
#include "linattn_device.h"

namespace cv {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// Four rows of 16 columns transposed: lane l of each 16 gives the address of row l / 4, columns 4 (l % 4) .. + 3,
// and receives column l of the four rows.
__device__ __forceinline__ u32x2 lds_tr(const uint16_t* base, uint32_t off) {
    typedef __attribute__((address_space(3))) s16x4* lds_ptr;
    return __builtin_bit_cast(
        u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(reinterpret_cast<const char*>(base) + off)));
}
__device__ __forceinline__ bf16x8 join8(u32x2 a, u32x2 b) {
    return __builtin_bit_cast(bf16x8, u32x4{a[0], a[1], b[0], b[1]});
}

// Where LDS holds element (row, c) of a tile of P columns (q, k: 64, 128 or 256; v: 64 or 128; scores: 64).  The 16-byte
// units of a row are permuted by an exclusive or with a number of the row, so that without padding (a row is a
// multiple of half the 64 banks) these take distinct banks: 16 rows of one unit, whether the 16 lanes served
// together are of one quad or of two (8 rows each, of neighbouring units: rows r < 4 and r >= 12 of a tile, or the
// others); 16 rows of half a unit; and rows r .. r + 3 and r + 8 .. r + 11 of two units, which two quads of a transposing
// load take.  k is read transposed by half of each of four units instead, so that a lane's rows of the state are 8
// neighbours and q comes in whole units; two quads share the banks there (two-way: a third of the state pass's LDS cycles, whose
// time is the same without; reading q in halves cost more).
// The number depends on row % 16 only, so 16 rows or 64 bytes (32 bytes ...) further on is an addition or an exclusive
// or with a constant: the kernel keeps one byte offset per access pattern (swz_at) and derives the others.
template <int P>
__device__ __forceinline__ uint32_t swz(int row) {
    const int h0 = row >> 2 & 1, h1 = row >> 3 & 1;
    return P == 64 ? (row & 2) << 1 | (h0 ^ h1) << 1 | h1  // two rows per 64 banks
                   : (row & 3) << 2 | (h0 ^ h1) << 1 | h1;
}
template <int P>
__device__ __forceinline__ uint32_t swz_at(int row, int c) {
    return row * (2 * P) + ((((uint32_t)c >> 3) ^ swz<P>(row)) << 4) + (c & 7) * 2;
}
template <typename V>
__device__ __forceinline__ V lds_read(const uint16_t* base, uint32_t off) {
    return *reinterpret_cast<const V*>(reinterpret_cast<const char*>(base) + off);
}
template <typename V>
__device__ __forceinline__ void lds_write(uint16_t* base, uint32_t off, V v) {
    *reinterpret_cast<V*>(reinterpret_cast<char*>(base) + off) = v;
}

// waves per SIMD that LDS leaves room for
constexpr int chunk_occupancy(int dkt, int waves) { return waves == 8 ? (dkt <= 4 ? 4 : 2) : dkt <= 2 ? 4 : dkt <= 4 ? 3 : 1; }

// Two fp32 values as PL bf16 planes.  INF: infinities stay so in every plane (the largest float is taken off them);
// without, the planes after the first are NaN.
template <bool INF, int PL>
__device__ __forceinline__ void bf16_planes(float a, float b, uint32_t (&p)[PL]) {
#pragma unroll
    for (int x = 0; x < PL; ++x) {
        p[x] = pack_bf16(a, b);
        if (x + 1 < PL) {
            constexpr float kMax = 3.402823466e38f;
            const float pa = __builtin_bit_cast(float, p[x] << 16), pb = __builtin_bit_cast(float, p[x] & 0xffff0000u);
            a -= INF ? __builtin_amdgcn_fmed3f(pa, -kMax, kMax) : pa;
            b -= INF ? __builtin_amdgcn_fmed3f(pb, -kMax, kMax) : pb;
        }
    }
}
template <int PL>
__device__ __forceinline__ void bf16_planes8(f32x4 a, f32x4 b, bf16x8 (&p)[PL]) {
    uint32_t w[4][PL];
    bf16_planes<true>(a[0], a[1], w[0]);
    bf16_planes<true>(a[2], a[3], w[1]);
    bf16_planes<true>(b[0], b[1], w[2]);
    bf16_planes<true>(b[2], b[3], w[3]);
#pragma unroll
    for (int x = 0; x < PL; ++x) p[x] = __builtin_bit_cast(bf16x8, u32x4{w[0][x], w[1][x], w[2][x], w[3][x]});
}

// Scores in LDS: the six blocks of 16 rows and 32 columns that are read (column half h of rows 16 it: h = 0, and h = 1
// from it = 2 on), one plane after the other, two blocks side by side in rows of 64.
__device__ __forceinline__ int score_block(int it, int h, int plane) { return 6 * plane + it + 2 * h; }
__device__ __forceinline__ uint32_t score_off(uint32_t at, int block) {
    return (at ^ ((block & 1) << 6)) + (block >> 1) * (32 * kChunk);
}

// PL: planes of the scores and of the state as an operand; three where results are fp32.
template <int DKT, int WAVES, bool STATE_ONLY, bool VEC, int PL>
__global__ __launch_bounds__(64 * WAVES, chunk_occupancy(DKT, WAVES)) void attn_chunks_bf16_kernel(AttnArgs A) {
    constexpr int C = kChunk, DKP = 32 * DKT, DVB = 16 * WAVES, NTHR = 64 * WAVES;
    constexpr int MT = 2 * DKT;                            // 16-row tiles of the state
    __shared__ __align__(16) uint16_t sQ[STATE_ONLY ? 1 : C * DKP];
    __shared__ __align__(16) uint16_t sK[C * DKP];
    __shared__ __align__(16) uint16_t sV[C * DVB];
    __shared__ __align__(16) uint16_t sP[STATE_ONLY ? 1 : PL * 6 * 16 * 32];
    __shared__ __align__(16) double sB[C];
    __shared__ __align__(16) float sE[C], sD[C];
    __shared__ float sTot;

    const int t = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    int lane = t & 63, l16 = lane & 15, quad = lane >> 4;
    AttnPlace pl;
    if (!attn_place(A, STATE_ONLY, &pl)) return;
    const int head = pl.head;
    const int64_t row0 = pl.row0, len = pl.len;
    const int c0 = pl.blk * DVB;          // first column of the workgroup
    const int wc = wave * 16;             // ... of the wave, within the workgroup's
    const int qh = head / A.rep;

    f32x4 S[MT];  // tile m: rows 32 (m / 2) + 8 quad + 4 (m % 2) + i, column c0 + wc + l16
    load_state<8, 4>(A, STATE_ONLY ? nullptr : attn_first_state(A, pl), c0 + wc + l16, quad, S);

    // Loads: thread t takes 8 elements of row t / (DKP / 8) + i * RS of q and k, likewise of v
    constexpr int RS = NTHR / (DKP / 8), RSV = NTHR / (DVB / 8), NQ = C / RS, NV = C / RSV;
    const int lr = t / (DKP / 8), lc = t % (DKP / 8) * 8, lrv = t / (DVB / 8), lcv = t % (DVB / 8) * 8;
    const uint16_t* gq = static_cast<const uint16_t*>(A.q) + row0 * A.q_row + qh * A.q_head;
    const uint16_t* gk = static_cast<const uint16_t*>(A.k) + row0 * A.k_row + qh * A.k_head;
    const uint16_t* gv = static_cast<const uint16_t*>(A.v) + row0 * A.v_row + head * A.v_head;
    const float* gg = A.g ? A.g + row0 * A.g_row + head : nullptr;
    const uint32_t q_row = (uint32_t)A.q_row, k_row = (uint32_t)A.k_row, v_row = (uint32_t)A.v_row;
    uint32_t cut, cut_v;  // (of q, k and of v: row_part)
    uint32_t q_at = row_part<uint16_t, VEC>(lr * q_row, lc, A.dk, &cut);
    uint32_t k_at = row_part<uint16_t, VEC>(lr * k_row, lc, A.dk, &cut);
    uint32_t v_at = row_part<uint16_t, VEC>(lrv * v_row, c0 + lcv, A.dv, &cut_v);
    u32x4 rq[STATE_ONLY ? 1 : NQ], rk[NQ], rv[NV];
    float rg = 0.0f;
    auto load = [&](int64_t c) {  // chunk starting at token c of the segment into registers
        const int n = (int)min<int64_t>(C, len - c);
        if constexpr (!STATE_ONLY) {
            const __amdgpu_buffer_rsrc_t r = chunk_rsrc(gq + c * A.q_row, n, q_row, A.dk);
#pragma unroll
            for (int i = 0; i < NQ; ++i) rq[i] = load_row<uint16_t, VEC>(r, q_at + i * (RS * 2) * q_row, A.dk);
        }
        const __amdgpu_buffer_rsrc_t r = chunk_rsrc(gk + c * A.k_row, n, k_row, A.dk);
        const __amdgpu_buffer_rsrc_t rr = chunk_rsrc(gv + c * A.v_row, n, v_row, A.dv);
#pragma unroll
        for (int i = 0; i < NQ; ++i) rk[i] = load_row<uint16_t, VEC>(r, k_at + i * (RS * 2) * k_row, A.dk);
#pragma unroll
        for (int i = 0; i < NV; ++i) rv[i] = load_row<uint16_t, VEC>(rr, v_at + i * (RSV * 2) * v_row, A.dv);
        if (wave == WAVES - 1) rg = load_decay(A, gg, c, lane, n);
    };

    // byte offsets in LDS of this thread's accesses: stores of a chunk's rows; rows of q and k as operands; k and v
    // transposed (tokens 0-3 and 4-7 of a quad's 8); scores
    uint32_t o_st = swz_at<DKP>(lr, lc), o_stv = swz_at<DVB>(lrv, lcv);
    uint32_t o_row = swz_at<DKP>(l16, 8 * quad);
    const int tr = 8 * quad + (l16 >> 2), tc = 4 * (l16 & 3);
    uint32_t o_k0 = swz_at<DKP>(tr, 2 * tc), o_k1 = swz_at<DKP>(tr + 4, 2 * tc);
    uint32_t o_v0 = swz_at<DVB>(tr, wc + tc), o_v1 = swz_at<DVB>(tr + 4, wc + tc);
    uint32_t o_pw = swz_at<C>(l16, 4 * quad), o_pr = swz_at<C>(l16, 8 * quad);

    double whole = 0.0;  // log2 of the segment's decay (last wave)
    if (len > 0) load(0);
    for (int64_t c = 0; c < len; c += C) {
        const int n = (int)min<int64_t>(C, len - c);
        // what follows from these offsets is cheaper computed again than kept in registers over the loop
        asm volatile("" : "+v"(o_st), "+v"(o_stv), "+v"(o_row), "+v"(o_k0), "+v"(o_k1), "+v"(o_pw), "+v"(o_pr),
                     "+v"(o_v0), "+v"(o_v1));
        asm volatile("" : "+v"(q_at), "+v"(k_at), "+v"(v_at), "+v"(l16), "+v"(quad), "+v"(lane));
        if constexpr (!VEC) asm volatile("" : "+v"(cut), "+v"(cut_v));
        // registers to LDS; decays
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
            // 8 rows further on the number of the row differs in its two low bits
            const uint32_t off = (RS == 8 && i % 2 ? o_st ^ (3u << 4) : o_st) + i * RS * 2 * DKP;
            if constexpr (!STATE_ONLY) lds_write(sQ, off, row_part_of<uint16_t, VEC>(rq[i], cut));
            lds_write(sK, off, row_part_of<uint16_t, VEC>(rk[i], cut));
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) lds_write(sV, o_stv + i * RSV * 2 * DVB, row_part_of<uint16_t, VEC>(rv[i], cut_v));
        if (wave == WAVES - 1) {
            const double tot = chunk_decays(rg, lane, sB, sD, sE, C);
            if (lane == 0) sTot = __builtin_amdgcn_exp2f((float)tot);
            whole += tot;
        }
        __syncthreads();
        if (c + C < len) load(c + C);

        if constexpr (!STATE_ONLY) {
            // Scores, transposed (a lane holds 4 neighbouring j of one i): the 10 of 16 tiles on or below the diagonal, and
            // the 2 above it that are read as zeros, dealt to the waves in turn: (it, jt) = (0,0) (1,0) (1,1) (2,0)
            // (2,1) (2,2) (0,1) (2,3) (3,0) (3,1) (3,2) (3,3)
            constexpr uint64_t kIt = 0x333320222110, kJt = 0x321031210100;
#pragma unroll
            for (int x = 0; x < 12; x += WAVES) {
                if (x + WAVES > 12 && x + wave >= 12) break;
                const int it = (int)(kIt >> (4 * (x + wave))) & 15, jt = (int)(kJt >> (4 * (x + wave))) & 15;
                f32x4 sc{0, 0, 0, 0};
#pragma unroll
                for (int k = 0; k < DKT; ++k)
                    sc = mfma16(lds_read<bf16x8>(sK, (o_row + jt * (32 * DKP)) ^ (k << 6)),
                                lds_read<bf16x8>(sQ, (o_row + it * (32 * DKP)) ^ (k << 6)), sc);
                const int i = 16 * it + l16, j = 16 * jt + 4 * quad;
                const double bi = sB[i];
                const f64x2 b01 = *reinterpret_cast<const f64x2*>(&sB[j]), b23 = *reinterpret_cast<const f64x2*>(&sB[j + 2]);
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const bool on = j + u <= i;
                    const float f = (float)(bi - (u < 2 ? b01[u] : b23[u - 2]));
                    sc[u] = (on ? sc[u] : 0.0f) * __builtin_amdgcn_exp2f(on ? f : 0.0f);
                }
                uint32_t p0[PL], p1[PL];
                bf16_planes<true>(sc[0], sc[1], p0);
                bf16_planes<true>(sc[2], sc[3], p1);
#pragma unroll
                for (int y = 0; y < PL; ++y)
                    lds_write(sP, score_off(o_pw ^ ((jt & 1) << 5), score_block(it, jt >> 1, y)), u32x2{p0[y], p1[y]});
            }
        }
        if constexpr (!STATE_ONLY) __syncthreads();
        // v as an operand: 8 tokens of one column per lane
        u32x4 vf[2];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const u32x2 a = lds_tr(sV, o_v0 + 32 * s * 2 * DVB), b = lds_tr(sV, o_v1 + 32 * s * 2 * DVB);
            vf[s] = u32x4{a[0], a[1], b[0], b[1]};
        }
        if constexpr (!STATE_ONLY) {
            f32x4 O[4];  // transposed: rows are columns of v, columns the 16 tokens of a tile
            // exp(b_i) q_i S
#pragma unroll
            for (int it = 0; it < 4; ++it) O[it] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int k = 0; k < DKT; ++k) {
                // (one step's planes at a time: 8192 tokens, 16 heads of 128 x 128 71 us, with the spills of several 74; three
                // planes spill more with it)
                if constexpr (PL == 2) __builtin_amdgcn_sched_barrier(0);
                bf16x8 sf[PL], qf[4];
                bf16_planes8(S[2 * k], S[2 * k + 1], sf);
#pragma unroll
                for (int it = 0; it < 4; ++it) qf[it] = lds_read<bf16x8>(sQ, (o_row ^ (k << 6)) + it * (32 * DKP));
#pragma unroll
                for (int x = PL - 1; x >= 0; --x)
#pragma unroll
                    for (int it = 0; it < 4; ++it) O[it] = mfma16(sf[x], qf[it], O[it]);
            }
#pragma unroll
            for (int it = 0; it < 4; ++it) O[it] *= sD[16 * it + l16];
            // The scores above the diagonal are zeros, but zero times an infinite or NaN v is NaN: a chunk with such a v
            // among the wave's is summed without those terms.
            u16x2 top{0, 0};
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int w = 0; w < 4; ++w)
                    top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, vf[s][w] & 0x7fff7fffu));
            if (__any(max(top[0], top[1]) >= 0x7f80)) {
#pragma unroll
                for (int it = 0; it < 4; ++it) {
                    const int i = 16 * it + l16;
#pragma unroll 1
                    for (int j = 0; j <= i; ++j) {
                        float p = 0.0f;
#pragma unroll
                        for (int x = PL - 1; x >= 0; --x)
                            p += to_f32(lds_read<uint16_t>(sP, score_off(swz_at<C>(l16, j & 31), score_block(it, j >> 5, x))));
                        const uint32_t v = swz_at<DVB>(j, wc + 4 * quad);
#pragma unroll
                        for (int u = 0; u < 4; ++u) O[it][u] = fmaf(p, to_f32(lds_read<uint16_t>(sV, v + 2 * u)), O[it][u]);
                    }
                }
            } else {
#pragma unroll
                for (int s = 0; s < 2; ++s)
#pragma unroll
                    for (int x = PL - 1; x >= 0; --x)
#pragma unroll
                        for (int it = 2 * s; it < 4; ++it)
                            O[it] = mfma16(__builtin_bit_cast(bf16x8, vf[s]),
                                           lds_read<bf16x8>(sP, score_off(o_pr, score_block(it, s, x))), O[it]);
            }
            attn_store<4, VEC, PL == 3>(A, pl, c, n, c0 + wc + 4 * quad, l16, O);
        }
        // the state moves on
        const float tot = sTot;
#pragma unroll
        for (int m = 0; m < MT; ++m) S[m] *= tot;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            __builtin_amdgcn_sched_barrier(0);  // (operands of both steps at once would spill)
            u32x4 vp[3];  // planes of exp(b_C - b_j) v_j
            const f32x4 e0 = *reinterpret_cast<const f32x4*>(&sE[32 * s + 8 * quad]);
            const f32x4 e1 = *reinterpret_cast<const f32x4*>(&sE[32 * s + 8 * quad + 4]);
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                uint32_t p[3];
                bf16_planes<false>(__builtin_bit_cast(float, vf[s][w] << 16) * (w < 2 ? e0[2 * w] : e1[2 * w - 4]),
                                   __builtin_bit_cast(float, vf[s][w] & 0xffff0000u) * (w < 2 ? e0[2 * w + 1] : e1[2 * w - 3]),
                                   p);
#pragma unroll
                for (int x = 0; x < 3; ++x) vp[x][w] = p[x];
            }
#pragma unroll
            for (int m = 0; m < MT; m += 2) {  // two tiles side by side: a product does not wait for the one before
                bf16x8 kf[2];
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const uint32_t at = m << 5, down = 32 * s * 2 * DKP + 8 * y;
                    kf[y] = join8(lds_tr(sK, (o_k0 ^ at) + down), lds_tr(sK, (o_k1 ^ at) + down));
                }
#pragma unroll
                for (int x = 2; x >= 0; --x)
#pragma unroll
                    for (int y = 0; y < 2; ++y) S[m + y] = mfma16(kf[y], __builtin_bit_cast(bf16x8, vp[x]), S[m + y]);
            }
        }
        __syncthreads();
    }

    float* s_left = attn_last_state(A, pl, STATE_ONLY);
    if (s_left) store_state<8, 4>(A, s_left, c0 + wc + l16, quad, S);
    if (STATE_ONLY && pl.blk == 0 && t == NTHR - 1) A.ws_decay[pl.ws * A.heads + head] = (float)whole;
}

template <int DKT, int WAVES, bool STATE_ONLY, int PL>
static void launch_rows(const AttnArgs& a, dim3 grid, hipStream_t s) {
    if (a.vec)
        hipLaunchKernelGGL((attn_chunks_bf16_kernel<DKT, WAVES, STATE_ONLY, true, PL>), grid, dim3(64 * WAVES), 0, s, a);
    else
        hipLaunchKernelGGL((attn_chunks_bf16_kernel<DKT, WAVES, STATE_ONLY, false, PL>), grid, dim3(64 * WAVES), 0, s, a);
}

template <int DKT, int WAVES>
static hipError_t launch_one(const AttnArgs& a, int odt, bool state_only, hipStream_t s) {
    const int64_t blocks = (a.ids * a.units + 7) / 8 * 8 * a.unit;
    if (blocks > 0x7fffffffLL) return hipErrorInvalidValue;
    const dim3 grid((unsigned)blocks);
    if (state_only)
        launch_rows<DKT, WAVES, true, 2>(a, grid, s);
    else if (odt == CONV2D_F32)
        launch_rows<DKT, WAVES, false, 3>(a, grid, s);
    else
        launch_rows<DKT, WAVES, false, 2>(a, grid, s);
    return hipGetLastError();
}

hipError_t launch_attn_chunks_bf16(const AttnArgs& a, int odt, bool state_only, hipStream_t s) {
    const int dkt = a.dk <= 64 ? 2 : a.dk <= 128 ? 4 : 8;
    if (a.block == 64)
        return dkt == 2 ? launch_one<2, 4>(a, odt, state_only, s)
               : dkt == 4 ? launch_one<4, 4>(a, odt, state_only, s)
                          : launch_one<8, 4>(a, odt, state_only, s);
    return dkt == 2 ? launch_one<2, 8>(a, odt, state_only, s)
           : dkt == 4 ? launch_one<4, 8>(a, odt, state_only, s)
                      : launch_one<8, 8>(a, odt, state_only, s);
}

}  // namespace cv
