// softmax_device.h -- the softmax attention kernels, for bf16 and fp32.
//
// A tile is 32 rows per wave, a row being a token for one head.  Scores are computed transposed, 32 keys x 32 rows per matrix
// instruction, so that a lane holds 16 keys of one row: the running maximum and sum of the softmax need no exchange but
// between the two halves of a wave, and the weights are already the operand of the product with v: the rows
// of the result that lane half h holds are keys 8 b + 4 h + i (b, i < 4), and v is read in that order.
#pragma once

#include <cfloat>

#include "seqmix_device.h"

namespace cv {

// What a workgroup works on: rows [t0, t0 + tile) of a sequence for the heads from `head` on, keys [0, keys).
struct SoftPlace {
    int seq, head, kv_head;
    int t0, len, keys;
    int64_t row0, slot;
    int64_t key0;  // packed: first row of the sequence's keys
};

__device__ __forceinline__ int seq_keys(const SoftArgs& A, int seq, int64_t slot, const SeqRange& r, int64_t* first) {
    *first = 0;
    if (A.paged) {
        const int64_t most = A.max_pages << A.shift;
        return (int)min<int64_t>(max(A.lens[slot], 0), most);
    }
    if (!A.koff) {
        *first = r.first;
        return (int)r.len;
    }
    const uint32_t b = clamp_row(A.koff[seq], A.key_tokens), e = clamp_row(A.koff[seq + 1], A.key_tokens);
    *first = b;
    return e > b ? (int)(e - b) : 0;
}

// False: nothing to do (in all threads).
__device__ __forceinline__ bool soft_place(const SoftArgs& A, uint32_t id, int block, SoftPlace* out) {
    const SeqPart sp = seq_part(A.sq, id, (uint32_t)A.tile);
    if (sp.seq >= A.sq.seqs || sp.part < 0) return false;
    const SeqRange r = seq_range(A.sq, sp.seq);
    const int64_t t0 = (int64_t)sp.part * A.tile;
    out->slot = seq_slot(A.sq, sp.seq);
    if (t0 >= r.len || out->slot < 0) return false;
    out->seq = sp.seq;
    out->t0 = (int)t0;
    out->len = (int)r.len;
    out->row0 = r.first;
    out->head = block * A.pack;
    out->kv_head = out->head / A.rep;
    out->keys = seq_keys(A, sp.seq, out->slot, r, &out->key0);
    return true;
}

// Element offset of a key's row, in k or v.
__device__ __forceinline__ int64_t key_row(const SoftArgs& A, const SoftPlace& pl, const CachePlace& c, int key) {
    if (!A.paged) return (pl.key0 + key) * c.row + pl.kv_head * c.head;
    const int page = A.table[pl.slot * A.max_pages + (key >> A.shift)];
    const int64_t p = min<int64_t>(max(page, 0), A.pages - 1);
    return p * c.page + (key & ((1 << A.shift) - 1)) * c.row + pl.kv_head * c.head;
}

// 16 bytes of a row of `dim` elements from unit u (of 16 bytes) on, zeros past its end.
template <typename T, bool VEC>
__device__ __forceinline__ u32x4 load_unit(const T* row, int u, int dim) {
    constexpr int E = 16 / sizeof(T);
    const int c = u * E;
    u32x4 v{0, 0, 0, 0};
    if constexpr (VEC) {
        if (c < dim) v = *reinterpret_cast<const u32x4_any*>(row + c);
    } else {
        T e[E];
#pragma unroll
        for (int i = 0; i < E; ++i) e[i] = c + i < dim ? row[c + i] : (T)0;
        __builtin_memcpy(&v, e, 16);
    }
    return v;
}

__device__ __forceinline__ float other_half(float v) { return __shfl_xor(v, 32); }

typedef short s16x4 __attribute__((ext_vector_type(4)));

// Where LDS holds unit u (16 bytes) of a row of k or v, in units.
template <int UNITS>
__device__ __forceinline__ int k_unit(int row, int u) { return row * UNITS + (u ^ (row & 7)); }
template <int UNITS>
__device__ __forceinline__ int v_unit(int row, int u) {
    const int f = UNITS >= 16 ? 4 * (row & 3) ^ 2 * (row >> 2 & 1) : 4 * (row >> 1 & 1) ^ 2 * (row >> 2 & 1);
    return row * UNITS + (u ^ f);
}

template <typename T>
struct SoftMath;

template <>
struct SoftMath<uint16_t> {
    static __device__ __forceinline__ f32x16 score(u32x4 k, u32x4 q, f32x16 s) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, k), __builtin_bit_cast(bf16x8, q), s, 0, 0, 0);
    }
    static __device__ __forceinline__ u32x4 sign(u32x4 q, int sign) {
        const uint32_t flip = sign < 0 ? 0x80008000u : 0u, on = sign ? ~0u : 0u;
#pragma unroll
        for (int i = 0; i < 4; ++i) q[i] = (q[i] ^ flip) & on;
        return q;
    }
};
template <>
struct SoftMath<float> {
    static __device__ __forceinline__ f32x16 score(u32x4 k, u32x4 q, f32x16 s) {
        const f32x4 a = __builtin_bit_cast(f32x4, k), b = __builtin_bit_cast(f32x4, q);
#pragma unroll
        for (int i = 0; i < 4; ++i) s = __builtin_amdgcn_mfma_f32_32x32x2f32(a[i], b[i], s, 0, 0, 0);
        return s;
    }
    static __device__ __forceinline__ u32x4 sign(u32x4 q, int sign) {
        const uint32_t flip = sign < 0 ? 0x80000000u : 0u, on = sign ? ~0u : 0u;
#pragma unroll
        for (int i = 0; i < 4; ++i) q[i] = (q[i] ^ flip) & on;
        return q;
    }
};

// A row's view of the keys.
struct RowMask {
    int limit;      // keys below this (TREE: of those before the sequence's own) are seen
    int own0;       // TREE: number of the first own key
    uint64_t own;   // TREE: own keys that are seen
    __device__ __forceinline__ bool sees(int key) const {
        const int i = key - own0;
        return key < limit || ((uint32_t)i < 64u && (own >> (i & 63) & 1));
    }
};
// ... of row t (t < 0: of none).  end: behind the last key that it sees; full: it sees all before this.
__device__ __forceinline__ RowMask row_mask(const SoftArgs& A, const SoftPlace& pl, int t) {
    RowMask m{pl.keys, 0x7fffffff, 0};
    if (t < 0) m.limit = 0;
    else if (A.mask == SEQMIX_MASK_CAUSAL) m.limit = min(max(pl.keys - pl.len + t + 1, 0), pl.keys);
    else if (A.mask == SEQMIX_MASK_TREE) {
        m.limit = max(pl.keys - pl.len, 0);
        m.own0 = pl.keys - pl.len;
        m.own = (uint64_t)A.tree[pl.row0 + t] & (pl.len < 64 ? (1ull << pl.len) - 1 : ~0ull);
    }
    return m;
}

constexpr float kSlack = 8.0f;  // weights are below 2^8 then

// The state of 32 rows of a wave.
template <typename T, int DKP, int DVP>
struct SoftRows {
    static constexpr int E = 16 / sizeof(T), KU = DKP / E, VU = DVP / E, MT = DVP / 32;
    u32x4 q[KU / 2];
    f32x16 o[MT];
    float m, l;

    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[mt][i] = 0.0f;
        m = -FLT_MAX;
        l = 0.0f;
    }

    // Scores of 32 keys, from row `row` of the tile in LDS on.
    __device__ __forceinline__ f32x16 scores(const u32x4* sK, int row) const {
        const int n = threadIdx.x & 31, h = threadIdx.x >> 5 & 1;
        f32x16 s;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = 0.0f;
#pragma unroll
        for (int c = 0; c < KU / 2; ++c) s = SoftMath<T>::score(sK[k_unit<KU>(row + n, 2 * c + h)], q[c], s);
        return s;
    }

    // Adds 32 keys with weights p (as scores() leaves them).  CAREFUL: values that are not finite count only for rows that see
    // them (`seen`, a bit for each of p), and make them NaN.
    template <bool CAREFUL>
    __device__ __forceinline__ void add(const u32x4* sV, int row, const f32x16& p, uint32_t seen) {
        const int l64 = threadIdx.x & 63, h = l64 >> 5;
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                bf16x8 hi, lo, on;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    hi[j] = (__bf16)p[8 * c + j];
                    lo[j] = (__bf16)(p[8 * c + j] - (float)hi[j]);
                    if constexpr (CAREFUL) on[j] = (__bf16)((seen >> (8 * c + j)) & 1 ? 1.0f : 0.0f);
                }
                const int r0 = row + 16 * c + 4 * h + (l64 & 15) / 4, col = 16 * (l64 >> 4 & 1) + 4 * (l64 & 3);
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    u32x4 v;
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        const int r = r0 + 8 * x;
                        const char* at = reinterpret_cast<const char*>(sV) + v_unit<VU>(r, (32 * mt + col) / 8) * 16 + (col & 4) * 2;
                        const u32x2 w = __builtin_bit_cast(
                            u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)at));
                        v[2 * x] = w[0];
                        v[2 * x + 1] = w[1];
                    }
                    if constexpr (CAREFUL) {
                        u32x4 odd;
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const bool a = (v[i] & 0x7f80u) == 0x7f80u, b = (v[i] & 0x7f800000u) == 0x7f800000u;
                            odd[i] = (a ? 0x3f80u : 0u) | (b ? 0x3f800000u : 0u);
                            v[i] &= (a ? 0u : 0xffffu) | (b ? 0u : 0xffff0000u);
                        }
                        f32x16 count;
#pragma unroll
                        for (int i = 0; i < 16; ++i) count[i] = 0.0f;
                        count = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, odd), on, count, 0, 0, 0);
#pragma unroll
                        for (int i = 0; i < 16; ++i) o[mt][i] = count[i] > 0.0f ? NAN : o[mt][i];
                    }
                    o[mt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v), hi, o[mt], 0, 0, 0);
                    o[mt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v), lo, o[mt], 0, 0, 0);
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int r = row + 8 * (i / 4) + 4 * h + i % 4;
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    const int col = 32 * mt + (l64 & 31);
                    float v = reinterpret_cast<const float*>(sV + v_unit<VU>(r, col / 4))[col & 3];
                    if constexpr (CAREFUL) {
                        const bool odd = !(__builtin_fabsf(v) <= FLT_MAX);
                        f32x16 count;
#pragma unroll
                        for (int j = 0; j < 16; ++j) count[j] = 0.0f;
                        count = __builtin_amdgcn_mfma_f32_32x32x2f32(odd ? 1.0f : 0.0f, seen >> i & 1 ? 1.0f : 0.0f, count, 0, 0, 0);
#pragma unroll
                        for (int j = 0; j < 16; ++j) o[mt][j] = count[j] > 0.0f ? NAN : o[mt][j];
                        v = odd ? 0.0f : v;
                    }
                    o[mt] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, p[i], o[mt], 0, 0, 0);
                }
            }
        }
    }

    // One tile of KT keys, of which lane i of s[b] is key key0 + 32 b + 8 (i / 4) + 4 h + i % 4.
    template <int KT, bool CAREFUL>
    __device__ __forceinline__ void step(const u32x4* sK, const u32x4* sV, int key0, bool masked, const RowMask& mask,
                                         float scale2) {
        constexpr int NB = KT / 32;
        const int h = threadIdx.x >> 5 & 1;
        f32x16 s[NB];
        uint32_t seen[NB];
        float mx = -INFINITY;
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            s[b] = scores(sK, 32 * b);
            seen[b] = 0xffff;
        }
        if (masked) {
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                seen[b] = 0;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const bool on = mask.sees(key0 + 32 * b + 8 * (i / 4) + 4 * h + i % 4);
                    s[b][i] = on ? s[b][i] : -INFINITY;
                    seen[b] |= on ? 1u << i : 0u;
                }
            }
        }
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[b][i]);
        mx = fmaxf(mx, other_half(mx)) * scale2;
        // sums are relative to a maximum that may be up to kSlack behind: most tiles leave them as they are
        if (__any(mx > m + kSlack)) {
            const float now = fmaxf(m, mx);
            const float fade = __builtin_amdgcn_exp2f(m - now);
            m = now;
            l *= fade;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[mt][i] *= fade;
        }
#pragma unroll
        for (int b = 0; b < NB; ++b) {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                s[b][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][i], scale2, -m));
                l += s[b][i];
            }
            add<CAREFUL>(sV, 32 * b, s[b], seen[b]);
        }
    }

    // Whether a value that is not finite came up (in any lane): what rows that do not see it hold has to be computed again.
    __device__ __forceinline__ bool spoilt() const {
        float bad = l * 0.0f;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int i = 0; i < 16; ++i) bad += o[mt][i] * 0.0f;
        return __any(!(bad == 0.0f));
    }
};

template <typename T, bool VEC>
__device__ __forceinline__ void store4(T* p, int live, f32x4 v) {
    if (VEC || live >= 4) {
        if (live > 0) {
            const float w[4] = {v[0], v[1], v[2], v[3]};
            store_pack<T, 4>(p, w);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (i < live) p[i] = from_f32<T>(v[i]);
    }
}

// A wave's 64 units of 16 bytes go from memory to LDS, from `to` on, without passing registers.  The compiler does not count
// these loads: loads_done() waits for them.
__device__ __forceinline__ void load_to_lds(__amdgpu_buffer_rsrc_t r, uint32_t off, const u32x4* to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(
                     __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)to)),
                 "v"(off), "s"(r)
                 : "memory");
}
__device__ __forceinline__ void loads_done() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// Loads the rows of tiles of keys (or values) into LDS, RI rows per instruction of a wave.  What lies past the last key or past a
// row's end reads as zero by the buffer's range.  In pages, at least RI rows of a page follow each other, and the
// pages of a tile are looked up (next) one tile before it is loaded.
template <typename T, int UNITS, int KT, bool OF_K>
struct DirectLoad {
    static constexpr int E = 16 / sizeof(T), RI = 64 / UNITS, N = KT / RI / 4;
    static constexpr int KINDS = RI == 1 ? 2 : 1;  // an instruction's rows are in LDS in one of these orders
    const T* base;
    uint32_t off[KINDS];  // of this lane, in bytes
    int page;             // lane i < N: of instruction i
    uint32_t row_bytes, last;  // last: bytes of a row that count

    __device__ __forceinline__ DirectLoad(const SoftArgs& A, const SoftPlace& pl, const void* p, const CachePlace& c, int dim) {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane / UNITS, at = lane % UNITS;
        base = static_cast<const T*>(p) + pl.kv_head * c.head + (A.paged ? 0 : pl.key0 * c.row);
        row_bytes = (uint32_t)c.row * sizeof(T);
        last = dim * sizeof(T);
        page = 0;
#pragma unroll
        for (int i = 0; i < KINDS; ++i) {
            const int row = first_row(i, wave) + r;
            const int u = (OF_K ? k_unit<UNITS>(row, at) : v_unit<UNITS>(row, at)) - row * UNITS;
            off[i] = u * E < dim ? r * row_bytes + u * 16 : OOB_OFF;
        }
    }
    static __device__ __forceinline__ int first_row(int i, int wave) { return (4 * i + wave) * RI; }
    __device__ __forceinline__ void next(const SoftArgs& A, const SoftPlace& pl, int key0) {
        if (!A.paged) return;
        const int key = key0 + first_row(threadIdx.x & 63, threadIdx.x >> 6);
        page = (threadIdx.x & 63) < N && key < pl.keys ? A.table[pl.slot * A.max_pages + (key >> A.shift)] : 0;
    }
    __device__ __forceinline__ void tile(const SoftArgs& A, const SoftPlace& pl, const CachePlace& c, int key0, const u32x4* to) const {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int in_page = A.paged ? (1 << A.shift) - 1 : -1;  // (packed: all in page 0)
        int at[N];
#pragma unroll
        for (int i = 0; i < N; ++i) at[i] = min(max(__builtin_amdgcn_readlane(page, i), 0), (int)A.pages - 1);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int row = first_row(i, wave), key = key0 + row;
            const int left = pl.keys - key;
            const T* p = base + at[i] * c.page + (int64_t)(key & in_page) * c.row;
            load_to_lds(make_rsrc(p, left > 0 ? (uint32_t)(min(left, RI) - 1) * row_bytes + last : 0u), off[i % KINDS],
                        to + row * UNITS);
        }
    }
};

template <typename T, int DKP, int DVP, int KT, bool VEC>
__global__ __launch_bounds__(256, DKP + DVP <= 256 ? 2 : 1) void softmax_prompt_kernel(SoftArgs A) {
    using R = SoftRows<T, DKP, DVP>;
    constexpr int KU = R::KU, VU = R::VU;
    __shared__ u32x4 sK[(VEC ? 2 : 1) * KT * KU], sV[(VEC ? 2 : 1) * KT * VU];
    const int tid = threadIdx.x, wave = tid >> 6, n = tid & 31, h = tid >> 5 & 1;
    const uint32_t at = blockIdx.x / (uint32_t)A.blocks;
    SoftPlace pl;
    if (!soft_place(A, (uint32_t)A.ids - 1 - at, (int)(blockIdx.x - at * A.blocks), &pl)) return;

    // this lane's row, and the rows of its wave and of the workgroup
    const int row = 32 * wave + n;
    const int t = pl.t0 + row / A.pack, head = pl.head + row % A.pack;
    const bool live = row < A.tile * A.pack && t < pl.len;
    const RowMask mask = row_mask(A, pl, live ? t : -1);
    const bool causal = A.mask == SEQMIX_MASK_CAUSAL, tree = A.mask == SEQMIX_MASK_TREE;
    const int back = pl.keys - pl.len;
    auto behind = [&](int tt) { return causal ? min(max(back + min(tt, pl.len - 1) + 1, 0), pl.keys) : pl.keys; };
    const int end = behind(pl.t0 + A.tile - 1);
    const int w0 = pl.t0 + 32 * wave / A.pack;
    const int wave_end = w0 < pl.len ? behind(pl.t0 + (32 * wave + 31) / A.pack) : 0;
    const int wave_full = tree ? max(back, 0) : behind(w0);

    R rows;
    const T* q = static_cast<const T*>(A.q) + (pl.row0 + t) * A.q_row + (int64_t)head * A.q_head;
#pragma unroll
    for (int c = 0; c < KU / 2; ++c) {
        rows.q[c] = u32x4{0, 0, 0, 0};
        if (live) rows.q[c] = SoftMath<T>::sign(load_unit<T, VEC>(q, 2 * c + h, A.dk), A.qsign);
    }

    auto pass = [&](auto careful) {
        auto step = [&](const u32x4* k, const u32x4* v, int key0) {
            if (key0 < wave_end)
                rows.template step<KT, decltype(careful)::value>(k, v, key0, key0 + KT > wave_full, mask, A.scale2);
        };
        rows.clear();
        if constexpr (VEC) {
            DirectLoad<T, KU, KT, true> load_k(A, pl, A.k, A.kp, A.dk);
            DirectLoad<T, VU, KT, false> load_v(A, pl, A.v, A.vp, A.dv);
            auto load = [&](int key0, int b) {  // ... and the pages of the tile after it
                load_k.tile(A, pl, A.kp, key0, sK + b * KT * KU);
                load_v.tile(A, pl, A.vp, key0, sV + b * KT * VU);
                load_k.next(A, pl, key0 + KT);
                load_v.next(A, pl, key0 + KT);
            };
            load_k.next(A, pl, 0);
            load_v.next(A, pl, 0);
            int b = 0;
            if (end > 0) load(0, 0);
            for (int key0 = 0; key0 < end; key0 += KT, b ^= 1) {
                loads_done();
                __syncthreads();  // this tile is there, and the one before has been used
                if (key0 + KT < end) load(key0 + KT, b ^ 1);
                step(sK + b * KT * KU, sV + b * KT * VU, key0);
            }
            __syncthreads();
        } else {
            for (int key0 = 0; key0 < end; key0 += KT) {
                __syncthreads();
                for (int x = tid; x < KT * KU; x += 256) {
                    const int r = x / KU, u = x % KU;
                    const int64_t from = key_row(A, pl, A.kp, min(key0 + r, pl.keys - 1));
                    sK[k_unit<KU>(r, u)] = load_unit<T, VEC>(static_cast<const T*>(A.k) + from, u, A.dk);
                }
                for (int x = tid; x < KT * VU; x += 256) {
                    const int r = x / VU, u = x % VU;
                    const int64_t from = key_row(A, pl, A.vp, min(key0 + r, pl.keys - 1));
                    sV[v_unit<VU>(r, u)] = load_unit<T, VEC>(static_cast<const T*>(A.v) + from, u, A.dv);
                }
                __syncthreads();
                step(sK, sV, key0);
            }
        }
    };
    pass(std::false_type{});
    __shared__ int s_again;
    if (tid == 0) s_again = 0;
    __syncthreads();
    if (rows.spoilt()) s_again = 1;
    __syncthreads();
    if (s_again) pass(std::true_type{});

    const float l = rows.l + other_half(rows.l);
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    if (!live) return;
    T* o = static_cast<T*>(A.o) + (pl.row0 + t) * A.o_row + (int64_t)head * A.o_head;
#pragma unroll
    for (int mt = 0; mt < R::MT; ++mt)
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const int c = 32 * mt + 8 * b + 4 * h;
            const f32x4 v{rows.o[mt][4 * b], rows.o[mt][4 * b + 1], rows.o[mt][4 * b + 2], rows.o[mt][4 * b + 3]};
            store4<T, VEC>(o + c, A.dv - c, v * inv);
        }
}

template <typename T, int DKP, int DVP, int KT, bool VEC>
hipError_t launch_softmax_prompt(const SoftArgs& a, hipStream_t s) {
    hipLaunchKernelGGL((softmax_prompt_kernel<T, DKP, DVP, KT, VEC>), dim3((unsigned)(a.ids * a.blocks)), dim3(256), 0, s, a);
    return hipGetLastError();
}

// Kernels for heads of up to 64, 128 and 256 elements; of dims that fill no 16 bytes, by the larger of the two.
template <typename T, int WIDE>
hipError_t launch_softmax(const SoftArgs& a, bool vec, hipStream_t s) {
    const int k = a.dk <= 64 ? 64 : a.dk <= 128 ? 128 : 256, v = a.dv <= 64 ? 64 : a.dv <= 128 ? 128 : 256;
    if (!vec) {
        const int d = k > v ? k : v;
        if (d == 64) return launch_softmax_prompt<T, 64, 64, 64, false>(a, s);
        if (d == 128) return launch_softmax_prompt<T, 128, 128, 64, false>(a, s);
        return launch_softmax_prompt<T, 256, 256, WIDE, false>(a, s);
    }
    switch (1000 * k + v) {
        case 64064: return launch_softmax_prompt<T, 64, 64, 64, true>(a, s);
        case 64128: return launch_softmax_prompt<T, 64, 128, 64, true>(a, s);
        case 64256: return launch_softmax_prompt<T, 64, 256, WIDE, true>(a, s);
        case 128064: return launch_softmax_prompt<T, 128, 64, 64, true>(a, s);
        case 128128: return launch_softmax_prompt<T, 128, 128, 64, true>(a, s);
        case 128256: return launch_softmax_prompt<T, 128, 256, WIDE, true>(a, s);
        case 256064: return launch_softmax_prompt<T, 256, 64, WIDE, true>(a, s);
        case 256128: return launch_softmax_prompt<T, 256, 128, WIDE, true>(a, s);
        default: return launch_softmax_prompt<T, 256, 256, WIDE, true>(a, s);
    }
}

}  // namespace cv
