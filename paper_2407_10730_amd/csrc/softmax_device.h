// softmax_device.h -- the softmax attention kernels, for bf16 and fp32.
//
// A tile is 32 rows per wave, a row being a token for one head.  Scores are computed transposed, 32 keys x 32 rows per matrix
// instruction, so that a lane holds 16 keys of one row: the running maximum and sum of the softmax need no exchange but
// between the two halves of a wave, and the weights are already the operand of the product with v: the rows
// of the result that lane half h holds are keys 8 b + 4 h + i (b, i < 4), and v is read in that order.
#pragma once

#include <algorithm>
#include <cfloat>
#include <type_traits>

#include "seqmix_device.h"

namespace cv {

// The arguments of the running kernel, its only parameter, to be read where they are used: held from the start on they fill the
// scalar registers and are kept in lanes of vector registers, which cost two thousand instructions (16 requests of 24
// drafts over up to 5000 keys 58 -> 54 us).
__device__ __forceinline__ const SoftArgs& args_here() {
    auto p = (const __attribute__((address_space(4))) SoftArgs*)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
    return *(const SoftArgs*)p;
}

// What a workgroup works on: a unit is rows [t0, t0 + tile) of a sequence for the heads from `head` on; a part of it is its keys
// [first, last).
struct SoftPlace {
    int head, kv_head;
    int t0, len, keys;
    int first, last;
    int64_t row0, slot;
    int64_t key0;           // packed: first row of the sequence's keys
    uint32_t part, parts;   // of the unit; part p is that of share `share` + p
    uint32_t share;

    // All of it in scalar registers (it is the same for all threads, which the compiler does not see everywhere).
    __device__ __forceinline__ void uniform() {
        auto one = [](auto& v) { v = __builtin_amdgcn_readfirstlane(v); };
        auto two = [](int64_t& v) {
            v = (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32 |
                          (uint32_t)__builtin_amdgcn_readfirstlane((int)v));
        };
        one(head), one(kv_head), one(t0), one(len), one(keys), one(first), one(last), one(part), one(parts), one(share);
        two(row0), two(slot), two(key0);
    }
};

__device__ __forceinline__ int seq_keys(const SoftArgs& A, int seq, int64_t slot, const SeqRange& r, int64_t* first) {
    *first = 0;
    if (A.table) {
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

__device__ __forceinline__ void soft_heads(const SoftArgs& A, int block, SoftPlace* out) {
    out->head = block * A.pack;
    out->kv_head = (int)fdiv(out->head, A.by_rep);
}

// Unit `id` of a block of heads, all of its keys.  False: there is none (in all threads).
__device__ __forceinline__ bool soft_unit(const SoftArgs& A, uint32_t id, int block, SoftPlace* out) {
    const SeqPart sp = seq_part(A.sq, id, (uint32_t)A.tile);
    if (sp.seq >= A.sq.seqs || sp.part < 0) return false;
    const SeqRange r = seq_range(A.sq, sp.seq);
    const int64_t t0 = (int64_t)sp.part * A.tile;
    out->slot = seq_slot(A.sq, sp.seq);
    if (t0 >= r.len || out->slot < 0) return false;
    soft_heads(A, block, out);
    out->t0 = (int)t0;
    out->len = (int)r.len;
    out->row0 = r.first;
    out->keys = seq_keys(A, sp.seq, out->slot, r, &out->key0);
    out->first = 0;
    out->last = out->keys;
    out->part = out->share = 0;
    out->parts = 1;
    return true;
}

// n / d and what is left, for quotients below 2^22 (the product in single precision is off by 2^-22 of them, less than 1), and for n
// up to 2^31 where d is a power of two of 256 or more.
__device__ __forceinline__ uint32_t quotient(uint32_t n, uint32_t d, uint32_t* left) {
    uint32_t q = (uint32_t)((float)n * __builtin_amdgcn_rcpf((float)d));
    int32_t m = (int32_t)(n - q * d);
    if (m < 0) --q, m += d;
    if (m >= (int32_t)d) ++q, m -= d;
    *left = (uint32_t)m;
    return q;
}
// ... of the last lane.
__device__ __forceinline__ uint32_t last_lane(uint32_t v) { return (uint32_t)__builtin_amdgcn_readlane((int)v, 63); }

// Shares.  Where units alone would not fill the card evenly, what there is to do is put in a row: the keys of a unit in
// quanta, unit after unit, sequence after sequence, block of heads after block of heads.  Each workgroup takes a share of the
// same number of quanta, which may begin and end inside units; parts of a unit are joined by the one that is done last.
// Every wave finds its share from the lengths of all sequences (a lane each), so nothing needs to be known on the host.  Where no
// unit has more than A.whole quanta, units are not divided: a share is a unit.
struct SoftSeq {
    uint32_t row0, len, keys, key0;
    int slot;
    uint32_t tiles, first, grow;  // tile t has first + grow t quanta
    __device__ __forceinline__ uint32_t quanta(uint32_t n) const { return n * first + grow * (n * (n - 1) / 2); }  // of n tiles
    __device__ __forceinline__ uint32_t longest() const { return tiles ? first + grow * (tiles - 1) : 0; }
};
__device__ __forceinline__ SoftSeq soft_seq(const SoftArgs& A, int i) {
    SoftSeq s{0, 0, 0, 0, -1, 0, 0, 0};
    // what is at hand is asked for at once: one after the other finding a workgroup's share took 5500 cycles, so 3600
    const int at = min(i, A.sq.seqs - 1);
    int64_t b = (int64_t)at * A.sq.seq_len, e = b + A.sq.seq_len, kb = 0, ke = 0;
    int slot = at;
    if (A.sq.off) b = A.sq.off[at], e = A.sq.off[at + 1];
    if (A.sq.slot) slot = A.sq.slot[at];
    if (A.koff) kb = A.koff[at], ke = A.koff[at + 1];
    const bool live = i < A.sq.seqs && slot >= 0 && (!A.sq.slot || slot < A.sq.slots);
    const int len = A.table ? A.lens[live ? slot : 0] : 0;
    if (!live) return s;
    const uint32_t b0 = clamp_row(b, A.sq.tokens), e0 = clamp_row(e, A.sq.tokens);
    s.slot = slot;
    s.row0 = b0;
    s.len = e0 > b0 ? e0 - b0 : 0;
    if (A.table) {
        s.keys = (uint32_t)min<int64_t>(max(len, 0), A.max_pages << A.shift);
    } else if (!A.koff) {
        s.key0 = s.row0;
        s.keys = s.len;
    } else {
        const uint32_t kb0 = clamp_row(kb, A.key_tokens), ke0 = clamp_row(ke, A.key_tokens);
        s.key0 = kb0;
        s.keys = ke0 > kb0 ? ke0 - kb0 : 0;
    }
    uint32_t left;
    s.tiles = quotient(s.len + A.tile - 1, A.tile, &left);
    const uint32_t round = (1u << A.quantum) - 1;
    s.first = max((s.keys + round) >> A.quantum, 1u);
    if (A.grow && s.tiles > 1 && s.keys >= s.len) {  // the triangle of a causal mask
        s.first = (s.keys - s.len + A.tile + round) >> A.quantum;
        s.grow = A.grow;
    }
    return s;
}

struct SoftShares {
    uint32_t each;       // quanta (or units) of a block of heads
    uint32_t size;       // of a share
    bool whole;          // units are not divided
    uint32_t share;      // this workgroup's: neighbouring ones go to one XCD, where they find keys and values in its L2, those
                         // that there are to all XCDs alike (4 requests of 24 drafts over up to 2000 keys 35 -> 28 us)
    uint32_t at, stop;
    bool none;           // it has nothing to do
    SoftSeq seq;         // of this lane (up to 64 sequences)

    __device__ __forceinline__ uint32_t weight(const SoftSeq& s) const { return whole ? s.tiles : s.quanta(s.tiles); }

    // Without shares workgroup n has one unit, the last ones (the longest of a prompt) first.
    __device__ __forceinline__ explicit SoftShares(const SoftArgs& A) {
        at = share = (uint32_t)A.first + blockIdx.x;
        stop = at + 1;
        none = false;
        if (!A.shares) return;
        const int lane = threadIdx.x & 63;
        seq = soft_seq(A, lane);
        whole = false;
        uint32_t work = weight(seq), units = seq.tiles, most = seq.longest();
#pragma unroll 1
        for (int c = 64; c < A.sq.seqs; c += 64) {
            const SoftSeq x = soft_seq(A, c + lane);
            work += weight(x);
            units += x.tiles;
            most = max(most, x.longest());
        }
        units = last_lane(scan_lanes(units));
        each = last_lane(scan_lanes(work));
        whole = __ballot(most > (uint32_t)A.whole) == 0 && units * A.blocks <= (uint32_t)A.shares;
        // (offsets that lie may make it more than the host counted on)
        if (!(lanes_sum<64>((float)work) <= (float)A.most) || units > (uint32_t)A.most) each = units = 0;
        uint32_t left;
        if (whole) {
            each = units;
            size = 1;
        } else {
            size = max(quotient(each * A.blocks + A.shares - 1, A.shares, &left), (uint32_t)A.least);
        }
        const uint32_t all = each * A.blocks;
        const uint32_t used = quotient(all + size - 1, size, &left);
        if (share < used) share = (uint32_t)xcd_remap((int)share, (int)used);
        at = min(share * size, all);
        stop = min(at + size, all);
        none = at >= stop;
    }

    // The part that begins at `at`, which moves to its end.
    __device__ __forceinline__ bool next(const SoftArgs& A, SoftPlace* out) {
        if (at >= stop) return false;
        uint32_t y;
        if (!A.shares) {
            const uint32_t id = fdiv(at, A.by_blocks);
            y = at++ - id * A.blocks;
            return soft_unit(A, (uint32_t)A.ids - 1 - id, (int)y, out);
        }
        soft_heads(A, (int)quotient(at, each, &y), out);
        uint32_t before = 0;
#pragma unroll 1
        for (int c = 0; c < A.sq.seqs; c += 64) {
            const SoftSeq s = A.sq.seqs > 64 ? soft_seq(A, c + (threadIdx.x & 63)) : seq;
            const uint32_t mine = weight(s), up = before + scan_lanes(mine), start = up - mine;
            const uint64_t hit = __ballot(y >= start && y - start < mine);
            if (hit) {
                const int l = __builtin_ctzll(hit);
                auto get = [&](uint32_t v) { return (uint32_t)__builtin_amdgcn_readlane((int)v, l); };
                SoftSeq u;
                u.len = get(s.len), u.keys = get(s.keys), u.first = get(s.first), u.grow = get(s.grow), u.tiles = get(s.tiles);
                const uint32_t in = y - get(start);
                out->slot = (int)get((uint32_t)s.slot);
                out->row0 = get(s.row0);
                out->key0 = get(s.key0);
                out->len = (int)u.len;
                out->keys = (int)u.keys;
                if (whole) {
                    out->t0 = (int)(in * A.tile);
                    out->first = 0;
                    out->last = (int)u.keys;
                    out->part = out->share = 0;
                    out->parts = 1;
                    ++at;
                    return true;
                }
                uint32_t tile, left;
                if (u.grow == 0) {
                    tile = quotient(in, u.first, &left);
                } else {  // the last whose tiles before it have `in` quanta at most: near the root of a quadratic
                    const float a = (float)u.first / (float)u.grow - 0.5f;
                    tile = (uint32_t)__builtin_amdgcn_readfirstlane(
                        (int)fminf(fmaxf(__builtin_amdgcn_sqrtf(a * a + 2.0f * (float)in / (float)u.grow) - a, 0.0f),
                                   (float)(u.tiles - 1)));
                    while (tile && u.quanta(tile) > in) --tile;
                    while (tile + 1 < u.tiles && u.quanta(tile + 1) <= in) ++tile;
                }
                const uint32_t unit = at - in + u.quanta(tile);  // where the unit begins
                const uint32_t behind = unit + u.first + u.grow * tile, end = min(stop, behind);
                out->t0 = (int)tile * A.tile;
                out->first = (int)min((at - unit) << A.quantum, u.keys);
                out->last = (int)min((end - unit) << A.quantum, u.keys);
                out->share = quotient(unit, size, &left);
                out->part = quotient(at, size, &left) - out->share;
                out->parts = quotient(behind - 1, size, &left) - out->share + 1;
                at = end;
                return true;
            }
            before = last_lane(up);
        }
        return false;
    }
};

// Element offset of a key's row, in k or v.
__device__ __forceinline__ int64_t key_row(const SoftArgs& A, const SoftPlace& pl, const CachePlace& c, int key) {
    if (!A.table) return (pl.key0 + key) * c.row + pl.kv_head * c.head;
    const int page = A.table[pl.slot * A.max_pages + (key >> A.shift)];
    const int64_t p = min<int64_t>(max(page, 0), A.pages - 1);
    return p * c.page + (key & ((1 << A.shift) - 1)) * c.row + pl.kv_head * c.head;
}

// 16 bytes, moved down by `bits` (below 128), zeros behind them.
__device__ __forceinline__ u32x4 moved_down(u32x4 v, uint32_t bits) {
    if (bits & 64) v = u32x4{v[2], v[3], 0, 0};
    if (bits & 32) v = u32x4{v[1], v[2], v[3], 0};
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = (uint32_t)(((uint64_t)(i < 3 ? v[i + 1] : 0u) << 32 | v[i]) >> (bits & 31));
    return w;
}

// 16 bytes of a row of `dim` elements from unit u (of 16 bytes) on, zeros past its end, at any address of the element's
// alignment: the last part is read where it ends with the row, and moved down; rows below 16 bytes are read by elements.
template <typename T>
__device__ __forceinline__ u32x4 load_unit(const T* row, int u, int dim) {
    constexpr int E = 16 / sizeof(T);
    const int c = u * E;
    u32x4 v{0, 0, 0, 0};
    if (dim >= E) {
        const int over = max(c + E - dim, 0);  // elements
        if (c < dim) v = moved_down(*reinterpret_cast<const u32x4_any*>(row + c - over), over * 8 * sizeof(T));
    } else {
        T e[E];
#pragma unroll
        for (int i = 0; i < E; ++i) e[i] = c + i < dim ? row[c + i] : (T)0;
        __builtin_memcpy(&v, e, 16);
    }
    return v;
}

// v of lane l and of lane l ^ 32, in either order.
__device__ __forceinline__ u32x2 both_halves(float v) {
    const uint32_t w = __builtin_bit_cast(uint32_t, v);
    const auto r = __builtin_amdgcn_permlane32_swap(w, w, false, false);
    return u32x2{r[0], r[1]};
}
__device__ __forceinline__ float max_of_halves(float v) {
    const f32x2 w = __builtin_bit_cast(f32x2, both_halves(v));
    return fmaxf(w[0], w[1]);
}
__device__ __forceinline__ float sum_of_halves(float v) {
    const f32x2 w = __builtin_bit_cast(f32x2, both_halves(v));
    return w[0] + w[1];
}

typedef short s16x4 __attribute__((ext_vector_type(4)));

// Where LDS holds unit u (16 bytes) of a row of k or v, in units.  An instruction that loads past registers fills 64 units in a
// row (RI rows); which rows and units those are, and where the next 64 begin, is free.  It is chosen such that what
// one access takes lies in distinct banks: 16 rows of one unit of k, four rows of four or eight rows of two units of v
// (8192 tokens, 16 heads of 128: a third of the LDS cycles were conflicts where 16 rows shared 8 places).
template <int UNITS>
struct KeyTile {
    static constexpr int RI = 64 / UNITS, TURN = RI >= 4 ? 3 : RI - 1, PAD = RI >= 4 ? 4 : RI;
    static constexpr int GROUP = 64 + PAD;  // units from RI rows to the next
    static __host__ __device__ constexpr int turn(int row) { return RI == 8 ? row >> 1 & 3 : row & TURN; }
    static __host__ __device__ constexpr int at(int row, int u) { return row / RI * GROUP + row % RI * UNITS + (u ^ turn(row)); }
    static constexpr int units(int rows) { return rows / RI * GROUP; }
};
template <int UNITS>
struct ValueTile {
    static constexpr int RI = 64 / UNITS, GROUP = 64;
    static __host__ __device__ constexpr int turn(int row) {
        return UNITS >= 16 ? 4 * (row & 3) ^ 2 * (row >> 2 & 1) : 4 * (row >> 1 & 1) ^ 2 * (row >> 2 & 1);
    }
    static __host__ __device__ constexpr int at(int row, int u) { return row * UNITS + (u ^ turn(row)); }
    static constexpr int units(int rows) { return rows * UNITS; }
};

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
    // Bit i: whether key key0 + i is seen.
    __device__ __forceinline__ uint64_t bits(int key0) const {
        const int n = limit - key0, d = own0 - key0;
        const uint64_t before = n >= 64 ? ~0ull : n > 0 ? (1ull << n) - 1 : 0ull;
        const uint64_t mine = d >= 64 || d <= -64 ? 0ull : d >= 0 ? own << d : own >> -d;
        return before | mine;
    }
};
// ... of row t (t < 0: of none).  end: behind the last key that it sees; full: it sees all before this.
__device__ __forceinline__ RowMask row_mask(const SoftArgs& A, const SoftPlace& pl, int t) {
    RowMask m{pl.keys, 0, 0};
    if (t < 0) m.limit = 0;
    else if (A.mask == SEQMIX_MASK_CAUSAL) m.limit = min(max(pl.keys - pl.len + t + 1, 0), pl.keys);
    else if (A.mask == SEQMIX_MASK_TREE) {
        m.limit = max(pl.keys - pl.len, 0);
        m.own0 = pl.keys - pl.len;
        m.own = (uint64_t)A.tree[pl.row0 + t] & (pl.len < 64 ? (1ull << pl.len) - 1 : ~0ull);
    }
    return m;
}

constexpr int kMfma = 0x8, kDsRead = 0x100, kValu = 0x2, kTrans = 0x400;  // kinds of instructions, for sched_group_barrier
constexpr int PLANES = 2;  // bf16 parts of a weight, where rows are few (of prompts one)
constexpr float kSlack = 8.0f;  // weights are below 2^8 then

// The state of 32 rows of a wave.
template <typename T, int DKP, int DVP>
struct SoftRows {
    static constexpr int E = 16 / sizeof(T), KU = DKP / E, VU = DVP / E, MT = DVP / 32;
    u32x4 q[KU / 2];
    f32x16 o[MT];
    float m, l;
    // The row at `from`, nullptr: zeros.  All loads are under way before one is waited for, and only the unit that is a row's
    // last is moved down (code that runs once costs most by its length).
    template <bool VEC>
    __device__ __forceinline__ void load_q(const SoftArgs& A, const T* from, int h) {
        if (VEC || A.dk >= E) {
#pragma unroll
            for (int c = 0; c < KU / 2; ++c) {
                const int at = (2 * c + h) * E;
                const bool there = from && at < A.dk;
                const T* p = there ? from + (VEC ? at : min(at, A.dk - E)) : static_cast<const T*>(A.q);
                const u32x4 v = *reinterpret_cast<const u32x4_any*>(p);
                q[c] = there ? v : u32x4{0, 0, 0, 0};
            }
            const int past = A.dk % E;
            if (!VEC && past) {
                u32x4 v{0, 0, 0, 0};
#pragma unroll
                for (int c = 0; c < KU / 2; ++c) v = 2 * c + h == A.dk / E ? q[c] : v;
                v = moved_down(v, (E - past) * 8 * sizeof(T));
#pragma unroll
                for (int c = 0; c < KU / 2; ++c) q[c] = 2 * c + h == A.dk / E ? v : q[c];
            }
        } else {
#pragma unroll
            for (int c = 0; c < KU / 2; ++c) q[c] = u32x4{0, 0, 0, 0};
            if (from) q[0] = load_unit<T>(from, h, A.dk);
        }
        if (A.qsign != 1) turn_q(A.qsign);
    }
    uint32_t odd[MT / 2];  // of o: results that are NaN

    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[mt][i] = 0.0f;
        m = -FLT_MAX;
        l = 0.0f;
    }

    // Where this lane's operands lie in a tile of k and of v, in bytes.  The units of a row are permuted by an exclusive or with
    // a number of the row below 16 (k: 4), which is the same for all of the lane's rows (of bf16, and of k), so four (two)
    // addresses and constant distances are enough.
    using KT_ = KeyTile<KU>;
    using VT_ = ValueTile<VU>;
    uint32_t at_k[2], at_v[4];
    __device__ __forceinline__ void place() {
        const int l64 = threadIdx.x & 63, n = l64 & 31, h = l64 >> 5;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            if (x < 2) at_k[x] = KT_::at(n, 2 * x + h) * 16;
            if constexpr (sizeof(T) == 2) {  // column 32 x, rows 4 h + 0 .. 3 by the lane's place among 16
                const int col = (32 * x + 16 * (l64 >> 4 & 1) + 4 * (l64 & 3)) % DVP;
                at_v[x] = VT_::at(4 * h + (l64 & 15) / 4, col / 8) * 16 + (col & 4) * 2;
            } else {  // row 4 h + x, less x rows
                at_v[x] = (VT_::at(4 * h + x, n / 4) - x * VU) * 16 + (n & 3) * 4;
            }
        }
    }
    template <typename V>
    static __device__ __forceinline__ V read(uint32_t at) {
        return *(const __attribute__((address_space(3))) V*)(uintptr_t)at;
    }

    // Scores of 32 NB keys, over the first 2 C units of a row.
    template <int C, int NB>
    __device__ __forceinline__ void scores_over(uint32_t tile, f32x16 (&s)[NB]) const {
        constexpr int X = NB * C, D = 4;  // operands are read D products ahead
        uint32_t at[2] = {tile + at_k[0], tile + at_k[1]};
        asm volatile("" : "+v"(at[0]), "+v"(at[1]));  // (or each address is computed anew, where a constant offset does)
        auto operand = [&](int x) {
            return read<u32x4>(at[x % C & 1] + ((x % C >> 1) * 64 + x / C * (KT_::units(32) * 16)));
        };
        u32x4 k[D];
#pragma unroll
        for (int x = 0; x < D; ++x) k[x] = operand(x);
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[b][i] = 0.0f;
#pragma unroll
        for (int x = 0; x < X; ++x) {
            s[x / C] = SoftMath<T>::score(k[x % D], q[x % C], s[x / C]);
            if (x + D < X) k[x % D] = operand(x + D);
        }
        constexpr int PER = sizeof(T) == 2 ? 1 : 4;  // matrix instructions of a product
        __builtin_amdgcn_sched_group_barrier(kDsRead, D, 0);
#pragma unroll
        for (int x = 0; x < X; ++x) {
            __builtin_amdgcn_sched_group_barrier(kMfma, PER, 0);
            if (x + D < X) __builtin_amdgcn_sched_group_barrier(kDsRead, 1, 0);
        }
    }
    // fp32 products take long: a last quarter that is only padding is left out, of k here and of v below, where rows are few (32
    // single tokens of 80 over up to 8000 keys 161 -> 140 us; the prompt kernel has no registers for two ways: 82 -> 106).
    template <int NB>
    __device__ __forceinline__ void scores(uint32_t tile, f32x16 (&s)[NB], int dk) const {
        if (sizeof(T) == 4 && dk <= 3 * DKP / 4) scores_over<3 * KU / 8>(tile, s);
        else scores_over<KU / 2>(tile, s);
    }

    // v as an operand: of bf16 the 16 keys from `row` on, columns 32 mt ..; of fp32 the keys that weight i of p belongs to.
    struct ValuePlaces {
        uint32_t at[4];
    };
    __device__ __forceinline__ ValuePlaces places(uint32_t tile) const {
        ValuePlaces p;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            p.at[x] = tile + at_v[x];
            asm volatile("" : "+v"(p.at[x]));
        }
        return p;
    }
    static __device__ __forceinline__ u32x4 values(const ValuePlaces& p, int row, int mt) {
        u32x4 v;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const uint32_t at = p.at[mt & 3] + ((mt >> 2) * 256 + (row + 8 * x) * (VU * 16));
            const u32x2 w = __builtin_bit_cast(
                u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(uintptr_t)at));
            v[2 * x] = w[0];
            v[2 * x + 1] = w[1];
        }
        return v;
    }
    __device__ __forceinline__ float value(uint32_t tile, int i, int mt) const {
        // (column 32 mt is 8 mt units on, of which the row's number may turn bit 3)
        const uint32_t row = 32 * (i / 16) + 8 * (i % 16 / 4) + i % 4;
        return read<float>(tile + ((at_v[i & 3]) ^ ((mt & 1) * 128)) + (mt >> 1) * 256 + row * (VU * 16));
    }

    // Adds 32 NB keys, of which the first `left` count, with weights p (as scores() leaves them) in P parts.
    template <int P, int NB>
    __device__ __forceinline__ void add(uint32_t tile, const f32x16 (&p)[NB], int left, int dv) {
        if constexpr (sizeof(T) == 2) {
            constexpr int X = 2 * NB * MT, D = P > 1 ? 2 : 4;  // operands are read D ahead
            const ValuePlaces at = places(tile);
            u32x4 v[D];
            bf16x8 part[P];
#pragma unroll
            for (int x = 0; x < D; ++x) v[x] = values(at, 16 * (x / MT), x % MT);
#pragma unroll
            for (int x = 0; x < X; ++x) {
                const int c = x / MT, mt = x % MT;
                if (mt == 0) planes(p[c / 2], 8 * (c % 2), part);
#pragma unroll
                for (int i = 0; i < P; ++i)
                    o[mt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v[x % D]), part[i], o[mt], 0, 0, 0);
                if (x + D < X) v[x % D] = values(at, 16 * ((x + D) / MT), (x + D) % MT);
            }
        } else {
            if (MT % 4 == 0 && dv <= 24 * MT) add_over<MT % 4 == 0 ? 3 * MT / 4 : MT>(tile, p, left);
            else add_over<MT>(tile, p, left);
        }
    }
    template <int LIVE, int NB>
    __device__ __forceinline__ void add_over(uint32_t tile, const f32x16 (&p)[NB], int left) {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < 16 * NB; ++i)
#pragma unroll
                for (int mt = 0; mt < LIVE; ++mt)
                    if (i < 4 || 8 * (i / 4) < left)  // (8 keys at a time)
                        o[mt] = __builtin_amdgcn_mfma_f32_32x32x2f32(value(tile, i, mt), p[i / 16][i % 16], o[mt], 0, 0, 0);
        }
    }

    // 8 weights, from number `first` of p on, as bf16 parts, each the rounding of what the ones before left.
    template <int P>
    static __device__ __forceinline__ void planes(const f32x16& p, int first, bf16x8 (&part)[P]) {
        u32x4 w[P];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float a = p[first + 2 * j], b = p[first + 2 * j + 1];
#pragma unroll
            for (int i = 0; i < P; ++i) {
                const uint32_t both = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
                w[i][j] = both;
                a -= __builtin_bit_cast(float, both << 16);
                b -= __builtin_bit_cast(float, both & 0xffff0000u);
            }
        }
#pragma unroll
        for (int i = 0; i < P; ++i) part[i] = __builtin_bit_cast(bf16x8, w[i]);
    }

    // (o of a pass that counts holds numbers of values, which no maximum makes fewer.)
    __device__ __forceinline__ void rescale(float mx, bool counting) {
        const float now = fmaxf(m, mx);
        const float fade = __builtin_amdgcn_exp2f(m - now);
        m = now;
        l *= fade;
        if (counting) return;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[mt][i] *= fade;
    }

    // One tile of KT keys, of which lane i of s[b] is key key0 + 32 b + 8 (i / 4) + 4 h + i % 4, with weights in P parts.  One part (prompts
    // in bf16) goes by blocks of 32 keys, each with a maximum of its own and sums in follow()'s order, so that a row has the same
    // numbers here and in the two steps below.
    template <int KT, int P = PLANES>
    __device__ __forceinline__ void step(uint32_t tile_k, uint32_t tile_v, int key0, int left, bool masked, bool counting,
                                         const RowMask& mask, float scale2, int dk, int dv) {
        constexpr int NB = KT / 32, G = P > 1 ? NB : 1;
        const int h = threadIdx.x >> 5 & 1;
        f32x16 s[NB];
        scores(tile_k, s, dk);
        uint64_t seen = ~0ull;
        auto sees = [&](int b, int i) { return (uint32_t)(seen >> (32 * b)) >> (8 * (i / 4) + i % 4) & 1; };
        if (masked) {
            seen = mask.bits(key0) >> (4 * h);
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[b][i] = sees(b, i) ? s[b][i] : -INFINITY;
        }
#pragma unroll
        for (int g = 0; g < NB; g += G) {
            float mx = -INFINITY;
#pragma unroll
            for (int b = g; b < g + G; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[b][i]);
            mx = max_of_halves(mx) * scale2;
            // sums are relative to a maximum that may be up to kSlack behind: most tiles leave them as they are
            if (__any(mx > m + kSlack)) rescale(mx, counting);
            float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            f32x16 w[G];
#pragma unroll
            for (int b = 0; b < G; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    w[b][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[g + b][i], scale2, -m));
                    if constexpr (P > 1) sum[i & 3] += w[b][i];
                    else if (i & 1) sum[i / 2 & 1] += w[b][i - 1] + w[b][i];
                }
            l += P > 1 ? (sum[0] + sum[1]) + (sum[2] + sum[3]) : sum[0] + sum[1];
            if (counting) {
#pragma unroll
                for (int b = 0; b < G; ++b)
#pragma unroll
                    for (int i = 0; i < 16; ++i) w[b][i] = sees(g + b, i) ? 1.0f : 0.0f;
            }
            add<P>(tile_v + g * (32 * VU * 16), w, left - 32 * g, dv);
        }
    }

    // After a pass that counted: which results see a value that is not finite.
    __device__ __forceinline__ void counted() {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int i = 0; i < 16; ++i) odd[mt / 2] |= o[mt][i] > 0.0f ? 1u << (mt % 2 * 16 + i) : 0u;
    }
    __device__ __forceinline__ void mark() {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[mt][i] = odd[mt / 2] >> (mt % 2 * 16 + i) & 1 ? NAN : o[mt][i];
    }

    // The same in two steps, for blocks of 32 keys of bf16, so that each has matrix instructions of one block beside vector
    // instructions of another: `lead` adds the weights w of the block before and finds the maximum of this one's scores s (and
    // rescales), `follow` turns them into weights and computes the scores of the next one.  The compiler puts the two kinds
    // one after the other (8192 tokens, 16 heads of 128: 322 us, 315), so each matrix instruction is fenced off
    // with what is to run beside it.  Each step begins with operands that the one before has read (AHEAD).
    static constexpr int AHEAD = 4;
    struct KeyPlaces {
        uint32_t at[2];
    };
    __device__ __forceinline__ KeyPlaces key_places(uint32_t tile) const {
        KeyPlaces p{{tile + at_k[0], tile + at_k[1]}};
        asm volatile("" : "+v"(p.at[0]), "+v"(p.at[1]));  // (or each address is computed anew, where a constant offset does)
        return p;
    }
    static __device__ __forceinline__ u32x4 keys(const KeyPlaces& p, int x) { return read<u32x4>(p.at[x & 1] + (x >> 1) * 64); }
    static __device__ __forceinline__ u32x4 values_of(const ValuePlaces& p, int x) { return values(p, 16 * (x / MT), x % MT); }
    static __device__ __forceinline__ void fence() { __builtin_amdgcn_sched_barrier(0); }

    __device__ __forceinline__ void lead(const ValuePlaces& at, u32x4 (&v)[AHEAD], const u32x4 (&w)[2], f32x16& s, bool masked,
                                         bool counting, uint32_t seen, float scale2, const KeyPlaces& then, u32x4 (&k)[AHEAD]) {
        if (masked) {
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = seen >> (8 * (i / 4) + i % 4) & 1 ? s[i] : -INFINITY;
        }
        constexpr int X = 2 * MT;
        float mx = -INFINITY;
        __builtin_amdgcn_s_setprio(1);  // the other wave has vector instructions: 318 us, 313
        fence();
#pragma unroll
        for (int x = 0; x < X; ++x) {
            o[x % MT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v[x % AHEAD]),
                                                                __builtin_bit_cast(bf16x8, w[x / MT]), o[x % MT], 0, 0, 0);
            if (x + AHEAD < X) v[x % AHEAD] = values_of(at, x + AHEAD);
            else k[x + AHEAD - X] = keys(then, x + AHEAD - X);
#pragma unroll
            for (int i = 16 * x / X; i < 16 * (x + 1) / X; ++i) mx = fmaxf(mx, s[i]);
            fence();
        }
        __builtin_amdgcn_s_setprio(0);
        mx = max_of_halves(mx) * scale2;
        if (__any(mx > m + kSlack)) rescale(mx, counting);
    }
    template <bool MORE>  // the next step's first values can be read
    __device__ __forceinline__ void follow(const KeyPlaces& at, u32x4 (&k)[AHEAD], const f32x16& s, float scale2, f32x16& next,
                                           u32x4 (&w)[2], const ValuePlaces& then, u32x4 (&v)[AHEAD]) {
        constexpr int X = KU / 2;
        float p[16], sum[2] = {0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < 16; ++i) next[i] = 0.0f;
        fence();
#pragma unroll
        for (int x = 0; x < X; ++x) {
            next = SoftMath<T>::score(k[x % AHEAD], q[x], next);
            if (x + AHEAD < X) k[x % AHEAD] = keys(at, x + AHEAD);
            else if (MORE) v[x + AHEAD - X] = values_of(then, x + AHEAD - X);
#pragma unroll
            for (int i = 16 * x / X; i < 16 * (x + 1) / X; ++i) {
                p[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], scale2, -m));
                if (i & 1) {
                    w[i / 8][i % 8 / 2] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{p[i - 1], p[i]}, bf16x2));
                    asm volatile("" : "+v"(w[i / 8][i % 8 / 2]));
                    sum[i / 2 & 1] += p[i - 1] + p[i];
                }
            }
            fence();
        }
        l += sum[0] + sum[1];
    }
    __device__ __forceinline__ void first_scores(uint32_t tile_k, f32x16& s) const {
        f32x16 x[1];
        scores(tile_k, x, DKP);
        s = x[0];
    }
    __device__ __forceinline__ void last_product(uint32_t tile_v, const u32x4 (&w)[2]) {
        const ValuePlaces at = places(tile_v);
#pragma unroll
        for (int x = 0; x < 2 * MT; ++x)
            o[x % MT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, values(at, 16 * (x / MT), x % MT)),
                                                                __builtin_bit_cast(bf16x8, w[x / MT]), o[x % MT], 0, 0, 0);
    }
    // (A pass that counts has ones for what is seen in place of weights.)
    __device__ __forceinline__ void seen_weights(uint32_t seen, u32x4 (&w)[2]) const {
#pragma unroll
        for (int i = 0; i < 16; i += 2) {
            const uint32_t b = seen >> (8 * (i / 4) + i % 4) & 3;
            w[i / 8][i % 8 / 2] = (b & 1 ? 0x3f80u : 0u) | (b & 2 ? 0x3f800000u : 0u);
        }
    }

    __device__ __forceinline__ void turn_q(int sign) {
#pragma unroll
        for (int c = 0; c < KU / 2; ++c) q[c] = SoftMath<T>::sign(q[c], sign);
    }

    // Whether a value that is not finite came up (in any lane that has a row): what rows that do not see it hold has to be
    // computed again.  Lanes without one multiply zeros with every key, so an infinite one alone would spoil them.
    __device__ __forceinline__ bool spoilt(bool live) const {
        float bad[4] = {l * 0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int i = 0; i < 16; ++i) bad[i & 3] = __builtin_fmaf(o[mt][i], 0.0f, bad[i & 3]);
        return __any(live && !((bad[0] + bad[1]) + (bad[2] + bad[3]) == 0.0f));
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

// What a part leaves in the workspace: for each row of its tile the maximum and the sum of the weights, and the sums over v.
// Parts of a row may run on different XCDs, whose L2 caches are not coherent: where the same launch joins them
// (SAME), everything is stored and loaded past the caches (device scope).
// They lie row by row then; else as waves have them in registers, so that a store writes 1 KB in a row (16 requests of 24 drafts
// over up to 5000 keys 69 -> 58 us, 4 prompts of 300 to 700 that go on from 12000 214 -> 206).
template <bool SAME>
struct PartRows {
    static constexpr int kDevice = SAME ? 1 << 4 : 0;  // cache policy bit of buffer accesses
    __amdgpu_buffer_rsrc_t r;
    uint32_t step;  // bytes from a row to the next, of 32 rows to the next 32
    uint32_t sums_at;
    // A share has places for two parts: of a unit that began before it, and of one that begins in it (part 0).
    __device__ __forceinline__ PartRows(const SoftArgs& A, const SoftPlace& pl, uint32_t part) {
        const uint32_t rows = (uint32_t)A.tile * A.pack;
        step = SAME ? ((uint32_t)A.dv + 3) / 4 * 16 + 16 : ((uint32_t)A.dv + 7) / 8 * 1024;
        sums_at = SAME ? 0 : (rows + 31) / 32 * step;
        const uint32_t bytes = SAME ? rows * step : sums_at + (rows + 31) / 32 * 256;
        r = make_rsrc(static_cast<char*>(A.ws) + (int64_t)(2 * (pl.share + part) + (part == 0)) * bytes, bytes);
    }
    __device__ __forceinline__ uint32_t at(int row, int c) const {
        return SAME ? row * step + 16 + c * 4 : (row >> 5) * step + (c >> 3) * 1024 + (c >> 2 & 1) * 512 + (row & 31) * 16;
    }
    __device__ __forceinline__ uint32_t at_sums(int row) const { return SAME ? row * step : sums_at + row * 8; }
    __device__ __forceinline__ void put_sums(int row, f32x2 v) const {
        __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u32x2, v), r, at_sums(row), 0, kDevice);
    }
    __device__ __forceinline__ void put(int row, int c, f32x4 v) const {
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v), r, at(row, c), 0, kDevice);
    }
    __device__ __forceinline__ f32x2 sums(int row) const {
        return __builtin_bit_cast(f32x2, __builtin_amdgcn_raw_buffer_load_b64(r, at_sums(row), 0, kDevice));
    }
    __device__ __forceinline__ f32x4 get(int row, int c) const {
        return __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(r, at(row, c), 0, kDevice));
    }
};

// 4 columns of a row over some of its parts, in their order.
struct Joined {
    f32x4 o{0, 0, 0, 0};
    float m = -FLT_MAX, l = 0.0f;
    __device__ __forceinline__ void add(f32x4 v, f32x2 s) {
        const float now = fmaxf(m, s[0]), a = __builtin_amdgcn_exp2f(m - now), b = __builtin_amdgcn_exp2f(s[0] - now);
        m = now;
        l = l * a + s[1] * b;
        o = o * a + v * b;
    }
    // Parts [p, end), AHEAD of them at a time.
    template <int AHEAD, bool SAME>
    __device__ __forceinline__ void parts(const SoftArgs& A, const SoftPlace& pl, int row, int c, uint32_t p, uint32_t end) {
#pragma unroll 1
        for (; p < end; p += AHEAD) {
            f32x2 s[AHEAD];
            f32x4 v[AHEAD];
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                const PartRows<SAME> part(A, pl, min(p + i, pl.parts - 1));
                s[i] = part.sums(row);
                v[i] = part.get(row, c);
            }
#pragma unroll
            for (int i = 0; i < AHEAD; ++i)
                if (p + i < end) add(v[i], s[i]);
        }
    }
    template <typename T, bool VEC>
    __device__ __forceinline__ void store(const SoftArgs& A, const SoftPlace& pl, int row, int c) const {
        const float inv = l == 0.0f ? 0.0f : 1.0f / l;
        const int t = pl.t0 + (int)fdiv(row, A.by_pack), head = pl.head + row - (int)fdiv(row, A.by_pack) * A.pack;
        store4<T, VEC>(static_cast<T*>(A.o) + (pl.row0 + t) * A.o_row + (int64_t)head * A.o_head + c, A.dv - c, o * inv);
    }
};

// Few rows are joined by the workgroup whose part is done last, which clears their count for the next call.  The others return
// at once.  Threads that rows leave idle take some of the parts, and what they have is joined in order through `lds` (2 tokens over
// 65536 keys, 32 parts each: 67 -> 62 us).
template <typename T, bool VEC>
__device__ __forceinline__ void join_last(const SoftArgs& A, const SoftPlace& pl, int threads, u32x4* lds) {
    __shared__ int s_last;
    uint32_t* const count = static_cast<uint32_t*>(A.marks) + pl.share;  // only one unit begins in a share and goes on behind it
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // this thread's results are where all XCDs see them
    __syncthreads();
    if (threadIdx.x == 0)
        s_last = __hip_atomic_fetch_add(count, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == pl.parts - 1;
    __syncthreads();
    if (!s_last) return;
    const uint32_t groups = (A.dv + 3) / 4, all = min(A.tile, pl.len - pl.t0) * A.pack * groups;
    uint32_t slices = 1;
    while (2 * slices * all <= (uint32_t)threads && 8 * slices < pl.parts) slices *= 2;
    const uint32_t each = (pl.parts + slices - 1) / slices;
    auto* const s_o = reinterpret_cast<f32x4*>(lds);
    auto* const s_sums = reinterpret_cast<f32x2*>(lds + threads);
#pragma unroll 1
    for (uint32_t x = threadIdx.x; x < slices * all; x += threads) {
        uint32_t at = x;
        const uint32_t slice = slices == 1 ? 0 : quotient(x, all, &at);
        const int row = (int)fdiv(at, A.by_groups), c = 4 * (at - row * groups);
        Joined of;
        of.parts<8, true>(A, pl, row, c, slice * each, min((slice + 1) * each, pl.parts));
        if (slices == 1) {
            of.store<T, VEC>(A, pl, row, c);
        } else {
            s_o[x] = of.o;
            s_sums[x] = f32x2{of.m, of.l};
        }
    }
    if (slices > 1) {
        __syncthreads();
        if (threadIdx.x < all) {
            const int row = (int)fdiv(threadIdx.x, A.by_groups), c = 4 * (threadIdx.x - row * groups);
            Joined of;
            for (uint32_t i = threadIdx.x; i < slices * all; i += all) of.add(s_o[i], s_sums[i]);
            of.store<T, VEC>(A, pl, row, c);
        }
    }
    if (threadIdx.x == 0) __hip_atomic_store(count, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Values that are not finite would reach rows that do not see them, as a product with zero.  Where a pass over the keys comes
// upon one (in the result, at no cost while there is none), two more passes follow: one counts, for each result, the
// values of that kind that its row sees, and one leaves them out.  For them the values in LDS are replaced: 16 bytes by
// ones where they are not finite and zeros else (COUNT), or by themselves with zeros there.
enum { PLAIN = 0, COUNT = 1, CLEAN = 2 };
template <typename T>
__device__ __forceinline__ u32x4 only_finite(u32x4 v, bool count) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 2) {
            const bool a = (v[i] & 0x7f80u) == 0x7f80u, b = (v[i] & 0x7f800000u) == 0x7f800000u;
            v[i] = count ? (a ? 0x3f80u : 0u) | (b ? 0x3f800000u : 0u) : v[i] & ((a ? 0u : 0xffffu) | (b ? 0u : 0xffff0000u));
        } else {
            const bool a = (v[i] & 0x7f800000u) == 0x7f800000u;
            v[i] = count ? (a ? 0x3f800000u : 0u) : a ? 0u : v[i];
        }
    }
    return v;
}
template <typename T>
__device__ __forceinline__ void clean_tile(u32x4* v, int units, int from, int step, int mode) {
#pragma unroll 1
    for (int x = from; x < units; x += step) v[x] = only_finite<T>(v[x], mode == COUNT);
}

// A wave's 64 units of 16 bytes go from memory to LDS, from byte `to` + MORE on, without passing registers.  The compiler does not count
// these loads: loads_done() waits for them.  Nor does it see that they read r and m0: a scalar instruction that writes m0 has to
// be 1 wait state before, a vector one that writes a part of r (a lane's value read, also by the compiler where it kept r in lanes) 5.
// FIRST: of those with this r.  The others follow the first at once, and a test holds the built code to it (waiting 5 states at each
// takes 2 % of prompts' time).
template <bool FIRST, int MORE>
__device__ __forceinline__ void load_to_lds(u32x4 r, uint32_t off, uint32_t to) {
    asm volatile("s_add_i32 m0, %0, %3\n\ts_nop %4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to), "v"(off), "s"(r), "n"(MORE),
                 "n"(FIRST ? 3 : 0)
                 : "memory", "scc", "m0");
}
template <int N, typename F>
__device__ __forceinline__ void each_of(F f) {  // f(0) .. f(N - 1), as constants
    if constexpr (N > 0) {
        each_of<N - 1>(f);
        f(std::integral_constant<int, N - 1>{});
    }
}
// ... 64 elements of 4 bytes.
__device__ __forceinline__ void load_words_to_lds(__amdgpu_buffer_rsrc_t r, uint32_t off, uint32_t to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(to), "v"(off), "s"(r) : "memory", "m0");
}
typedef __attribute__((address_space(3))) const void* lds_address;
__device__ __forceinline__ void loads_done() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// The page that holds the rows of lane i's instruction.
__device__ __forceinline__ int clamp_page(const SoftArgs& A, int page) { return min(max(page, 0), (int)A.pages - 1); }

// Loads the rows of tiles of keys (or values) into LDS, RI rows per instruction of a wave.  What lies past the last key or past a
// row's end reads as zero by the buffer's range.  Where a page (of packed rows: some rows that a 32-bit offset
// reaches) begins, and how much of it counts, is worked out for all instructions of a tile at once, a lane each.
template <typename T, int UNITS, int KT, int WAVES, typename LDS>
struct DirectLoad {
    static constexpr int E = 16 / sizeof(T), RI = 64 / UNITS, N = KT / RI / WAVES;
    static constexpr int KINDS = RI * WAVES < 8 ? 8 / (RI * WAVES) : 1;  // rows of instructions i and i + KINDS have one order
    uint64_t base;
    uint32_t off[KINDS];  // of this lane, in bytes
    uint32_t page_bytes, row_bytes, last;  // last: bytes of a row that count
    int wave;             // (0: each wave loads its own tiles)

    __device__ __forceinline__ DirectLoad(const SoftArgs& A, const SoftPlace& pl, const void* p, const CachePlace& c, int dim) {
        const int lane = threadIdx.x & 63, r = lane / UNITS, at = lane % UNITS;
        base = reinterpret_cast<uint64_t>(static_cast<const T*>(p) + pl.kv_head * c.head + pl.key0 * c.row);
        page_bytes = (uint32_t)c.page * sizeof(T);
        row_bytes = (uint32_t)c.row * sizeof(T);
        last = dim * sizeof(T);
        wave = WAVES > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0;
#pragma unroll
        for (int i = 0; i < KINDS; ++i) {
            const int row = first_row(i) + r;
            const int u = at ^ LDS::turn(row);
            off[i] = u * E < dim ? r * row_bytes + min(u * 16u, last - 16) : OOB_OFF;
        }
    }
    // WAVES waves load a tile together, or each its own (1).
    __device__ __forceinline__ int first_row(int i) const { return (WAVES * i + wave) * RI; }
    // `page` of lane i: of instruction i's rows.  What an instruction's buffer is comes from its lane, or from lane 0 for
    // all where the tile lies in one page (tiles begin at multiples of KT).
    __device__ __forceinline__ void tile(const SoftArgs& A, const SoftPlace& pl, int key0, int page, uint32_t to) const {
        constexpr int LINE = LDS::GROUP * 16;
        auto get = [&](uint32_t v, int i) { return (uint32_t)__builtin_amdgcn_readlane((int)v, i); };
        to += wave * LINE;
        if ((1 << A.shift) >= KT) {
            const uint32_t key = (uint32_t)(key0 + wave * RI), at = A.table ? get((uint32_t)page, 0) : key >> A.shift;
            const uint64_t p = base + (uint64_t)at * page_bytes + (uint64_t)(key & ((1u << A.shift) - 1)) * row_bytes;
            const int left = pl.keys - (int)key;
            const uint32_t rows = left < KT ? left : KT, each = WAVES * RI * row_bytes;
            const uint32_t bytes = left > 0 ? (rows - 1) * row_bytes + last : 0u;
            const u32x4 r{(uint32_t)p, (uint32_t)(p >> 32), bytes, RSRC_WORD3};
            each_of<N>([&](auto i) { load_to_lds<i == 0, i * WAVES * LINE>(r, off[i % KINDS] + i * each, to); });
        } else {
            const int key = key0 + first_row(threadIdx.x & 63);
            const uint64_t p = base + (uint64_t)(uint32_t)page * page_bytes +
                               (uint64_t)(uint32_t)(key & ((1 << A.shift) - 1)) * row_bytes;
            const int rows = min(max(pl.keys - key, 0), RI);
            const uint32_t bytes = rows ? (rows - 1) * row_bytes + last : 0u;
            each_of<N>([&](auto i) {
                load_to_lds<true, i * WAVES * LINE>(u32x4{get((uint32_t)p, i), get((uint32_t)(p >> 32), i), get(bytes, i), RSRC_WORD3},
                                                    off[i % KINDS], to);
            });
        }
    }
    // Rows of any alignment and size (16 bytes at least): into registers, with the scalar work of `tile` and no more (each
    // address by itself, in 64 bits, and pages by lanes: 64 single tokens of 127 over up to 8000 keys 323 us, so 198;
    // 2048 tokens 152 and 127),
    __device__ __forceinline__ void fetch(const SoftArgs& A, const SoftPlace& pl, int key0, int page, u32x4 (&v)[N]) const {
        auto get = [&](uint32_t x, int i) { return (uint32_t)__builtin_amdgcn_readlane((int)x, i); };
        auto load = [&](uint64_t p, uint32_t bytes, uint32_t o) {
            return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(make_rsrc((const void*)p, bytes), o, 0, 0));
        };
        if ((1 << A.shift) >= KT) {
            const uint32_t key = (uint32_t)(key0 + wave * RI), at = A.table ? get((uint32_t)page, 0) : key >> A.shift;
            const uint64_t p = base + (uint64_t)at * page_bytes + (uint64_t)(key & ((1u << A.shift) - 1)) * row_bytes;
            const int left = pl.keys - (int)key;
            const uint32_t rows = left < KT ? left : KT, each = WAVES * RI * row_bytes;
            const uint32_t bytes = left > 0 ? (rows - 1) * row_bytes + last : 0u;
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = load(p, bytes, off[i % KINDS] + i * each);
        } else {
            const int key = key0 + first_row(threadIdx.x & 63);
            const uint64_t p = base + (uint64_t)(uint32_t)page * page_bytes +
                               (uint64_t)(uint32_t)(key & ((1 << A.shift) - 1)) * row_bytes;
            const int rows = min(max(pl.keys - key, 0), RI);
            const uint32_t bytes = rows ? (rows - 1) * row_bytes + last : 0u;
#pragma unroll
            for (int i = 0; i < N; ++i)
                v[i] = load((uint64_t)get((uint32_t)(p >> 32), i) << 32 | get((uint32_t)p, i), get(bytes, i), off[i % KINDS]);
        }
    }
    // ... and on to LDS, where the last part of a row, which was read where it ends with the row, is moved down.
    __device__ __forceinline__ void store(const u32x4 (&v)[N], u32x4* to) const {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int i = 0; i < N; ++i) to[(i * WAVES + wave) * LDS::GROUP + lane] = v[i];
        if (last & 15) {
            static_assert(RI * N <= 64);
            if (lane < RI * N) {
                u32x4& end = to[LDS::at(first_row(lane / RI) + lane % RI, (int)(last / 16))];
                end = moved_down(end, (16 - (last & 15)) * 8);
            }
        }
    }
    // The page of instruction `lane`'s rows of the tile from key0 on.
    __device__ __forceinline__ int look(const SoftArgs& A, const SoftPlace& pl, int key0) const {
        const int lane = threadIdx.x & 63, key = key0 + first_row(lane);
        return A.table && lane < N && key < pl.keys ? A.table[pl.slot * A.max_pages + (key >> A.shift)] : 0;
    }
};
// ... rows that lie otherwise: through registers, N units of each thread at a time.
template <typename T, int UNITS, int N, int THREADS, typename LDS>
struct RegisterLoad {
    u32x4 v[N];
    __device__ __forceinline__ void fetch(const SoftArgs& A, const SoftPlace& pl, const void* p, const CachePlace& c, int dim, int key0,
                                          int x0) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int x = x0 + i * THREADS, r = x / UNITS, u = x % UNITS;
            const int64_t from = key_row(A, pl, c, min(key0 + r, pl.keys - 1));
            v[i] = load_unit<T>(static_cast<const T*>(p) + from, u, dim);
        }
    }
    __device__ __forceinline__ void store(u32x4* to, int x0) const {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int x = x0 + i * THREADS;
            to[LDS::at(x / UNITS, x % UNITS)] = v[i];
        }
    }
};
// A whole tile of ROWS rows so: as many units in flight as divide it, four at most.
template <typename T, int UNITS, int ROWS, int THREADS, typename LDS>
__device__ __forceinline__ void copy_rows(const SoftArgs& A, const SoftPlace& pl, const void* p, const CachePlace& c, int dim, int key0,
                                          u32x4* to, int thread) {
    constexpr int EACH = ROWS * UNITS / THREADS, N = EACH % 4 == 0 ? 4 : EACH % 3 == 0 ? 3 : EACH % 2 == 0 ? 2 : 1;
    static_assert(EACH * THREADS == ROWS * UNITS);
#pragma unroll 1
    for (int x = thread; x < ROWS * UNITS; x += N * THREADS) {
        RegisterLoad<T, UNITS, N, THREADS, LDS> l;
        l.fetch(A, pl, p, c, dim, key0, x);
        l.store(to, x);
    }
}
constexpr int kPromptWaves = kPromptRows / 32;

// One part of a unit.
template <typename T, int DKP, int DVP, int KT, bool VEC>
__device__ __forceinline__ void prompt_part(const SoftArgs& A, const SoftPlace& pl, u32x4* lds) {
    using R = SoftRows<T, DKP, DVP>;
    constexpr int KU = R::KU, VU = R::VU, KEYS = KeyTile<KU>::units(KT);
    u32x4 *const sK = lds, *const sV = lds + (VEC ? 2 : 1) * KEYS;
    const int tid = threadIdx.x, wave = tid >> 6, n = tid & 31, h = tid >> 5 & 1;
    // this lane's row, and the rows of its wave and of the workgroup
    const int row = 32 * wave + n;
    const int t = pl.t0 + (int)fdiv(row, A.by_pack), head = pl.head + row - (int)fdiv(row, A.by_pack) * A.pack;
    const bool live = row < A.tile * A.pack && t < pl.len;
    const RowMask mask = row_mask(A, pl, live ? t : -1);
    const bool causal = A.mask == SEQMIX_MASK_CAUSAL, tree = A.mask == SEQMIX_MASK_TREE;
    const int back = pl.keys - pl.len;
    auto behind = [&](int tt) { return causal ? min(max(back + min(tt, pl.len - 1) + 1, 0), pl.keys) : pl.keys; };
    const int end = min(behind(pl.t0 + A.tile - 1), pl.last);
    const int w0 = pl.t0 + (int)fdiv(32 * wave, A.by_pack);
    const int wave_end = w0 < pl.len ? behind(pl.t0 + (int)fdiv(32 * wave + 31, A.by_pack)) : 0;
    const int wave_full = tree ? max(back, 0) : behind(w0);

    R rows;
#pragma unroll
    for (int i = 0; i < R::MT / 2; ++i) rows.odd[i] = 0;
    rows.place();
    rows.template load_q<VEC>(A, live ? static_cast<const T*>(A.q) + (pl.row0 + t) * A.q_row + (int64_t)head * A.q_head : nullptr, h);

    const uint32_t at_k = (uint32_t)(uintptr_t)(lds_address)sK, at_v = (uint32_t)(uintptr_t)(lds_address)sV;
#pragma unroll 1
    for (int mode = PLAIN;; ++mode) {
        auto step = [&](int b, int key0) {
            if (mode) {
                clean_tile<T>(sV + b * KT * VU, KT * VU, tid, 64 * kPromptWaves, mode);
                __syncthreads();
            }
            if (key0 < wave_end)
                rows.template step<KT, sizeof(T) == 2 ? 1 : PLANES>(at_k + b * (KEYS * 16), at_v + b * (KT * VU * 16), key0, end - key0,
                                                                    key0 + KT > wave_full, mode == COUNT, mask, A.scale2, DKP, DVP);
        };
        rows.clear();
        if constexpr (VEC) {
            constexpr bool PIPED = sizeof(T) == 2;
            DirectLoad<T, KU, KT, kPromptWaves, KeyTile<KU>> load_k(A, pl, A.k, A.kp, A.dk);
            DirectLoad<T, VU, KT, kPromptWaves, ValueTile<VU>> load_v(A, pl, A.v, A.vp, A.dv);
            auto look = [&](const auto& load, int j) {  // the pages of tile j
                const int lane = tid & 63, key = pl.first + j * KT + load.first_row(lane);
                return A.table && lane < load.N && key < pl.keys ? A.table[pl.slot * A.max_pages + (key >> A.shift)] : 0;
            };
            if constexpr (PIPED) {
                // Scores run a block ahead, products with v a block behind.  After the first block of tile j the values of tile
                // j - 1 have been used (and the keys of j - 1 long since), and after the last the keys of j + 1 are
                // needed: between the two, k of j + 1 and v of j have to be there, and the loads of k of j + 2 and of v of
                // j + 1 start, with the time of a whole tile to arrive.
                const int tiles = (end - pl.first + KT - 1) / KT;
                constexpr int NB = KT / 32;
                f32x16 s[2];
                u32x4 w[2] = {u32x4{0, 0, 0, 0}, u32x4{0, 0, 0, 0}};
                auto clean = [&](int j) {
                    if (mode) {
                        clean_tile<T>(sV + (j & 1) * KT * VU, KT * VU, tid, 64 * kPromptWaves, mode);
                        __syncthreads();
                    }
                };
                u32x4 first_k[R::AHEAD], first_v[R::AHEAD];
                auto keys_at = [&](int j, int b) { return rows.key_places(at_k + (j & 1) * (KEYS * 16) + b * (KEYS / NB * 16)); };
                auto values_at = [&](int j, int b) { return rows.places(at_v + (j & 1) * (KT * VU * 16) + b * (32 * VU * 16)); };
                auto read_values = [&](const typename R::ValuePlaces& p) {
#pragma unroll
                    for (int x = 0; x < R::AHEAD; ++x) first_v[x] = R::values_of(p, x);
                };
                auto seen_of = [&](int key0) { return (uint32_t)(mask.bits(key0) >> (4 * h)); };
                auto load_keys = [&](int j, int page) {
                    if (j < tiles) load_k.tile(A, pl, pl.first + j * KT, clamp_page(A, page), at_k + (j & 1) * (KEYS * 16));
                };
                auto load_values = [&](int j, int page) {
                    if (j < tiles) load_v.tile(A, pl, pl.first + j * KT, clamp_page(A, page), at_v + (j & 1) * (KT * VU * 16));
                };
                if (tiles > 0) {
                    int page_k = 0, page_v = 0;
                    if (A.table) {
                        const int page_0 = look(load_k, 0), page_1 = look(load_k, 1), page = look(load_v, 0);
                        page_k = look(load_k, 2), page_v = look(load_v, 1);
                        load_keys(0, page_0);
                        load_values(0, page);
                        load_keys(1, page_1);
                    } else {
                        load_keys(0, 0);
                        load_values(0, 0);
                        load_keys(1, 0);
                    }
                    loads_done();
                    __syncthreads();
                    clean(0);
                    rows.first_scores(at_k, s[0]);
                    typename R::ValuePlaces vp = values_at(0, 0);  // (at first some values with weights of zero)
                    read_values(vp);
#pragma unroll 1
                    for (int j = 0; j < tiles; ++j) {
                        const int key0 = pl.first + j * KT;
#pragma unroll
                        for (int b = 0; b < NB; ++b) {
                            const bool masked = key0 + 32 * b + 32 > wave_full;
                            const uint32_t seen = masked || mode == COUNT ? seen_of(key0 + 32 * b) : 0;
                            // (at last some scores that are not used)
                            const auto kp = b + 1 < NB ? keys_at(j, b + 1) : keys_at(j + 1, 0);
                            rows.lead(vp, first_v, w, s[b & 1], masked, mode == COUNT, seen, A.scale2, kp, first_k);
                            if (b == 0) {
                                rows.template follow<false>(kp, first_k, s[0], A.scale2, s[1], w, vp, first_v);
                            } else {
                                vp = values_at(j, b);
                                rows.template follow<true>(kp, first_k, s[b & 1], A.scale2, s[b + 1 & 1], w, vp, first_v);
                            }
                            if (mode == COUNT) rows.seen_weights(seen, w);
                            if (b == 0) {
                                loads_done();
                                __syncthreads();
                                if (j) clean(j);
                                vp = values_at(j, 0);
                                read_values(vp);
                                load_keys(j + 2, page_k);
                                load_values(j + 1, page_v);
                                if (A.table) page_k = look(load_k, j + 3), page_v = look(load_v, j + 2);
                            }
                        }
                    }
                    rows.last_product(at_v + ((tiles - 1) & 1) * (KT * VU * 16) + (KT - 32) * VU * 16, w);
                }
                loads_done();
            } else {
                auto load = [&](int j) {
                    load_k.tile(A, pl, pl.first + j * KT, clamp_page(A, look(load_k, j)), at_k + (j & 1) * (KEYS * 16));
                    load_v.tile(A, pl, pl.first + j * KT, clamp_page(A, look(load_v, j)), at_v + (j & 1) * (KT * VU * 16));
                };
                if (pl.first < end) load(0);
                for (int j = 0, key0 = pl.first; key0 < end; ++j, key0 += KT) {
                    loads_done();
                    __syncthreads();  // this tile is there, and the one before has been used
                    if (key0 + KT < end) load(j + 1);
                    step(j & 1, key0);
                }
            }
            __syncthreads();
        } else {
            constexpr int THREADS = 64 * kPromptWaves;
            const SoftArgs L = A;  // (what the loops need, read once)
            const DirectLoad<T, KU, KT, kPromptWaves, KeyTile<KU>> load_k(L, pl, L.k, L.kp, L.dk);
            const DirectLoad<T, VU, KT, kPromptWaves, ValueTile<VU>> load_v(L, pl, L.v, L.vp, L.dv);
            u32x4 k[load_k.N], v[load_v.N];
            int page_k = 0, page_v = 0;
            auto look = [&](int key0) { page_k = load_k.look(L, pl, key0), page_v = load_v.look(L, pl, key0); };
            if (!L.near) {
                for (int key0 = pl.first; key0 < end; key0 += KT) {
                    __syncthreads();
                    copy_rows<T, KU, KT, THREADS, KeyTile<KU>>(L, pl, L.k, L.kp, L.dk, key0, sK, tid);
                    copy_rows<T, VU, KT, THREADS, ValueTile<VU>>(L, pl, L.v, L.vp, L.dv, key0, sV, tid);
                    __syncthreads();
                    step(0, key0);
                }
            } else if constexpr (sizeof(T) == 2 && DKP + DVP <= 256) {
                // the next tile's while this one is used (wider rows and fp32 have no registers for it)
                auto fetch = [&](int key0) {
                    load_k.fetch(L, pl, key0, clamp_page(L, page_k), k);
                    load_v.fetch(L, pl, key0, clamp_page(L, page_v), v);
                    look(key0 + KT);
                };
                look(pl.first);
                if (pl.first < end) fetch(pl.first);
                for (int key0 = pl.first; key0 < end; key0 += KT) {
                    __syncthreads();
                    load_k.store(k, sK);
                    load_v.store(v, sV);
                    __syncthreads();
                    if (key0 + KT < end) fetch(key0 + KT);
                    step(0, key0);
                }
            } else {
                look(pl.first);
                for (int key0 = pl.first; key0 < end; key0 += KT) {
                    load_k.fetch(L, pl, key0, clamp_page(L, page_k), k);
                    __syncthreads();
                    load_k.store(k, sK);
                    load_v.fetch(L, pl, key0, clamp_page(L, page_v), v);
                    look(key0 + KT);
                    load_v.store(v, sV);
                    __syncthreads();
                    step(0, key0);
                }
            }
        }
        if (mode == COUNT) rows.counted();
        if (mode == CLEAN) {
            rows.mark();
            break;
        }
        if (mode == PLAIN) {
            __shared__ int s_again;
            if (tid == 0) s_again = 0;
            __syncthreads();
            if (rows.spoilt(live)) s_again = 1;
            __syncthreads();
            if (!s_again) break;
        }
    }

    const SoftArgs& E = args_here();
    const float l = sum_of_halves(rows.l);
    if (pl.parts == 1) {
        const float inv = l == 0.0f ? 0.0f : 1.0f / l;
        if (!live) return;
        T* o = static_cast<T*>(E.o) + (pl.row0 + t) * E.o_row + (int64_t)head * E.o_head;
#pragma unroll
        for (int mt = 0; mt < R::MT; ++mt)
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const int c = 32 * mt + 8 * b + 4 * h;
                const f32x4 v{rows.o[mt][4 * b], rows.o[mt][4 * b + 1], rows.o[mt][4 * b + 2], rows.o[mt][4 * b + 3]};
                store4<T, VEC>(o + c, E.dv - c, v * inv);
            }
        return;
    }
    const PartRows<false> part(E, pl, pl.part);
    if (live) {
        part.put_sums(row, f32x2{rows.m, l});
#pragma unroll
        for (int mt = 0; mt < R::MT; ++mt)
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const int c = 32 * mt + 8 * b + 4 * h;
                if (c < E.dv)
                    part.put(row, c, f32x4{rows.o[mt][4 * b], rows.o[mt][4 * b + 1], rows.o[mt][4 * b + 2], rows.o[mt][4 * b + 3]});
            }
    }
}

template <typename T, int DKP, int DVP, int KT, bool VEC>
__global__ __launch_bounds__(64 * kPromptWaves, DKP + DVP <= 256 ? 2 : 1) void softmax_prompt_kernel(SoftArgs) {
    using R = SoftRows<T, DKP, DVP>;
    __shared__ u32x4 lds[(VEC ? 2 : 1) * (KeyTile<R::KU>::units(KT) + KT * R::VU)];
    SoftPlace pl;
    SoftShares shares(args_here());
    while (shares.next(args_here(), &pl)) {
        pl.uniform();
        prompt_part<T, DKP, DVP, KT, VEC>(args_here(), pl, lds);
        __syncthreads();
    }
    const SoftArgs& A = args_here();
    // for the launch that joins: the unit that begins in this share and goes on behind it
    if (A.shares && threadIdx.x == 0) {
        if (shares.none || pl.part != 0) pl.parts = 1;
        static_assert(sizeof(SoftPlace) <= kMarkBytes && alignof(SoftPlace) <= 8);
        static_cast<SoftPlace*>(A.marks)[shares.share] = pl;
    }
}

// Many rows are joined by a launch of their own: blockIdx.x is a share, in which one unit at most begins and goes on behind it;
// each blockIdx.y takes kJoinRows of its rows, neighbouring threads neighbouring ones.  Two parts at a time (4 prompts of 300 to
// 700 that go on from 12000 194 us, with eight 202: most units have two or three parts).
constexpr int kJoinRows = 8;
template <typename T, bool VEC>
__global__ __launch_bounds__(256) void softmax_join_kernel(SoftArgs A) {
    SoftPlace pl = static_cast<const SoftPlace*>(A.marks)[blockIdx.x];
    pl.uniform();
    if (pl.parts == 1) return;
    const int rows = min(A.tile, pl.len - pl.t0) * A.pack;
#pragma unroll 1
    for (int x = threadIdx.x; x < kJoinRows * ((A.dv + 3) / 4); x += 256) {
        const int row = blockIdx.y * kJoinRows + x % kJoinRows, c = 4 * (x / kJoinRows);
        if (row >= rows) return;
        Joined of;
        of.parts<2, false>(A, pl, row, c, 0, pl.parts);
        of.store<T, VEC>(A, pl, row, c);
    }
}

// Few rows: each wave takes every WAVES-th 32 keys of the unit's, for the same rows, through LDS of its own, so that
// waves do not wait for each other until the end.  Two waves on a SIMD with a tile each: while one works the other's
// comes (eight waves with a tile each, not four with two: 64 tokens over up to 8000 keys 115 -> 110 us, 4 over up to 600
// 15.7 -> 12.5).
template <int BYTES>  // of 32 keys and values
constexpr int step_waves() { return BYTES <= 16384 ? 8 : BYTES <= 32768 ? 4 : 2; }

template <typename T, int DKP, int DVP>
struct StepTiles {
    static constexpr int KT = 32, E = 16 / sizeof(T), KEYS = KeyTile<DKP / E>::units(KT), TILE = KEYS + KT * DVP / E;
    static constexpr int WAVES = step_waves<KT * (DKP + DVP) * sizeof(T)>();
    static constexpr int PITCH = DVP + 4;  // of a row of results in LDS, in floats
    static constexpr int LDS = WAVES * (TILE > 8 * PITCH ? TILE : 8 * PITCH);
};

template <typename T, int DKP, int DVP, bool VEC>
__device__ __forceinline__ void step_part(const SoftArgs& A, const SoftPlace& pl, u32x4* lds, f32x2 (*s_sums)[32],
                                          int (*s_pages)[64]) {
    using R = SoftRows<T, DKP, DVP>;
    using S = StepTiles<T, DKP, DVP>;
    constexpr int KU = R::KU, VU = R::VU, KT = S::KT, KEYS = S::KEYS, TILE = S::TILE, WAVES = S::WAVES;
    constexpr int PITCH = S::PITCH;
    const int tid = threadIdx.x, n = tid & 31, h = tid >> 5 & 1;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int t = pl.t0 + (int)fdiv(n, A.by_pack), head = pl.head + n - (int)fdiv(n, A.by_pack) * A.pack;
    const bool live = n < A.tile * A.pack && t < pl.len;
    const RowMask mask = row_mask(A, pl, live ? t : -1);
    const bool causal = A.mask == SEQMIX_MASK_CAUSAL, tree = A.mask == SEQMIX_MASK_TREE;
    const int back = pl.keys - pl.len;
    auto behind = [&](int tt) { return causal ? min(max(back + min(tt, pl.len - 1) + 1, 0), pl.keys) : pl.keys; };
    const int end = min(behind(pl.t0 + A.tile - 1), pl.last);
    const int full = tree ? max(back, 0) : behind(pl.t0);

    u32x4* const mine = lds + wave * TILE;
    const uint32_t to = (uint32_t)(uintptr_t)(lds_address)lds + wave * (TILE * 16);
    const int first = pl.first + wave * KT;
    constexpr int STRIDE = WAVES * KT;
    // The pages of a tile's rows go through LDS too: a load to a register would be waited for together with all before it.
    const __amdgpu_buffer_rsrc_t table =
        make_rsrc(A.table ? A.table + pl.slot * A.max_pages : nullptr, A.table ? (uint32_t)A.max_pages * 4 : 0u);
    const int lane = tid & 63;
    const uint32_t to_pages = (uint32_t)(uintptr_t)(lds_address)&s_pages[wave][0];
    auto look = [&](int key0) {
        if (A.table) load_words_to_lds(table, (uint32_t)((key0 + lane) >> A.shift) * 4u, to_pages);
    };
    if constexpr (VEC) look(first);
    R rows;
#pragma unroll
    for (int i = 0; i < R::MT / 2; ++i) rows.odd[i] = 0;
    rows.place();
    rows.template load_q<VEC>(A, live ? static_cast<const T*>(A.q) + (pl.row0 + t) * A.q_row + (int64_t)head * A.q_head : nullptr, h);
#pragma unroll 1
    for (int mode = PLAIN;; ++mode) {
        auto step = [&](int key0) {
            if (mode) {
                clean_tile<T>(mine + KEYS, KT * VU, tid & 63, 64, mode);
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            }
            rows.template step<KT>(to, to + KEYS * 16, key0, end - key0, key0 + KT > full, mode == COUNT, mask, A.scale2, A.dk, A.dv);
        };
        rows.clear();
        if constexpr (VEC) {
            DirectLoad<T, KU, KT, 1, KeyTile<KU>> load_k(A, pl, A.k, A.kp, A.dk);
            DirectLoad<T, VU, KT, 1, ValueTile<VU>> load_v(A, pl, A.v, A.vp, A.dv);
            auto load = [&](int key0) {
                const int k = load_k.first_row(lane), v = load_v.first_row(lane);
                int page_k = 0, page_v = 0;
                if (A.table) {
                    page_k = clamp_page(A, s_pages[wave][k & 63]);
                    page_v = KU == VU ? page_k : clamp_page(A, s_pages[wave][v & 63]);
                    asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(page_k), "+v"(page_v)::"memory");  // read before the next ones come
                }
                load_k.tile(A, pl, key0, page_k, to);
                load_v.tile(A, pl, key0, page_v, to + KEYS * 16);
                look(key0 + STRIDE);
            };
            // a wave's tile comes while the other waves work; with it the pages of its next one
            if (mode) look(first);
            loads_done();
            if (first < end) load(first);
            for (int key0 = first; key0 < end; key0 += STRIDE) {
                loads_done();
                step(key0);
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the tile has been read
                if (key0 + STRIDE < end) load(key0 + STRIDE);
            }
            loads_done();
        } else {
            const SoftArgs L = A;  // (what the loops need, read once)
            const DirectLoad<T, KU, KT, 1, KeyTile<KU>> load_k(L, pl, L.k, L.kp, L.dk);
            const DirectLoad<T, VU, KT, 1, ValueTile<VU>> load_v(L, pl, L.v, L.vp, L.dv);
            u32x4 k[load_k.N], v[load_v.N];
            int page_k = 0, page_v = 0;
            auto look = [&](int key0) { page_k = load_k.look(L, pl, key0), page_v = load_v.look(L, pl, key0); };
            look(first);
            for (int key0 = first; key0 < end; key0 += STRIDE) {
                if (!L.near) {
                    copy_rows<T, KU, KT, 64, KeyTile<KU>>(L, pl, L.k, L.kp, L.dk, key0, mine, lane);
                    copy_rows<T, VU, KT, 64, ValueTile<VU>>(L, pl, L.v, L.vp, L.dv, key0, mine + KEYS, lane);
                } else {
                    load_k.fetch(L, pl, key0, clamp_page(L, page_k), k);
                    if (load_k.N > 8) load_k.store(k, mine);
                    load_v.fetch(L, pl, key0, clamp_page(L, page_v), v);
                    look(key0 + STRIDE);
                    if (load_k.N <= 8) load_k.store(k, mine);
                    load_v.store(v, mine + KEYS);
                }
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                step(key0);
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            }
        }
        if (mode == COUNT) rows.counted();
        if (mode == CLEAN) {
            rows.mark();
            break;
        }
        if (mode == PLAIN && !rows.spoilt(live)) break;
    }

    // the waves' results, in their order
    const SoftArgs& E = args_here();
    __syncthreads();
    float* const sO = reinterpret_cast<float*>(lds);
    const float l = sum_of_halves(rows.l);
    if (h == 0) s_sums[wave][n] = f32x2{rows.m, l};
#pragma unroll
    for (int mt = 0; mt < R::MT; ++mt)
#pragma unroll
        for (int b = 0; b < 4; ++b)
            *reinterpret_cast<f32x4*>(&sO[(wave * 32 + n) * PITCH + 32 * mt + 8 * b + 4 * h]) =
                f32x4{rows.o[mt][4 * b], rows.o[mt][4 * b + 1], rows.o[mt][4 * b + 2], rows.o[mt][4 * b + 3]};
    __syncthreads();
    const PartRows<true> part(E, pl, pl.part);
    const int groups = (E.dv + 3) / 4, count = min(E.tile, pl.len - pl.t0) * E.pack;
#pragma unroll 1
    for (int x = tid; x < count * groups; x += 64 * WAVES) {
        const int row = (int)fdiv(x, E.by_groups), c = 4 * (x - row * groups);
        float m = -FLT_MAX, sum = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) m = fmaxf(m, s_sums[w][row][0]);
        f32x4 o{0, 0, 0, 0};
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const f32x2 s = s_sums[w][row];
            const float f = __builtin_amdgcn_exp2f(s[0] - m);
            sum += s[1] * f;
            o += *reinterpret_cast<const f32x4*>(&sO[(w * 32 + row) * PITCH + c]) * f;
        }
        if (pl.parts > 1) {
            part.put(row, c, o);
            if (c == 0) part.put_sums(row, f32x2{m, sum});
        } else {
            const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
            const int tt = pl.t0 + (int)fdiv(row, E.by_pack), hh = pl.head + row - (int)fdiv(row, E.by_pack) * E.pack;
            store4<T, VEC>(static_cast<T*>(E.o) + (pl.row0 + tt) * E.o_row + (int64_t)hh * E.o_head + c, E.dv - c, o * inv);
        }
    }
    if (pl.parts > 1) join_last<T, VEC>(E, pl, 64 * WAVES, lds);
}

template <typename T, int DKP, int DVP, bool VEC>
__global__ __launch_bounds__(64 * step_waves<32 * (DKP + DVP) * sizeof(T)>())
__attribute__((amdgpu_waves_per_eu(DKP + DVP <= 256 ? 2 : 1))) void softmax_step_kernel(SoftArgs) {
    __shared__ u32x4 lds[StepTiles<T, DKP, DVP>::LDS];
    __shared__ f32x2 sums[StepTiles<T, DKP, DVP>::WAVES][32];
    __shared__ int pages[StepTiles<T, DKP, DVP>::WAVES][64];
    SoftPlace pl;
    SoftShares shares(args_here());
    while (shares.next(args_here(), &pl)) {
        pl.uniform();
        step_part<T, DKP, DVP, VEC>(args_here(), pl, lds, sums, pages);
        __syncthreads();
    }
}

template <typename T, bool STEP, int DKP, int DVP, bool VEC>
hipError_t launch_softmax_one(const SoftArgs& a, hipStream_t s) {
    constexpr int THREADS = 64 * (STEP ? step_waves<32 * (DKP + DVP) * sizeof(T)>() : kPromptWaves);
    constexpr int64_t MOST = kMostThreads / THREADS;  // workgroups
    const int64_t all = a.shares ? a.shares : a.ids * a.blocks;
    SoftArgs b = a;
    for (int64_t first = 0; first < all; first += MOST) {
        b.first = (int32_t)first;
        const dim3 grid((unsigned)std::min(MOST, all - first));
        if constexpr (STEP) {
            hipLaunchKernelGGL((softmax_step_kernel<T, DKP, DVP, VEC>), grid, dim3(THREADS), 0, s, b);
        } else {
            constexpr int KT = sizeof(T) == 4 && DKP + DVP > 128 ? 32 : 64;
            hipLaunchKernelGGL((softmax_prompt_kernel<T, DKP, DVP, KT, VEC>), grid, dim3(THREADS), 0, s, b);
            if (a.shares)
                hipLaunchKernelGGL((softmax_join_kernel<T, VEC>),
                                   dim3((unsigned)a.shares, (unsigned)((a.tile * a.pack + kJoinRows - 1) / kJoinRows)), dim3(256), 0, s, b);
        }
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// Kernels for heads of up to 64, 128 and 256 elements.
template <typename T, bool STEP, bool VEC>
hipError_t launch_softmax_dims(const SoftArgs& a, hipStream_t s) {
    const int k = a.dk <= 64 ? 64 : a.dk <= 128 ? 128 : 256, v = a.dv <= 64 ? 64 : a.dv <= 128 ? 128 : 256;
    switch (1000 * k + v) {
        case 64064: return launch_softmax_one<T, STEP, 64, 64, VEC>(a, s);
        case 64128: return launch_softmax_one<T, STEP, 64, 128, VEC>(a, s);
        case 64256: return launch_softmax_one<T, STEP, 64, 256, VEC>(a, s);
        case 128064: return launch_softmax_one<T, STEP, 128, 64, VEC>(a, s);
        case 128128: return launch_softmax_one<T, STEP, 128, 128, VEC>(a, s);
        case 128256: return launch_softmax_one<T, STEP, 128, 256, VEC>(a, s);
        case 256064: return launch_softmax_one<T, STEP, 256, 64, VEC>(a, s);
        case 256128: return launch_softmax_one<T, STEP, 256, 128, VEC>(a, s);
        default: return launch_softmax_one<T, STEP, 256, 256, VEC>(a, s);
    }
}
template <typename T, bool STEP>
hipError_t launch_softmax(const SoftArgs& a, bool vec, hipStream_t s) {
    return vec ? launch_softmax_dims<T, STEP, true>(a, s) : launch_softmax_dims<T, STEP, false>(a, s);
}

}  // namespace cv
