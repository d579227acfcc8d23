// seqmix_device.h -- device helpers of the token-mixing kernels.
#pragma once

#include "device_common.h"
#include "seqmix_internal.h"

namespace cv {

typedef u32x4 u32x4_any __attribute__((aligned(2)));  // at any address that an element may have

constexpr float kLog2e = 1.4426950408889634f;

// 16-bit storage stands for bf16 throughout (uint16_t).
__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(uint16_t v) { return __builtin_bit_cast(float, (uint32_t)v << 16); }
template <typename T>
__device__ __forceinline__ T from_f32(float v);
template <>
__device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ uint16_t from_f32<uint16_t>(float v) {  // the hardware's conversion: nearest even, NaN kept
    return __builtin_bit_cast(uint16_t, (__bf16)v);
}

// N consecutive elements as they lie in memory, at any address that an element may have: 8 and 16 bytes are still one load
// or store.
template <typename T, int N>
struct Pack {
    T e[N];
};
template <typename T, int N>
__device__ __forceinline__ void load_pack(const T* p, float (&out)[N]) {
    const Pack<T, N> v = *reinterpret_cast<const Pack<T, N>*>(p);
#pragma unroll
    for (int i = 0; i < N; ++i) out[i] = to_f32(v.e[i]);
}
template <typename T, int N>
__device__ __forceinline__ void store_pack(T* p, const float (&in)[N]) {
    Pack<T, N> v;
#pragma unroll
    for (int i = 0; i < N; ++i) v.e[i] = from_f32<T>(in[i]);
    *reinterpret_cast<Pack<T, N>*>(p) = v;
}

// The N of a thread's elements of a row of n >= N (N is 1, or fewer than N are one by one): from `first` on, and where that passes
// the end the row's last N, of which the thread owns those from `skip` on.
template <int N>
struct RowPlace {
    int c, skip;
    bool on;
    __device__ __forceinline__ RowPlace(int first, int n) {
        on = first < n;
        c = on ? min(first, n - N) : first;
        skip = first - c;
    }
};

// ... past the caches where `past` (full 16-byte stores only): results larger than the L2s push out what is still to be
// read, and their lines are not fetched for writing.
template <typename T, int N>
__device__ __forceinline__ void store_result(T* p, const float (&in)[N], bool past) {
    Pack<T, N> v;
#pragma unroll
    for (int i = 0; i < N; ++i) v.e[i] = from_f32<T>(in[i]);
    if constexpr (sizeof(v) == 16) {
        if (past) {
            asm volatile("" ::: "memory");  // or the two stores become one, without the hint
            __builtin_nontemporal_store(__builtin_bit_cast(u32x4_any, v), reinterpret_cast<u32x4_any*>(p));
            asm volatile("" ::: "memory");
            return;
        }
    }
    *reinterpret_cast<Pack<T, N>*>(p) = v;
}

// ... of those from `skip` on.
template <typename T, int N>
__device__ __forceinline__ void store_owned(T* p, const float (&in)[N], int skip, bool past) {
    if (N == 1 || skip == 0) {
        store_result<T, N>(p, in, past);
    } else {
#pragma unroll
        for (int i = 1; i < N; ++i)
            if (i >= skip) p[i] = from_f32<T>(in[i]);
    }
}

// Rows [first, first + len) of sequence i, clamped so that no offsets lead outside the call's rows.  Row numbers, slots
// and parts are below 2^31 (the descriptors refuse more), so their divisions are 32-bit ones.
struct SeqRange {
    int64_t first, len;
};
__device__ __forceinline__ uint32_t clamp_row(int64_t r, int64_t tokens) {
    return (uint32_t)(r < 0 ? 0 : r > tokens ? tokens : r);
}
__device__ __forceinline__ SeqRange seq_range(const SeqArgs& a, int i) {
    if (!a.off) return {(int64_t)i * a.seq_len, a.seq_len};
    const int64_t b = clamp_row(a.off[i], a.tokens), e = clamp_row(a.off[i + 1], a.tokens);
    return {b, e > b ? e - b : 0};
}
// Pool entry of sequence i, -1: the sequence is skipped.
__device__ __forceinline__ int64_t seq_slot(const SeqArgs& a, int i) {
    if (!a.slot) return i;
    const int64_t s = a.slot[i];
    return s >= 0 && s < a.slots ? s : -1;
}

// Parts of `size` tokens of all sequences, numbered so that no prefix sum over the sequences is needed:
// sequence i owns the ids [offsets[i] / size + i, offsets[i+1] / size + i + 1), at least
// ceil(len / size) and at least one, so the ids of a call are below tokens / size + seqs.  Sequences of
// equal length own exactly as many as they have parts (seq_parts).
// `places` (with offsets): from mul offsets[i] / size on instead, without an id of their own for sequences without parts.
struct SeqPart {
    int seq;
    int part;  // number of the part within the sequence; negative: none (offsets that lie)
};
__device__ __forceinline__ SeqPart seq_part(const SeqArgs& a, uint32_t id, uint32_t size, bool places = false,
                                            uint32_t mul = 1) {
    if (!a.off) {
        const uint32_t len = (uint32_t)a.seq_len, per = len > size ? (len + size - 1) / size : 1;
        const uint32_t i = id / per;
        return {(int)i, (int)(id - i * per)};
    }
    // the last sequence whose first id is at most `id`: a wave's lanes look at 64 of them at a time, so that the
    // search waits for memory once up to 64 sequences and twice up to 4096 (all lanes of the wave take part)
    auto first_id = [&](int i) { return (places ? mul : 1u) * clamp_row(a.off[i], a.tokens) / size + (places ? 0 : i); };
    int lo = 0;
    const int lane = threadIdx.x & 63;
    for (int n = a.seqs; n > 1;) {
        const int step = (n + 63) / 64, i = lane * step;
        const bool at_most = i < n && first_id(lo + i) <= id;
        const int k = max((int)__popcll(__ballot(at_most)) - 1, 0);  // (none where offsets lie; the count is unsigned)
        lo += k * step;
        n = min(step, n - k * step);
    }
    lo = __builtin_amdgcn_readfirstlane(lo);
    return {lo, (int)id - (int)first_id(lo)};
}

// Log2 of a decay from its natural log.  Logs below -1000 (-infinity among them) have an
// exponential of exactly zero in fp32 anyway; the bound keeps differences of sums finite.  NaN stays.
__device__ __forceinline__ double decay_log2(float g) {
    return (double)(g < -1000.0f ? -1000.0f : g) * 1.4426950408889634;
}

// Sum over groups of N lanes (16 or 64), in every lane.
template <int N>
__device__ __forceinline__ float lanes_sum(float v) {
#define ROTATE_ADD(n) v += __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), 0x120 + n, 0xf, 0xf, false))
    ROTATE_ADD(8);
    ROTATE_ADD(4);
    ROTATE_ADD(2);
    ROTATE_ADD(1);
#undef ROTATE_ADD
    if constexpr (N == 16) return v;
    auto row = [&](int lane) {
        return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane));
    };
    return (row(0) + row(16)) + (row(32) + row(48));
}

// Sums over the lanes up to this one.
__device__ __forceinline__ uint32_t scan_lanes(uint32_t v) {
#define SCAN_STEP(ctrl, rows) v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, ctrl, rows, 0xf, false);
    SCAN_STEP(0x111, 0xf)
    SCAN_STEP(0x112, 0xf)
    SCAN_STEP(0x114, 0xf)
    SCAN_STEP(0x118, 0xf)
    SCAN_STEP(0x142, 0xa)
    SCAN_STEP(0x143, 0xc)
#undef SCAN_STEP
    return v;
}

// 1 / (1 + exp(-x)) on the hardware's exponential and reciprocal (each within 1 ulp of fp32).
__device__ __forceinline__ float sigmoid(float x) {
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-kLog2e * x));
}
__device__ __forceinline__ float silu(float x) { return x * sigmoid(x); }

}  // namespace cv
