// rotary.hip -- rotary positions of q and k, with k and v written into the cache.
//
// Pair (a, b) turns by the angle position * freq: a' = A (a cos - b sin), b' = A (b cos + a sin).  The angle of a far position
// has many turns, of which only the fraction counts: it is taken in 64 bits as turns, the fraction rounded to 32 (an
// error of 2^-24 turns at most, whatever the position).  A workgroup computes the factors of its tokens once, in LDS, for all heads.
// Bound by memory: each element is read and written once.
#include <algorithm>
#include <type_traits>

#include "seqmix_device.h"

namespace cv {

// Elements of a head as units of a thread: pairs of V elements (or single pairs), then copies of V (or single ones).
template <int V, bool HALF>
struct HeadUnits {
    static __host__ __device__ int pairs(int rot) { return HALF ? rot / 2 / V : rot / V; }           // of V
    static __host__ __device__ int singles(int rot) { return HALF ? rot / 2 % V : rot % V / 2; }     // pairs
    static __host__ __device__ int turned(int rot) { return pairs(rot) + singles(rot); }
    static __host__ __device__ int copies(int n) { return n / V + n % V; }
    static __host__ __device__ int all(int dk, int rot) { return turned(rot) + copies(dk - rot); }
};

template <typename T, int V>
__device__ __forceinline__ void copy_unit(const T* from, T* to, T* too, int n, int u) {
    if (u < n / V) {
        const Pack<T, V> x = *reinterpret_cast<const Pack<T, V>*>(from + u * V);
        if (to) *reinterpret_cast<Pack<T, V>*>(to + u * V) = x;
        if (too) *reinterpret_cast<Pack<T, V>*>(too + u * V) = x;
    } else {
        const int c = n / V * V + (u - n / V);
        const T x = from[c];
        if (to) to[c] = x;
        if (too) too[c] = x;
    }
}

template <typename T, int N>
__device__ __forceinline__ void store_both(T* to, T* too, int c, const float (&v)[N], bool past) {
    if (to) store_result<T, N>(to + c, v, past);
    if (too) store_result<T, N>(too + c, v, past);
}

// Unit u of a head: from -> to and too (NULL: not), f the factors of the token's pairs.
template <typename T, int V, bool HALF>
__device__ __forceinline__ void turn_unit(const T* from, T* to, T* too, const f32x2* f, int dk, int rot, int u, bool past) {
    using U = HeadUnits<V, HALF>;
    const int np = U::pairs(rot), nt = U::turned(rot);
    if (u >= nt) {
        copy_unit<T, V>(from + rot, to ? to + rot : nullptr, too ? too + rot : nullptr, dk - rot, u - nt);
    } else if constexpr (HALF) {
        const int half = rot / 2;
        auto turn = [&](auto n, int c) {
            constexpr int N = decltype(n)::value;
            float a[N], b[N], x[N], y[N];
            load_pack<T, N>(from + c, a);
            load_pack<T, N>(from + half + c, b);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const f32x2 w = f[c + i];
                x[i] = a[i] * w[0] - b[i] * w[1];
                y[i] = b[i] * w[0] + a[i] * w[1];
            }
            store_both<T, N>(to, too, c, x, past);
            store_both<T, N>(to, too, half + c, y, past);
        };
        if (u < np) turn(std::integral_constant<int, V>{}, u * V);
        else turn(std::integral_constant<int, 1>{}, np * V + (u - np));
    } else {
        auto turn = [&](auto n, int c) {
            constexpr int N = decltype(n)::value;
            float a[N], x[N];
            load_pack<T, N>(from + c, a);
#pragma unroll
            for (int i = 0; i < N; i += 2) {
                const f32x2 w = f[(c + i) / 2];
                x[i] = a[i] * w[0] - a[i + 1] * w[1];
                x[i + 1] = a[i + 1] * w[0] + a[i] * w[1];
            }
            store_both<T, N>(to, too, c, x, past);
        };
        if (u < np) turn(std::integral_constant<int, V>{}, u * V);
        else turn(std::integral_constant<int, 2>{}, np * V + 2 * (u - np));
    }
}

constexpr int kRotaryThreads = 256;

template <typename T, int V, bool HALF>
__global__ __launch_bounds__(kRotaryThreads) void rotary_kernel(RotaryArgs A, int tokens_each, FastDiv by_units, FastDiv by_head,
                                                                FastDiv by_value) {
    extern __shared__ f32x2 s_factor[];  // [tokens_each][rot / 2]
    const int half = A.rot / 2;
    const int64_t first = (int64_t)blockIdx.x * tokens_each;
    const int n = (int)min<int64_t>(tokens_each, A.tokens - first);
    for (int x = threadIdx.x; x < n * half; x += kRotaryThreads) {
        const int t = x / half, i = x - t * half;
        const double turns = (double)A.position[first + t] * (A.freqs[i] * 0.15915494309189535);
        float sn, cs;
        sincospif((float)(2.0 * (turns - rint(turns))), &sn, &cs);
        s_factor[x] = f32x2{cs * A.amplitude, sn * A.amplitude};
    }
    __syncthreads();
    using U = HeadUnits<V, HALF>;
    const int heads = A.q ? A.heads : 0, per_head = U::all(A.dk, A.rot), per_value = U::copies(A.dv);
    const int turned = (heads + (A.k ? A.kv_heads : 0)) * per_head;
    const int units = turned + (A.vc ? A.kv_heads * per_value : 0);
    for (int x = threadIdx.x; x < n * units; x += kRotaryThreads) {
        const int t = (int)fdiv((uint32_t)x, by_units);
        int u = x - t * units;
        const int64_t row = first + t;
        int64_t page = -1, at = 0;
        const bool of_q = u < heads * per_head;
        if (!of_q && A.place) {
            const int64_t place = A.place[row];
            if (place >= 0 && place < A.rows) page = place >> A.shift, at = place & ((1 << A.shift) - 1);
        }
        if (u < turned) {
            int h = (int)fdiv((uint32_t)u, by_head);
            u -= h * per_head;
            const f32x2* f = s_factor + t * half;
            if (of_q) {
                turn_unit<T, V, HALF>(static_cast<const T*>(A.q) + row * A.q_row + h * A.q_head,
                                      static_cast<T*>(A.qo) + row * A.qo_row + h * A.qo_head, nullptr, f, A.dk, A.rot, u, A.past);
            } else {
                h -= heads;
                T* const to = A.ko ? static_cast<T*>(A.ko) + row * A.ko_row + h * A.ko_head : nullptr;
                T* const too = A.kc && page >= 0
                                   ? static_cast<T*>(A.kc) + page * A.kp.page + at * A.kp.row + h * A.kp.head : nullptr;
                if (to || too)
                    turn_unit<T, V, HALF>(static_cast<const T*>(A.k) + row * A.k_row + h * A.k_head, to, too, f, A.dk, A.rot, u, A.past);
            }
        } else if (page >= 0) {
            u -= turned;
            const int h = (int)fdiv((uint32_t)u, by_value);
            copy_unit<T, V>(static_cast<const T*>(A.v) + row * A.v_row + h * A.v_head,
                            static_cast<T*>(A.vc) + page * A.vp.page + at * A.vp.row + h * A.vp.head, nullptr, A.dv,
                            u - h * per_value);
        }
    }
}

template <typename T, bool HALF>
static hipError_t launch(const RotaryArgs& a, hipStream_t s) {
    constexpr int V = 16 / sizeof(T);
    using U = HeadUnits<V, HALF>;
    const int heads = (a.q ? a.heads : 0) + (a.k ? a.kv_heads : 0);
    const int per_head = U::all(a.dk, a.rot), per_value = U::copies(a.dv);
    const int units = heads * per_head + (a.vc ? a.kv_heads * per_value : 0);
    if (a.tokens == 0 || units == 0) return hipSuccess;
    const int each = a.tokens >= 1024 ? 4 : 1;
    constexpr int64_t MOST = 1 << 25;  // tokens of a launch: up to 2^31 threads
    RotaryArgs b = a;
    for (int64_t t0 = 0; t0 < a.tokens; t0 += MOST) {
        b.tokens = std::min(MOST, a.tokens - t0);
        const int64_t blocks = (b.tokens + each - 1) / each;
        hipLaunchKernelGGL((rotary_kernel<T, V, HALF>), dim3((unsigned)blocks), dim3(kRotaryThreads),
                           (size_t)each * (a.rot / 2) * sizeof(f32x2), s, b, each, make_fastdiv((uint32_t)units),
                           make_fastdiv((uint32_t)per_head), make_fastdiv((uint32_t)std::max(per_value, 1)));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        auto on = [](auto& p, int64_t row) {  // to the next launch's first row
            if (p) p = static_cast<const T*>(p) + MOST * row;
        };
        auto on_out = [](void*& p, int64_t row) {
            if (p) p = static_cast<T*>(p) + MOST * row;
        };
        on(b.q, a.q_row), on(b.k, a.k_row), on(b.v, a.v_row);
        on_out(b.qo, a.qo_row), on_out(b.ko, a.ko_row);
        b.position += MOST;
        if (b.place) b.place += MOST;
    }
    return hipSuccess;
}

hipError_t launch_rotary(const RotaryArgs& a, int dt, int layout, hipStream_t s) {
    const bool half = layout == SEQMIX_ROTARY_HALF;
    if (dt == CONV2D_BF16) return half ? launch<uint16_t, true>(a, s) : launch<uint16_t, false>(a, s);
    return half ? launch<float, true>(a, s) : launch<float, false>(a, s);
}

}  // namespace cv
