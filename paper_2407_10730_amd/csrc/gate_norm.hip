// gate_norm.hip -- the norms after and before a block with its gate, residual scale and sum.
//
//   n = post(u) act(gate)   or   post(u act(gate));    y = residual + scale scale_vec n;    h = pre(y)
//
// Bound by memory: each tensor is read or written once (8192 x 2048 bf16 by heads of 128 with a gate in 20.7 us, 4.9
// TB/s; with residual and the next norm in 26.0, 5.1 TB/s; 13 rows of 1537 fp32 in 4.5, a launch and four reductions).
// TPR threads hold one group (a row, or a head of it) in registers between the reductions; statistics, products and y
// stay in fp32 until they are stored.  The mean of a LAYER norm is taken off before the squares are summed, so a large
// mean costs no digits.
#include "seqmix_device.h"

namespace cv {

// Sum over the TPR threads of a group; `red` (one float per wave) is used when a group spans waves.
template <int TPR>
__device__ __forceinline__ float group_sum(float v, float* red) {
    v = lanes_sum<(TPR < 64 ? TPR : 64)>(v);
    if constexpr (TPR > 64) {
        __syncthreads();  // the previous sum has been read
        if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0.0f;
#pragma unroll
        for (int i = 0; i < TPR / 64; ++i) v += red[i];
    }
    return v;
}

// fp32 values [width] that a thread needs at its places.  EARLY loads them before the reductions that they wait for.
template <int TPR, int V, int ITEMS, bool EARLY>
struct Vec {
    static constexpr bool kEarly = EARLY;
    const float* p;
    float e[kEarly ? ITEMS : 1][V];
    __device__ __forceinline__ Vec(const float* q, int n) : p(q) {
        if constexpr (kEarly) {
#pragma unroll
            for (int i = 0; i < ITEMS; ++i) {
                const RowPlace<V> at((i * TPR + threadIdx.x % TPR) * V, n);
                if (p && at.on) load_pack<float, V>(p + at.c, e[i]);
            }
        }
    }
    __device__ __forceinline__ void get(int i, int c, float (&out)[V]) const {
        if constexpr (kEarly) {
#pragma unroll
            for (int v = 0; v < V; ++v) out[v] = e[i][v];
        } else {
            load_pack<float, V>(p + c, out);
        }
    }
};

// Zeros in the places that the thread does not own.
template <int TPR, int V, int ITEMS>
__device__ __forceinline__ void clear_unowned(float (&x)[ITEMS][V], int n) {
    if (V == 1 || n % V == 0) return;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const RowPlace<V> at((i * TPR + threadIdx.x % TPR) * V, n);
#pragma unroll
        for (int v = 0; v < V; ++v) x[i][v] = v < at.skip ? 0.0f : x[i][v];
    }
}

// Norms x in place: V * ITEMS values per thread, those at or past `n` being zero.
template <int TPR, int V, int ITEMS, bool EARLY>
__device__ __forceinline__ void norm_in_place(float (&x)[ITEMS][V], int kind, float eps, const Vec<TPR, V, ITEMS, EARLY>& w,
                                              const Vec<TPR, V, ITEMS, EARLY>& b, int n, float* red) {
    const int t = threadIdx.x % TPR;
    const float inv = 1.0f / (float)n;
    clear_unowned<TPR, V, ITEMS>(x, n);
    if (kind == SEQMIX_NORM_LAYER) {
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i)
#pragma unroll
            for (int v = 0; v < V; ++v) s += x[i][v];
        const float mean = group_sum<TPR>(s, red) * inv;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i)
#pragma unroll
            for (int v = 0; v < V; ++v) x[i][v] = (i * TPR + t) * V < n ? x[i][v] - mean : 0.0f;
        clear_unowned<TPR, V, ITEMS>(x, n);
    }
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i)
#pragma unroll
        for (int v = 0; v < V; ++v) s = fmaf(x[i][v], x[i][v], s);
    const float r = 1.0f / sqrtf(fmaf(group_sum<TPR>(s, red), inv, eps));
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const RowPlace<V> at((i * TPR + t) * V, n);
        if (at.on) {
            float e[V];
            w.get(i, at.c, e);
#pragma unroll
            for (int v = 0; v < V; ++v) x[i][v] *= r * e[v];
            if (b.p) {
                b.get(i, at.c, e);
#pragma unroll
                for (int v = 0; v < V; ++v) x[i][v] += e[v];
            }
        }
    }
}

template <typename T, typename TR, int TPR, int V, int ITEMS, bool EARLY>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void gate_norm_kernel(NormArgs A) {
    constexpr int NT = TPR < 256 ? 256 : TPR;
    __shared__ float red[NT / 64];
    const int t = threadIdx.x % TPR;
    int64_t id = (int64_t)blockIdx.x * (NT / TPR) + threadIdx.x / TPR;
    const bool live = id < A.rows;  // TPR > 64 has one group per block: all its threads agree
    id = live ? id : A.rows - 1;
    // (64-bit divisions take longer than a small group's sums: 8105 x 4096 bf16 by groups of 128 53.2 us, 49.9; 64 x 200
    // 4.3, 4.0)
    const bool few = A.rows <= 0x7fffffff;
    const int64_t row = few ? fdiv((uint32_t)id, A.by_groups) : id / A.ngroups;
    const int64_t col = (id - row * A.ngroups) * A.group;
    const int n = A.group;

    float x[ITEMS][V];
    Pack<T, V> gate[ITEMS];
    Pack<TR, V> res[ITEMS];
    const T* u = static_cast<const T*>(A.u) + row * A.u_row + col;
    const T* gp = static_cast<const T*>(A.gate) + (A.gate ? (int64_t)fdiv((uint32_t)row, A.by_run) * A.gate_row + col : 0);
    const TR* rp = static_cast<const TR*>(A.res) + (A.res ? row * A.res_row + col : 0);
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const RowPlace<V> at((i * TPR + t) * V, n);
#pragma unroll
        for (int v = 0; v < V; ++v) x[i][v] = 0.0f;
        if (at.on) {
            load_pack<T, V>(u + at.c, x[i]);
            if (A.gate) gate[i] = *reinterpret_cast<const Pack<T, V>*>(gp + at.c);
            if (A.res) res[i] = *reinterpret_cast<const Pack<TR, V>*>(rp + at.c);
        }
    }
    const Vec<TPR, V, ITEMS, EARLY> post_w(A.post_w, n), post_b(A.post_b, n), scale_vec(A.scale_vec ? A.scale_vec + col : nullptr, n),
        pre_w(A.pre_w, n), pre_b(A.pre_b, n);
    auto apply_gate = [&] {
#pragma unroll
        for (int i = 0; i < ITEMS; ++i)
            if ((i * TPR + t) * V < n) {
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const float z = to_f32(gate[i].e[v]);
                    x[i][v] *= A.gate_act == SEQMIX_ACT_LINEAR ? z
                               : A.gate_act == SEQMIX_ACT_SILU ? silu(z)
                                                               : sigmoid(z);
                }
            }
    };
    if (A.gate && A.gate_first) apply_gate();
    if (A.post != SEQMIX_NORM_NONE) norm_in_place<TPR, V, ITEMS, EARLY>(x, A.post, A.post_eps, post_w, post_b, n, red);
    if (A.gate && !A.gate_first) apply_gate();

    TR* yp = static_cast<TR*>(A.y) + (A.y ? row * A.y_row + col : 0);
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const RowPlace<V> at((i * TPR + t) * V, n);
        if (at.on) {
            float e[V];
#pragma unroll
            for (int v = 0; v < V; ++v) e[v] = 1.0f;
            if (scale_vec.p) scale_vec.get(i, at.c, e);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                x[i][v] *= A.scale * e[v];
                if (A.res) x[i][v] += to_f32(res[i].e[v]);
            }
            if (A.y && live) store_owned<TR, V>(yp + at.c, x[i], at.skip, A.past);
        }
    }
    if (A.pre == SEQMIX_NORM_NONE) return;
    norm_in_place<TPR, V, ITEMS, EARLY>(x, A.pre, A.pre_eps, pre_w, pre_b, n, red);
    T* hp = static_cast<T*>(A.h) + row * A.h_row + col;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const RowPlace<V> at((i * TPR + t) * V, n);
        if (at.on && live) store_owned<T, V>(hp + at.c, x[i], at.skip, A.past);
    }
}

template <typename T, typename TR, int TPR, int V, int ITEMS>
static hipError_t launch_one(const NormArgs& a, hipStream_t s) {
    constexpr int NT = TPR < 256 ? 256 : TPR;
    const int64_t blocks = (a.rows + NT / TPR - 1) / (NT / TPR);
    if (blocks > 0x7fffffffLL) return hipErrorInvalidValue;
    // With fewer than two blocks per CU the time is one block's chain of loads: weights early take one wait out of it (13 rows of
    // 1537 fp32 6.5 -> 5.1 us).  With many, their registers cost waves (8192 x 2048 bf16 by heads of 128: 26 us, late 23.5).
    if (ITEMS * V <= 8 && blocks < 2 * kSeqmixCUs)
        hipLaunchKernelGGL((gate_norm_kernel<T, TR, TPR, V, ITEMS, (ITEMS * V <= 8)>), dim3((unsigned)blocks), dim3(NT), 0, s, a);
    else
        hipLaunchKernelGGL((gate_norm_kernel<T, TR, TPR, V, ITEMS, false>), dim3((unsigned)blocks), dim3(NT), 0, s, a);
    return hipGetLastError();
}

// V values per access: 16 bytes, or 1 in groups below that.  Groups up to 16 accesses: 16 lanes each; up to 64: a wave;
// above, a block of 256 to 1024 threads.  The sizes between take half of the threads with two accesses each (fewer idle
// ones and shorter sums): 8105 x 4096 fp32 by groups of 128 with 64 lanes 117 us, with 16 81; 16000 x 1000 bf16 45.8,
// 35.1; 2000 x 4096 fp32 34.5, 31.4.  Two accesses of 8 values wait longer for their weights, so in bf16 only where
// there are rows for all CUs (64 x 1000: 4.4, 6.0 us); in fp32 from one row per CU on (64 x 1500: 4.2, 4.4; x 4096: 5.3,
// 5.1).
template <typename T, typename TR, int V>
static hipError_t launch_v(const NormArgs& a, hipStream_t s) {
    const int64_t packs = (a.group + V - 1) / V;
    const bool two = a.rows >= (V <= 4 ? 1 : 8) * kSeqmixCUs;
    if (packs <= 16) return launch_one<T, TR, 16, V, 1>(a, s);
    if constexpr (V > 1) {
        if (packs <= 32 && two) return launch_one<T, TR, 16, V, 2>(a, s);
        if (packs <= 64) return launch_one<T, TR, 64, V, 1>(a, s);
        if (packs <= 128 && two) return launch_one<T, TR, 64, V, 2>(a, s);
        if (packs <= 256) return launch_one<T, TR, 256, V, 1>(a, s);
        if (packs <= 512) return two ? launch_one<T, TR, 256, V, 2>(a, s) : launch_one<T, TR, 512, V, 1>(a, s);
        if (packs <= 1024) return two || V <= 4 ? launch_one<T, TR, 512, V, 2>(a, s) : launch_one<T, TR, 1024, V, 1>(a, s);
        if (packs <= 2048) return launch_one<T, TR, 1024, V, 2>(a, s);
        if constexpr (V == 4) return launch_one<T, TR, 1024, V, 4>(a, s);
    }
    return hipErrorInvalidValue;
}

hipError_t launch_norm(const NormArgs& a, int dt, int rdt, hipStream_t s) {
    if (a.rows == 0) return hipSuccess;
    if (dt == CONV2D_F32) return a.group < 4 ? launch_v<float, float, 1>(a, s) : launch_v<float, float, 4>(a, s);
    if (rdt == CONV2D_F32) return a.group < 8 ? launch_v<uint16_t, float, 1>(a, s) : launch_v<uint16_t, float, 8>(a, s);
    return a.group < 8 ? launch_v<uint16_t, uint16_t, 1>(a, s) : launch_v<uint16_t, uint16_t, 8>(a, s);
}

}  // namespace cv
