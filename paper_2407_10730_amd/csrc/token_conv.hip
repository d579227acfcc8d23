// token_conv.hip -- causal depthwise convolution over tokens with a carried window.
//
//   y[t,c] = act(bias[c] + sum_i w[c,i] x[t - W + 1 + i, c])
//
// Bound by memory: x is read and y written once, 2W operations per value (8192 x 4096 bf16 in 26 us, 5.2 TB/s; a step of 64
// tokens in 4.5, a launch and one chain of loads).  A thread owns V
// neighbouring channels and walks along a tile of tokens with the last W - 1 rows in registers,
// so each row of x is loaded once per tile (and W - 1 of them once more by the next tile).
// A tile lies within one sequence, so the window pool is read by each sequence's tile 0 alone; that
// tile also writes the new window, after its read, which makes the update in place free of races.
#include "seqmix_device.h"

namespace cv {

// Tokens per tile: at width 4 the rows loaded twice are under a tenth of 32; with fewer than two workgroups per CU of
// those, tiles of 8 (shorter chains of loads).  8192 x 4096 bf16: 32 as good as 64, 16 a tenth slower.
constexpr int kConvTile = 32, kConvTileFew = 8, kConvAhead = 8;

// EVEN: the channels are a multiple of V (a step of 64 x 4096 takes 4.65 us without the other case's code, 5.05 with it).
template <typename T, int W, int V, bool EVEN>
__global__ __launch_bounds__(256) void token_conv_kernel(ConvArgs A, int tile) {
    const SeqPart sp = seq_part(A.sq, blockIdx.y + blockIdx.z * 65535u, tile);
    const RowPlace<V> at((blockIdx.x * 256 + threadIdx.x) * V, A.channels);
    const int c = at.c, skip = EVEN ? 0 : at.skip;
    if (!at.on || sp.seq >= A.sq.seqs) return;
    const SeqRange r = seq_range(A.sq, sp.seq);
    const int64_t t0 = (int64_t)sp.part * tile;
    if (sp.part < 0 || (sp.part > 0 && t0 >= r.len)) return;
    const int n = (int)min<int64_t>(r.len - t0, tile);
    const T* __restrict__ x = static_cast<const T*>(A.x) + (r.first + t0) * A.x_row + c;
    T* __restrict__ y = static_cast<T*>(A.y) + (r.first + t0) * A.y_row + c;

    // the first rows and the weights are on their way while the slot, and then the window, are looked up
    Pack<T, V> next[kConvAhead];
#pragma unroll
    for (int u = 0; u < kConvAhead; ++u)
        if (u < n) next[u] = *reinterpret_cast<const Pack<T, V>*>(x + (int64_t)u * A.x_row);
    float w[V * W], bias[V];
    if constexpr (V > 1) {
        load_pack<T, V * W>(static_cast<const T*>(A.w) + (int64_t)c * W, w);
    } else {
#pragma unroll
        for (int i = 0; i < W; ++i) w[i] = to_f32(static_cast<const T*>(A.w)[(int64_t)c * W + i]);
    }
    if (A.bias) {
        load_pack<float, V>(A.bias + c, bias);
    } else {
#pragma unroll
        for (int v = 0; v < V; ++v) bias[v] = 0.0f;
    }
    const int64_t slot = seq_slot(A.sq, sp.seq);
    if (slot < 0) return;
    float row[W][V];  // row[i]: x of tap i
    if constexpr (W > 1) {
        const T* win = static_cast<const T*>(A.win_in) + (slot * (W - 1)) * A.channels + c;
#pragma unroll
        for (int i = 0; i < W - 1; ++i) {
            const int64_t t = t0 - (W - 1) + i;
            if (t >= 0) {
                load_pack<T, V>(x + (int64_t)(i - (W - 1)) * A.x_row, row[i]);
            } else if (A.win_in) {
                load_pack<T, V>(win + (int64_t)i * A.channels, row[i]);
            } else {
#pragma unroll
                for (int v = 0; v < V; ++v) row[i][v] = 0.0f;
            }
        }
        if (sp.part == 0 && A.win_out) {  // rows len .. len + W - 2 of window and sequence together
            T* out = static_cast<T*>(A.win_out) + (slot * (W - 1)) * A.channels + c;
#pragma unroll
            for (int i = 0; i < W - 1; ++i) {
                const int64_t t = r.len + i - (W - 1);
                float e[V];
                if (t >= 0) {
                    load_pack<T, V>(x + t * A.x_row, e);
                } else {  // row i + len of the window, in registers
#pragma unroll
                    for (int j = 0; j < W - 1; ++j)
                        if (j == i + r.len) {
#pragma unroll
                            for (int v = 0; v < V; ++v) e[v] = row[j][v];
                        }
                }
                store_owned<T, V>(out + (int64_t)i * A.channels, e, skip, false);
            }
        }
    }
    for (int t = 0; t < n; t += kConvAhead) {
        Pack<T, V> now[kConvAhead];
#pragma unroll
        for (int u = 0; u < kConvAhead; ++u) {
            now[u] = next[u];
            if (t + kConvAhead + u < n)
                next[u] = *reinterpret_cast<const Pack<T, V>*>(x + (int64_t)(t + kConvAhead + u) * A.x_row);
        }
#pragma unroll
        for (int u = 0; u < kConvAhead; ++u) {
            if (t + u < n) {
                float o[V];
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    row[W - 1][v] = to_f32(now[u].e[v]);
                    o[v] = bias[v];
#pragma unroll
                    for (int i = 0; i < W; ++i) o[v] = fmaf(w[v * W + i], row[i][v], o[v]);
                    if (A.silu) o[v] = silu(o[v]);
                }
                store_owned<T, V>(y + (int64_t)(t + u) * A.y_row, o, skip, A.past);
#pragma unroll
                for (int i = 0; i + 1 < W; ++i)
#pragma unroll
                    for (int v = 0; v < V; ++v) row[i][v] = row[i + 1][v];
            }
        }
    }
}

template <typename T, int V, bool EVEN>
static hipError_t launch_conv_w(const ConvArgs& a, hipStream_t s) {
    const int64_t across = (a.channels + 256 * V - 1) / (256 * V);
    const int tile = a.sq.tokens / kConvTile * across < 2 * kSeqmixCUs ? kConvTileFew : kConvTile;
    const int64_t ids = seq_part_ids(a.sq, tile);
    const int64_t gz = (ids + 65534) / 65535;
    if (gz > 65535) return hipErrorInvalidValue;
    const dim3 grid((unsigned)across, (unsigned)(gz > 1 ? 65535 : ids), (unsigned)gz);
    switch (a.width) {
#define CASE(W)                                                                            \
    case W:                                                                                \
        hipLaunchKernelGGL((token_conv_kernel<T, W, V, EVEN>), grid, dim3(256), 0, s, a, tile); \
        break;
        CASE(1) CASE(2) CASE(3) CASE(4) CASE(5) CASE(6) CASE(7) CASE(8)
#undef CASE
        default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

template <typename T>
static hipError_t launch_conv_t(const ConvArgs& a, hipStream_t s) {
    constexpr int V = 16 / sizeof(T);
    if (a.channels < V) return launch_conv_w<T, 1, true>(a, s);
    return a.channels % V == 0 ? launch_conv_w<T, V, true>(a, s) : launch_conv_w<T, V, false>(a, s);
}

hipError_t launch_token_conv(const ConvArgs& a, int dt, hipStream_t s) {
    return dt == CONV2D_BF16 ? launch_conv_t<uint16_t>(a, s) : launch_conv_t<float>(a, s);
}

}  // namespace cv
