// Router: the k largest logits of every token and their softmax weights, and the gradient with respect to the logits.
//
// One warp per token.  Forward: the token's logits live in the lanes' registers as integers whose order is the order of the
// values (0 = masked); a round takes the warp's largest integer and, among the lanes that hold it, the lowest expert id --
// two warp reductions, no shared memory, no sort.  A logit is read once, and the table and weights are written once.
#include <cstdint>

#include "ubep_common.cuh"
#include "ubep_experts.h"
#include "ubep_launch.cuh"

namespace ubep {

namespace {

constexpr int kRouteThreads = 128;
constexpr unsigned kFull = 0xffffffffu;

__device__ __forceinline__ float as_float(float v) { return v; }
__device__ __forceinline__ float as_float(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(uint16_t* p, float v) {
    const __nv_bfloat16 b = __float2bfloat16_rn(v);
    *p = *reinterpret_cast<const uint16_t*>(&b);
}

// Integers in the order of the values; 0 for minus infinity and for no number.  (Both zeros are the same value.)
__device__ __forceinline__ unsigned order_key(float v) {
    if (!(v > -INFINITY)) return 0u;
    const unsigned u = v == 0.0f ? 0u : __float_as_uint(v);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float key_value(unsigned key) {
    if (key == 0u) return -INFINITY;
    return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key);
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(kFull, v, o);
    return v;
}

// V > 0: up to 32 V experts, V logits per lane in registers.  V = 0: any number of experts, a pass over the row per round.
template <typename T, int V>
__global__ void __launch_bounds__(kRouteThreads) route_kernel(const T* logits, int tokens, int E, int k, int renormalize,
                                                             int32_t* topk_idx, float* topk_w) {
    griddep_wait();
    const int lane = threadIdx.x & 31;
    const int64_t t = (int64_t)blockIdx.x * (kRouteThreads / 32) + (threadIdx.x >> 5);
    if (t >= tokens) return;
    const T* row = logits + t * E;
    unsigned key[V ? V : 1];
    if constexpr (V > 0) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int e = i * 32 + lane;
            key[i] = e < E ? order_key(as_float(ld_plain(row + e))) : 0u;
        }
    }
    unsigned my_key = 0u, last_key = kFull, top_key = 0u;
    int my_idx = -1, last_idx = -1;
    float total = 0.0f;
    for (int j = 0; j < k; ++j) {
        unsigned best = 0u;
        int at = 0;
        if constexpr (V > 0) {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (key[i] > best) {
                    best = key[i];
                    at = i * 32 + lane;
                }
        } else {
            // the largest pair behind the last one taken
            for (int e = lane; e < E; e += 32) {
                const unsigned u = order_key(as_float(ld_plain(row + e)));
                if (u > best && (u < last_key || (u == last_key && e > last_idx))) {
                    best = u;
                    at = e;
                }
            }
        }
        const unsigned m = __reduce_max_sync(kFull, best);
        if (m == 0u) break;
        const int e = (int)__reduce_min_sync(kFull, best == m ? (unsigned)at : kFull);
        if (j == 0) {
            top_key = m;
            if (!renormalize) {
                const float most = key_value(m);
                if constexpr (V > 0) {
#pragma unroll
                    for (int i = 0; i < V; ++i) total += expf(key_value(key[i]) - most);
                } else {
                    for (int i = lane; i < E; i += 32) total += expf(key_value(order_key(as_float(ld_plain(row + i)))) - most);
                }
            }
        }
        if (lane == j) {
            my_key = m;
            my_idx = e;
        }
        last_key = m;
        last_idx = e;
        if constexpr (V > 0) {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (i * 32 + lane == e) key[i] = 0u;
        }
    }
    const float value = my_idx >= 0 ? expf(key_value(my_key) - key_value(top_key)) : 0.0f;
    total = warp_sum(renormalize ? value : total);
    if (lane < k) {
        topk_idx[t * k + lane] = my_idx;
        topk_w[t * k + lane] = my_idx >= 0 ? value / total : 0.0f;
    }
}

// With the weights w of the chosen experts (renormalised: their softmax; otherwise every expert's probability p) and
// m = sum_j w_j g_j: renormalised w_j (g_j - m) for the chosen and 0 elsewhere, otherwise p_e ([chosen] g_e - m).
template <typename T>
__global__ void __launch_bounds__(kRouteThreads) route_grad_kernel(const T* logits, const int32_t* topk_idx, const float* grad_w, int tokens,
                                                                  int E, int k, int renormalize, T* grad_logits) {
    griddep_wait();
    const int lane = threadIdx.x & 31;
    const int64_t t = (int64_t)blockIdx.x * (kRouteThreads / 32) + (threadIdx.x >> 5);
    if (t >= tokens) return;
    const T* row = logits + t * E;
    T* out = grad_logits + t * E;
    int idx = lane < k ? ld_plain(topk_idx + t * k + lane) : -1;
    if (idx < 0 || idx >= E) idx = -1 - lane;
    // a second slot with the same expert counts as empty, as in dispatch
    const bool first = __ffs(__match_any_sync(kFull, idx)) - 1 == lane;
    const bool used = idx >= 0 && first;
    const float mine = used ? key_value(order_key(as_float(ld_plain(row + idx)))) : -INFINITY;
    float most = mine, total;
    if (!renormalize)
        for (int e = lane; e < E; e += 32) most = fmaxf(most, key_value(order_key(as_float(ld_plain(row + e)))));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(kFull, most, o));
    const bool any = most > -INFINITY;
    if (renormalize) {
        total = used && any ? expf(mine - most) : 0.0f;
    } else {
        total = 0.0f;
        if (any)
            for (int e = lane; e < E; e += 32) total += expf(key_value(order_key(as_float(ld_plain(row + e)))) - most);
    }
    total = warp_sum(total);
    const float w = used && any ? expf(mine - most) / total : 0.0f;
    const float g = used ? ld_plain(grad_w + t * k + lane) : 0.0f;
    const float mean = warp_sum(w * g);
    for (int e = lane; e < E; e += 32) {
        float v = 0.0f;
        if (!renormalize && any) v = -(expf(key_value(order_key(as_float(ld_plain(row + e)))) - most) / total) * mean;
        put(out + e, v);
    }
    __syncwarp();
    if (used) put(out + idx, w * (g - mean));
}

template <typename T>
cudaError_t launch(const void* logits, int tokens, int E, int k, int renormalize, int32_t* idx, float* w, cudaStream_t st) {
    const int grid = (int)(((int64_t)tokens + kRouteThreads / 32 - 1) / (kRouteThreads / 32));
    auto go = [&](auto kern) {
        return launch_overlapped(kern, grid, kRouteThreads, 0, st, false, 1, static_cast<const T*>(logits), tokens, E, k, renormalize, idx, w);
    };
    if (E <= 32) return go(route_kernel<T, 1>);
    if (E <= 64) return go(route_kernel<T, 2>);
    if (E <= 128) return go(route_kernel<T, 4>);
    if (E <= 256) return go(route_kernel<T, 8>);
    if (E <= 512) return go(route_kernel<T, 16>);
    if (E <= 1024) return go(route_kernel<T, 32>);
    return go(route_kernel<T, 0>);
}

}  // namespace

cudaError_t launch_route(const void* logits, int type, int T, int E, int k, int renormalize, int32_t* topk_idx, float* topk_w,
                         cudaStream_t st) {
    return type == UBEP_LOGITS_F32 ? launch<float>(logits, T, E, k, renormalize, topk_idx, topk_w, st)
                                   : launch<uint16_t>(logits, T, E, k, renormalize, topk_idx, topk_w, st);
}

cudaError_t launch_route_backward(const void* logits, int type, const int32_t* topk_idx, const float* grad_w, int T, int E, int k,
                                  int renormalize, void* grad_logits, cudaStream_t st) {
    const int grid = (int)(((int64_t)T + kRouteThreads / 32 - 1) / (kRouteThreads / 32));
    if (type == UBEP_LOGITS_F32)
        return launch_overlapped(route_grad_kernel<float>, grid, kRouteThreads, 0, st, false, 1, static_cast<const float*>(logits), topk_idx,
                                 grad_w, T, E, k, renormalize, static_cast<float*>(grad_logits));
    return launch_overlapped(route_grad_kernel<uint16_t>, grid, kRouteThreads, 0, st, false, 1, static_cast<const uint16_t*>(logits),
                             topk_idx, grad_w, T, E, k, renormalize, static_cast<uint16_t*>(grad_logits));
}

}  // namespace ubep
