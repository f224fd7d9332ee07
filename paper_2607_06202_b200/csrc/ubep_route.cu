// Router: the k largest logits of every token and their softmax weights, and the gradient with respect to the logits.
//
// One warp per token.  Forward: every lane makes a number of each of its logits whose order is (value, then lower expert id), 0 for a
// masked one, and knows its two largest; a round takes the largest of the warp with a reduction, and the lane that held it moves
// its second one up, or looks its numbers over again where that one is gone too.  Of bf16 logits value and id fit in 32 bits, one
// reduction; fp32 logits take 64 and two.  A logit is read once, the table and weights are written once.  What bounds it is
// issuing instructions, 433 per token of 256 bf16 logits (70 % of the issue slots busy), 633 of fp32 (50 %, the two reductions wait).
// 16384 tokens x 256 experts of bf16, k = 8: 9.0 us with the logits in L2, 10.5 from memory (fp32: 20.9); searched anew in every
// round 18.0, every lane's numbers sorted 10.8 (in L2), the lanes' sorted lists merged over the warp 13.1.
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

// Integers in the order of the values; 0 for minus infinity and for no number.  (Both zeros are the same value: the sum with zero.)
__device__ __forceinline__ unsigned order_key(float v) {
    const unsigned u = __float_as_uint(__fadd_rn(v, 0.0f));
    const unsigned key = u ^ ((unsigned)((int)u >> 31) | 0x80000000u);
    return v > -INFINITY ? key : 0u;
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

// Value and expert id as one number: larger value first, then the lower id; 0 = masked.
template <typename T> struct Ranked;
template <> struct Ranked<uint16_t> {
    typedef unsigned Num;
    static __device__ __forceinline__ Num make(float v, int e) {
        const unsigned key = order_key(v);   // (of a bf16 the lower half of the key is all ones or all zeros)
        return key ? (key & 0xffff0000u) | (0xffffu - (unsigned)e) : 0u;
    }
    static __device__ __forceinline__ Num largest(Num n) { return __reduce_max_sync(kFull, n); }
    static __device__ __forceinline__ int id(Num n) { return (int)(0xffffu - (n & 0xffffu)); }
    static __device__ __forceinline__ float value(Num n) {
        if (n == 0u) return -INFINITY;
        return __uint_as_float(n & 0x80000000u ? (n ^ 0x80000000u) & 0xffff0000u : ~n & 0xffff0000u);
    }
};
template <> struct Ranked<float> {
    typedef unsigned long long Num;
    static __device__ __forceinline__ Num make(float v, int e) {
        const unsigned key = order_key(v);
        return key ? ((Num)key << 32) | (0xffffu - (unsigned)e) : 0ull;
    }
    static __device__ __forceinline__ Num largest(Num n) {
        const unsigned high = (unsigned)(n >> 32), top = __reduce_max_sync(kFull, high);
        return ((Num)top << 32) | __reduce_max_sync(kFull, high == top ? (unsigned)n : 0u);
    }
    static __device__ __forceinline__ int id(Num n) { return (int)(0xffffu - ((unsigned)n & 0xffffu)); }
    static __device__ __forceinline__ float value(Num n) { return key_value((unsigned)(n >> 32)); }
};

// V > 0: up to 32 V experts, V logits per lane in registers.  V = 0: any number of experts, a pass over the row per round.
template <typename T, int V>
__global__ void __launch_bounds__(kRouteThreads) route_kernel(const T* logits, int tokens, int E, int k, int renormalize,
                                                             int32_t* topk_idx, float* topk_w) {
    typedef Ranked<T> R;
    typedef typename R::Num Num;
    griddep_wait();
    const int lane = threadIdx.x & 31;
    const int64_t t = (int64_t)blockIdx.x * (kRouteThreads / 32) + (threadIdx.x >> 5);
    if (t >= tokens) return;
    const T* row = logits + t * E;
    Num mine[V ? V : 1];
    if constexpr (V > 0) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int e = i * 32 + lane;
            mine[i] = e < E ? R::make(as_float(ld_plain(row + e)), e) : 0;
        }
    }
    Num best = 0, second = 0;   // of this lane; second = 0: none, or not known
    if constexpr (V > 0) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const Num low = mine[i] < best ? mine[i] : best;
            best = mine[i] < best ? best : mine[i];
            second = low < second ? second : low;
        }
    }
    Num chosen = 0, last = ~(Num)0, top = 0;
    float total = 0.0f;
    for (int j = 0; j < k; ++j) {
        if constexpr (V == 0) {
            // the largest behind the last one taken
            best = 0;
            for (int e = lane; e < E; e += 32) {
                const Num n = R::make(as_float(ld_plain(row + e)), e);
                if (n > best && n < last) best = n;
            }
        }
        last = R::largest(best);
        if (last == 0) break;
        if (j == 0) {
            top = last;
            if (!renormalize) {
                const float most = R::value(last);
                if constexpr (V > 0) {
#pragma unroll
                    for (int i = 0; i < V; ++i) total += expf(R::value(mine[i]) - most);
                } else {
                    for (int e = lane; e < E; e += 32) total += expf(R::value(R::make(as_float(ld_plain(row + e)), e)) - most);
                }
            }
        }
        if (lane == j) chosen = last;
        if constexpr (V > 0) {
            if (best == last) {
                best = second;
                second = 0;
                if (best == 0) {
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const Num n = mine[i] < last ? mine[i] : 0;
                        best = n > best ? n : best;
                    }
                }
            }
        }
    }
    const float value = chosen ? expf(R::value(chosen) - R::value(top)) : 0.0f;
    total = warp_sum(renormalize ? value : total);
    if (lane < k) {
        topk_idx[t * k + lane] = chosen ? R::id(chosen) : -1;
        topk_w[t * k + lane] = chosen ? value / total : 0.0f;
    }
}

// With the weights w of the chosen experts (renormalised: their softmax; otherwise every expert's probability p) and
// m = sum_j w_j g_j: renormalised w_j (g_j - m) for the chosen and 0 elsewhere, otherwise p_e ([chosen] g_e - m).
// V > 0: up to 32 V experts, a lane's exponentials in registers.
template <typename T, int V>
__global__ void __launch_bounds__(kRouteThreads) route_grad_kernel(const T* logits, const int32_t* topk_idx, const float* grad_w, int tokens,
                                                                  int E, int k, int renormalize, T* grad_logits) {
    griddep_wait();
    const int lane = threadIdx.x & 31;
    const int64_t t = (int64_t)blockIdx.x * (kRouteThreads / 32) + (threadIdx.x >> 5);
    if (t >= tokens) return;
    const T* row = logits + t * E;
    T* out = grad_logits + t * E;
    auto logit = [&](int e) {   // masked: minus infinity
        const float v = as_float(ld_plain(row + e));
        return v > -INFINITY ? v : -INFINITY;
    };
    int idx = lane < k ? ld_plain(topk_idx + t * k + lane) : -1;
    const float given = lane < k ? ld_plain(grad_w + t * k + lane) : 0.0f;
    float p[V ? V : 1];
    float most = -INFINITY;
    if (!renormalize) {
        if constexpr (V > 0) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int e = i * 32 + lane;
                p[i] = e < E ? logit(e) : -INFINITY;
                most = fmaxf(most, p[i]);
            }
        } else {
            for (int e = lane; e < E; e += 32) most = fmaxf(most, logit(e));
        }
    }
    if (idx < 0 || idx >= E) idx = -1 - lane;
    // a second slot with the same expert counts as empty, as in dispatch
    const bool first = __ffs(__match_any_sync(kFull, idx)) - 1 == lane;
    const float mine = idx >= 0 && first ? logit(idx) : -INFINITY;
    const bool used = mine > -INFINITY;   // (a masked expert has no weight: whatever its slot's gradient is, it is not looked at)
    most = fmaxf(most, mine);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(kFull, most, o));
    const bool any = most > -INFINITY;
    const float base = any ? most : 0.0f;   // (without a logit left every exponential is 0)
    const float value = expf(mine - base);
    float total = value;
    if (!renormalize) {
        total = 0.0f;
        if constexpr (V > 0) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                p[i] = expf(p[i] - base);
                total += p[i];
            }
        } else {
            for (int e = lane; e < E; e += 32) total += expf(logit(e) - base);
        }
    }
    total = warp_sum(total);
    const float share = any ? 1.0f / total : 0.0f;
    const float w = value * share, g = used ? given : 0.0f;
    const float mean = warp_sum(w * g);
    if constexpr (V > 0) {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i * 32 + lane < E) put(out + i * 32 + lane, renormalize ? 0.0f : -p[i] * share * mean);
    } else {
        for (int e = lane; e < E; e += 32) put(out + e, renormalize ? 0.0f : -expf(logit(e) - base) * share * mean);
    }
    __syncwarp();   // (the row is written by now: the chosen ones' own values come last)
    if (used) put(out + idx, w * (g - mean));
}

int route_grid(int tokens) { return (int)(((int64_t)tokens + kRouteThreads / 32 - 1) / (kRouteThreads / 32)); }

template <typename T>
cudaError_t launch(const void* logits, int tokens, int E, int k, int renormalize, int32_t* idx, float* w, cudaStream_t st) {
    auto go = [&](auto kern) {
        return launch_overlapped(kern, route_grid(tokens), kRouteThreads, 0, st, false, 1, static_cast<const T*>(logits), tokens, E, k,
                                 renormalize, idx, w);
    };
    if (E <= 32) return go(route_kernel<T, 1>);
    if (E <= 64) return go(route_kernel<T, 2>);
    if (E <= 128) return go(route_kernel<T, 4>);
    if (E <= 192) return go(route_kernel<T, 6>);
    if (E <= 256) return go(route_kernel<T, 8>);
    if (E <= 320) return go(route_kernel<T, 10>);
    if (E <= 512) return go(route_kernel<T, 16>);
    return go(route_kernel<T, 0>);
}

template <typename T>
cudaError_t launch_grad(const void* logits, const int32_t* idx, const float* grad_w, int tokens, int E, int k, int renormalize, void* out,
                        cudaStream_t st) {
    auto go = [&](auto kern) {
        return launch_overlapped(kern, route_grid(tokens), kRouteThreads, 0, st, false, 1, static_cast<const T*>(logits), idx, grad_w, tokens,
                                 E, k, renormalize, static_cast<T*>(out));
    };
    if (E <= 64) return go(route_grad_kernel<T, 2>);
    if (E <= 128) return go(route_grad_kernel<T, 4>);
    if (E <= 320) return go(route_grad_kernel<T, 10>);
    return go(route_grad_kernel<T, 0>);
}

}  // namespace

cudaError_t launch_route(const void* logits, int type, int T, int E, int k, int renormalize, int32_t* topk_idx, float* topk_w,
                         cudaStream_t st) {
    return type == UBEP_LOGITS_F32 ? launch<float>(logits, T, E, k, renormalize, topk_idx, topk_w, st)
                                   : launch<uint16_t>(logits, T, E, k, renormalize, topk_idx, topk_w, st);
}

cudaError_t launch_route_backward(const void* logits, int type, const int32_t* topk_idx, const float* grad_w, int T, int E, int k,
                                  int renormalize, void* grad_logits, cudaStream_t st) {
    return type == UBEP_LOGITS_F32 ? launch_grad<float>(logits, topk_idx, grad_w, T, E, k, renormalize, grad_logits, st)
                                   : launch_grad<uint16_t>(logits, topk_idx, grad_w, T, E, k, renormalize, grad_logits, st);
}

}  // namespace ubep
