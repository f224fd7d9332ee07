// The expert products' arithmetic and the walk over ragged segments, shared by their kernels.
#pragma once

#include "ubep_common.cuh"

namespace ubep {

enum { kActNone = 0, kActSilu = 1, kActGelu = 2, kActRelu = 3 };

// Sums and activations are taken in 32 bits.  The exponential and the quotient are the fast ones, off by (2 + 1.2 |argument|) and 2 units of
// 2^-23; with them silu is good to (8 + 1.2 |z|) units of its value (below z = -87, where the quotient is under 2^-126, it is 0) and gelu to
// (12 + 0.9 z^2), 2e-5 at z = -13 -- far inside the half step (2^-8 at most) of the bf16 results, in the tails too.
// The normal distribution's Phi(z), and exp(-z^2 / 2): Phi(-|z|) = exp(-z^2 / 2) q(t), t = 1 / (1 + 0.23334524 |z|), with the polynomial q fitted
// here by linear programming to exp(z^2 / 2) Phi(-|z|) for |z| up to 14, so that the largest error relative to the value is least
// (7e-8; 4 units of 2^-23 when evaluated in 32 bits).  The tail is a product, nothing cancels in it.  erff made the epilogue of a
// product half as long again.
__device__ __forceinline__ float normal_cdf(float z, float& density) {
    const float t = __fdividef(1.0f, fmaf(0.23334524f, fabsf(z), 1.0f));
    density = __expf(-0.5f * z * z);
    float q = fmaf(t, -0.06745391f, 0.22915734f);
    q = fmaf(t, q, -0.17382519f);
    q = fmaf(t, q, 0.2025465f);
    q = fmaf(t, q, 0.024563838f);
    q = fmaf(t, q, 0.10030637f);
    q = fmaf(t, q, 0.091529734f);
    q = fmaf(t, q, 0.09317533f);
    q *= t * density;
    return z < 0.0f ? q : 1.0f - q;
}
__device__ __forceinline__ float act_value(float z, int act) {
    if (act == kActSilu) return __fdividef(z, 1.0f + __expf(-z));
    if (act == kActGelu) {
        float density;
        return z * normal_cdf(z, density);
    }
    if (act == kActRelu) return z > 0.0f || z != z ? z : 0.0f;
    return z;
}
// The same of several at once: one branch for all of them, so that they are worked on side by side.
template <int N>
__device__ __forceinline__ void act_values(float* z, int act) {
    if (act == kActSilu) {
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] = act_value(z[i], kActSilu);
    } else if (act == kActGelu) {
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] = act_value(z[i], kActGelu);
    } else if (act == kActRelu) {
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] = act_value(z[i], kActRelu);
    }
}
// The value and the derivative.
__device__ __forceinline__ void act_both(float z, int act, float& value, float& slope) {
    if (act == kActSilu) {
        const float p = __fdividef(1.0f, 1.0f + __expf(-z));
        value = z * p;
        slope = p * (1.0f + z * (1.0f - p));
    } else if (act == kActGelu) {
        float density;
        const float c = normal_cdf(z, density);
        value = z * c;
        slope = c + z * density * 0.39894228f;
    } else if (act == kActRelu) {
        value = z > 0.0f || z != z ? z : 0.0f;
        slope = z > 0.0f ? 1.0f : 0.0f;
    } else {
        value = z;
        slope = 1.0f;
    }
}

// Of eight at once, one branch for all of them.
__device__ __forceinline__ void act_both8(const float* z, int act, float* value, float* slope) {
    if (act == kActSilu) {
#pragma unroll
        for (int i = 0; i < 8; ++i) act_both(z[i], kActSilu, value[i], slope[i]);
    } else if (act == kActGelu) {
#pragma unroll
        for (int i = 0; i < 8; ++i) act_both(z[i], kActGelu, value[i], slope[i]);
    } else if (act == kActRelu) {
#pragma unroll
        for (int i = 0; i < 8; ++i) act_both(z[i], kActRelu, value[i], slope[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) act_both(z[i], kActNone, value[i], slope[i]);
    }
}

__device__ __forceinline__ void unpack8(const uint4 in, float* f) {
    const uint32_t w[4] = {in.x, in.y, in.z, in.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(w[i] << 16);
        f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ uint4 pack8(const float* f) {
    return make_uint4(pack2(f[0], f[1]), pack2(f[2], f[3]), pack2(f[4], f[5]), pack2(f[6], f[7]));
}

// The experts' segments.  Whatever the arrays hold, a segment lies inside its region.
struct Segments {
    const int32_t *offset, *count;
    int E, L, cap;   // experts, experts per region, rows per region
};
__device__ __forceinline__ void segment(const Segments& s, int e, int& first, int& rows) {
    first = min(max(ld_plain(s.offset + e), 0), s.cap);
    rows = min(max(ld_plain(s.count + e), 0), s.cap - first);
    first += e / s.L * s.cap;
}

// Tiles of one expert: `rows` rows cut into equal pieces of at most `most`, the pieces whole multiples of `unit` rows.
__device__ __forceinline__ int row_tiles(int rows, int most) { return (rows + most - 1) / most; }

// Walks the experts' tiles in order, 32 experts at a time; every lane of a converged warp takes part.  Tile numbers only grow.
struct TileWalk {
    int base, before;          // first expert of the window, tiles in front of it
    int first, rows, upto;     // this lane's expert: its segment, tiles of the window up to and with it
    __device__ __forceinline__ void load(const Segments& s, int per_row_tile, int most, bool every) {
        const int lane = threadIdx.x & 31, e = base + lane;
        first = rows = 0;
        int n = 0;
        if (e < s.E) {
            segment(s, e, first, rows);
            n = every ? per_row_tile : row_tiles(rows, most) * per_row_tile;
        }
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int u = __shfl_up_sync(0xffffffffu, n, o);
            if (lane >= o) n += u;
        }
        upto = n;
    }
    // Tile t: its expert, segment and place among the expert's tiles; false behind the last one.
    __device__ __forceinline__ bool find(const Segments& s, int per_row_tile, int most, bool every, int t, int& e, int& seg_first,
                                         int& seg_rows, int& place) {
        for (;;) {
            const int all = __shfl_sync(0xffffffffu, upto, 31);
            if (t < before + all) break;
            before += all;
            base += 32;
            if (base >= s.E) return false;
            load(s, per_row_tile, most, every);
        }
        const int src = __ffs(__ballot_sync(0xffffffffu, t < before + upto)) - 1;
        const int in_front = __shfl_sync(0xffffffffu, upto, max(src - 1, 0));
        e = base + src;
        seg_first = __shfl_sync(0xffffffffu, first, src);
        seg_rows = __shfl_sync(0xffffffffu, rows, src);
        place = t - before - (src ? in_front : 0);
        return true;
    }
};

}  // namespace ubep
