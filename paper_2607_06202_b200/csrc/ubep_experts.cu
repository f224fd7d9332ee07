// The experts' products on ragged segments of rows: the gated feed-forward block, the product with bias, activation, row
// weight and residual, and both backward passes.
//
//   forward   D^T[feature, row] = W[feature, :] . x[row, :]              W and x along the contraction
//   rows' gradient   D^T[feature, row] = sum_n W[n, feature] dz[row, n]  W across it
//   weights' gradient   D[n, feature] = sum_row dz[row, n] x[row, feature]   both across it, the rows being the contraction
//
// One persistent kernel, one CTA per SM: a thread loads operand tiles with tensor-map copies into a ring in shared memory, a thread
// issues tcgen05.mma, eight or sixteen warps turn sums in tensor memory into results.  The rows are the N dimension of the
// instruction, the features its M: a segment of 139 rows costs 144 (160 in pairs), where rows as M would cost 256, and sixteen rows of a
// decode step cost sixteen.
//   single CTAs (few rows per expert): two tiles of 128 features, one of up to 64 rows; 32 KB of weights per step of 64 of the
//     contraction.  Reading the weights bounds them: 32 experts of 7168 x 2048, 16 rows each, 270 - 282 us for 1.88 GB.
//   pairs (cta_group::2): 256 features x up to 256 rows, half of either brought by each CTA, two accumulators, so that the results
//     of one tile leave while the next is multiplied.  A step brings 32 KB per CTA for 512 cycles of the tensor cores, about what an SM
//     takes in from L2.  8 experts of 4096 x 2048, 1024 rows each: gated 176 - 189 us (1460 - 1560 TFLOP/s), tensor cores active 93 % of
//     the time, linear 96 - 99, the rows' gradient 99 - 104, the weights' 99 - 104; one cuBLAS product of the same rows 93 - 95.
#include <cstdint>
#include <atomic>

#include "../../include/ubep.h"
#include "ubep_experts.cuh"
#include "ubep_launch.cuh"
#include "ubep_tensor.cuh"

#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "ubep_experts.h"

namespace ubep {

namespace {

enum { kGated = 0, kLinear = 1, kRowsGrad = 2, kWeightsGrad = 3, kGatedScaled = 4 };
__host__ __device__ constexpr bool gated(int mode) { return mode == kGated || mode == kGatedScaled; }   // kGatedScaled: rows of an FP8 dispatch

// A warpgroup with a loading warp, a multiplying warp and (weights' gradient in pairs) one that mends the last rows; the others turn
// sums into results: in groups of four warps, which share the tile's columns.
constexpr int kFirstResult = 4;
__host__ __device__ constexpr int result_groups(int mode, int cg) { return mode == kLinear || (mode == kGatedScaled && cg == 2) ? 4 : 2; }
__host__ __device__ constexpr int gemm_threads(int mode, int cg) { return 32 * (kFirstResult + 4 * result_groups(mode, cg)); }
constexpr int kStepK = 64;               // of the contraction per stage: 128 bytes of bf16, the swizzle's width
constexpr int kHalfBytes = 128 * 128;    // 128 features of one stage
constexpr int kMaxRing = 8;
constexpr int kColumns = 512;            // tensor memory: all of it (one CTA per SM)
// Finished results go through shared memory, so that whole lines are written.  Rows: tiles of 16 rows per column group, two of them
// in turn, or one beside those of the saved products; weights' gradient: a tile of 32 x 64 per warp, one tensor copy each.
constexpr int kWide = 272;               // bytes per row of 128 results (16 to spread the banks), 16 rows per tile, 8 of them
constexpr int kNarrow = 160;             // ... of 64 (the gated block in pairs): two neighbouring rows in different banks
constexpr int kBlockBytes = 32 * 128;
__host__ __device__ constexpr int tile_bytes(int mode, int cg) {
    return mode == kWeightsGrad ? 4 * kBlockBytes : gated(mode) ? (cg == 1 ? 8 * kWide : 16 * kNarrow) : 16 * kWide;
}

struct Product {
    Segments seg;
    int F;           // features (of the gated block: inner features)
    int K;           // contraction (weights' gradient: the segment's rows instead)
    int FB;          // weights' gradient: features of x
    int most;        // rows per tile at most; columns of one accumulator
    int stages, stage_bytes, accs;
    int tiles;       // of results per column group
    int span;        // features per tile: 128 per CTA, or 256 for a single one (gated block: 128 of each matrix, 64 in pairs)
    int act;
    uint16_t *out, *pre;
    const uint16_t *bias, *residual;
    const float *row_scale, *x_scale;
    int planes;      // weights' gradient: 2 = x is the sum of two bf16 arrays
    int32_t* status;
};

struct Shared {
    uint64_t full[kMaxRing], empty[kMaxRing], ends[kMaxRing], cleared[kMaxRing], acc_full[2], acc_empty[2], drained;
    uint32_t tmem;
    int abort;
};

// Waits of a whole warp; all lanes agree on the outcome.  CG = 2: for what the other CTA of the pair may have done.
template <int CG>
__device__ __forceinline__ bool warp_wait(uint64_t* bar, unsigned parity, Shared* sh, int32_t* status) {
    bool ok;
    if constexpr (CG == 1) {
        ok = mbar_wait_idle(bar, parity, &sh->abort);
    } else {
        ok = mbar_try_wait_pair(bar, parity, 1000u);
        if (!ok) {
            const unsigned long long t_end = global_ns() + kWaitLimitNs;
            while (!(ok = mbar_try_wait_pair(bar, parity, 1000u)))
                if (*(volatile int*)&sh->abort || global_ns() > t_end) break;
        }
    }
    if (__all_sync(0xffffffffu, ok)) return true;
    if ((threadIdx.x & 31) == 0) {
        *(volatile int*)&sh->abort = 1;
        if (status) report(status, kErrTimeout);
    }
    return false;
}

// The same of one thread.
template <int CG>
__device__ __forceinline__ bool thread_wait(uint64_t* bar, unsigned parity, Shared* sh, int32_t* status) {
    if (CG == 1 ? mbar_try_wait(bar, parity, 1000u) : mbar_try_wait_pair(bar, parity, 1000u)) return true;
    const unsigned long long t_end = global_ns() + kWaitLimitNs;
    while (!(CG == 1 ? mbar_try_wait(bar, parity, 1000u) : mbar_try_wait_pair(bar, parity, 1000u)))
        if (*(volatile int*)&sh->abort || global_ns() > t_end) {
            *(volatile int*)&sh->abort = 1;
            if (status) report(status, kErrTimeout);
            return false;
        }
    return true;
}

// Place of a tile: expert, rows and features.
struct Tile {
    int e, row, rows, f0, fb0;   // global row of its first row, its rows, first feature, weights' gradient: first feature of x
};

template <int MODE, int CG>
struct Walk {
    TileWalk w;
    const Product& p;
    int per_row_tile, fb_tiles;
    static constexpr bool kEvery = MODE == kWeightsGrad;
    static constexpr int kUnit = 16 * CG;
    __device__ __forceinline__ explicit Walk(const Product& p_) : p(p_) {
        fb_tiles = kEvery ? (p.FB + 255) / 256 : 1;
        per_row_tile = (p.F + p.span - 1) / p.span * fb_tiles;
        w.base = w.before = 0;
        w.load(p.seg, per_row_tile, p.most, kEvery);
    }
    __device__ __forceinline__ bool find(int t, Tile& o) {
        int first, rows, place;
        if (!w.find(p.seg, per_row_tile, p.most, kEvery, t, o.e, first, rows, place)) return false;
        if (kEvery) {
            // (neighbours share the tile of the first operand)
            o.f0 = place / fb_tiles * p.span;
            o.fb0 = place % fb_tiles * 256;
            o.row = first;
            o.rows = rows;
        } else {
            // (neighbours share the tile of the weights, which comes from memory once)
            const int n = row_tiles(rows, p.most);
            const int piece = ((rows + n - 1) / n + kUnit - 1) / kUnit * kUnit;
            const int i = place % n;
            o.f0 = place / n * p.span;
            o.fb0 = 0;
            o.row = first + i * piece;
            o.rows = min(piece, rows - i * piece);
        }
        return true;
    }
};

// Rows left .. of a stage of the weights' gradient, up to the next multiple of 16: behind the segment there is another expert's
// row, or nobody's, and whatever it holds must not be multiplied.  Blocks of 64 rows x 128 bytes.
__device__ __forceinline__ void clear_rows(uint8_t* stage, int blocks, int left, int lane) {
    const int end = (left + 15) / 16 * 16;   // (the instructions take 16 rows each)
    for (int r = left; r < end; ++r)
        for (int v = lane; v < blocks * 8; v += 32)
            *reinterpret_cast<uint4*>(stage + (v >> 3) * 8192 + r * 128 + (v & 7) * 16) = make_uint4(0, 0, 0, 0);
    fence_proxy_async_smem();
    __syncwarp();
}

__device__ __forceinline__ void put_bf16(uint8_t* at, float v) { *reinterpret_cast<__nv_bfloat16*>(at) = __float2bfloat16_rn(v); }
__device__ __forceinline__ uint4 ld_vec(const uint16_t* p);
// What the linear product's epilogue reads besides the sums, fetched two chunks of 16 rows ahead: the bias of the thread's features,
// the rows' weights (lane l: row l of the chunk) and the thread's 16-byte pieces of the residual, rows and columns as they are
// written out.
template <bool USED, int HALVES, int GROUPS>
struct Extras {
    float bias[2], scale, scale1;
    uint4 rows[2], rows1[2];
    int h, c, start, vec, vec_row, lane;
    __device__ __forceinline__ void fetch(const Product& p, const Tile& t, int rank, uint4* to, float& s) {
        const int f = t.f0 + (h + rank) * 128 + vec;
        const bool in = h < HALVES && (h == 0 || p.span == 256) && f < p.F;
        if (p.residual) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int r = c + vec_row + i * 8;
                to[i] = in && r < t.rows ? ld_vec(p.residual + (int64_t)(t.row + r) * p.F + f) : make_uint4(0, 0, 0, 0);
            }
        }
        if (p.row_scale) s = lane < 16 && c + lane < t.rows ? ld_plain(p.row_scale + t.row + c + lane) : 0.0f;
        c += GROUPS * 16;
        if (c >= t.rows) {
            c = start;
            ++h;
        }
    }
    __device__ __forceinline__ void begin(const Product& p, const Tile& t, int rank, int group, int lane_) {
        if constexpr (!USED) return;
        const int me = threadIdx.x - kFirstResult * 32 - group * 128;
        lane = lane_;
        h = 0;
        c = start = group * 16;
        vec = me % 16 * 8;
        vec_row = me / 16;
#pragma unroll
        for (int i = 0; i < HALVES; ++i) {
            const int f = t.f0 + (i + rank) * 128 + (me >> 5) % 4 * 32 + lane;
            bias[i] = p.bias && f < p.F ? __uint_as_float((uint32_t)ld_plain(p.bias + (int64_t)t.e * p.F + f) << 16) : 0.0f;
        }
        fetch(p, t, rank, rows, scale);
        fetch(p, t, rank, rows1, scale1);
    }
    __device__ __forceinline__ void next(const Product& p, const Tile& t, int rank) {
        scale = scale1;
        rows[0] = rows1[0];
        rows[1] = rows1[1];
        fetch(p, t, rank, rows1, scale1);
    }
};

__device__ __forceinline__ uint4 ld_vec(const uint16_t* p) { return *reinterpret_cast<const uint4*>(p); }
__device__ __forceinline__ void st_vec(uint16_t* p, uint4 v) { *reinterpret_cast<uint4*>(p) = v; }

template <int MODE, int CG>
__global__ void __launch_bounds__(gemm_threads(MODE, CG), 1) expert_kernel(const __grid_constant__ CUtensorMap map_a,
                                                                          const __grid_constant__ CUtensorMap map_b,
                                                                          const __grid_constant__ CUtensorMap map_c, const Product p) {
    extern __shared__ uint8_t dynamic[];
    __shared__ Shared sh;
    constexpr int kHalves = CG == 1 ? 2 : 1;                              // tiles of 128 features that this CTA multiplies with one tile of rows
    constexpr bool kAcross = MODE == kRowsGrad || MODE == kWeightsGrad;   // the features' operand
    constexpr bool kMends = MODE == kWeightsGrad;
    constexpr bool kScaled = MODE == kGatedScaled;
    constexpr int kGroups = result_groups(MODE, CG), kTile = tile_bytes(MODE, CG);
    // Rows with scales, in pairs: a tile's sums are kept in the result warps' registers, which get some of the others'.
    constexpr bool kRowsFirst = kScaled && CG == 2, kSplits = kGroups == 4;
    // 640 threads x 96 = 61440: 128 x 48 + 512 x 104 = 59392, 128 x 32 + 512 x 112 = 61440
    constexpr int kFewRegisters = kRowsFirst ? 32 : 48, kManyRegisters = kRowsFirst ? 112 : 104;
    uint8_t* ring = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(dynamic) + 1023) & ~(uintptr_t)1023);
    uint8_t* results = ring + (size_t)p.stages * p.stage_bytes;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = CG == 1 ? 0 : (int)pair_rank();
    if (threadIdx.x == 0) {
        for (int i = 0; i < p.stages; ++i) {
            mbar_init(&sh.full[i], 1);
            mbar_init(&sh.empty[i], 1);
        }
        for (int i = 0; i < kMaxRing; ++i) {
            mbar_init(&sh.ends[i], 1);
            mbar_init(&sh.cleared[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&sh.acc_full[i], 1);
            mbar_init(&sh.acc_empty[i], 4 * kGroups * CG);
        }
        mbar_init(&sh.drained, 1);
        sh.abort = 0;
        mbar_fence_init();
    }
    if (warp == 1) {
        if (lane == 0) {
            map_prefetch(&map_a);
            map_prefetch(&map_b);
            map_prefetch(&map_c);
        }
        __syncwarp();
        tmem_alloc<CG>(&sh.tmem, kColumns);
    }
    tc_fence_before();
    __syncwarp();
    if constexpr (CG == 1) __syncthreads();
    else pair_sync();
    tc_fence_after();
    const uint32_t tmem = *(volatile uint32_t*)&sh.tmem;
    griddep_wait();
    griddep_launch();   // (the next kernel's set-up, where it fits beside this one)
    const int unit = blockIdx.x / CG, units = gridDim.x / CG;
    Walk<MODE, CG> walk(p);
    Tile t;
    if (warp >= kFirstResult) {
        // ------------------------------------------------------------------ results
        if constexpr (kSplits) registers_up<kManyRegisters>();
        const int quarter = warp & 3, group = (warp - kFirstResult) >> 2;   // lanes of tensor memory this warp may read; which columns
        uint8_t* tiles = results + (MODE == kWeightsGrad ? (warp - kFirstResult) * kBlockBytes : group * p.tiles * kTile);
        int acc = 0, flip = 0;
        unsigned acc_phase = 0;
        for (int id = unit; walk.find(id, t); id += units) {
            const bool empty = MODE == kWeightsGrad && t.rows == 0;
            Extras<MODE == kLinear, kHalves, kGroups> extras;   // under way while the products are
            extras.begin(p, t, rank, group, lane);
            if constexpr (kRowsFirst) {
                // Rows with scales, in a pair: the rows are the lanes of tensor memory, so that a row's scale is one register of the thread
                // that adds up its sums -- as columns every sum would need another scale, and those loads alone took as long as the
                // products.  (The rows are half a pair's tile, the columns sixteens of gate and up of eight features.)  8 experts of 4096 x
                // 2048, 1024 rows each: 211 us and 19 for widening the rows, bf16 rows 179 - 185; the tensor cores are active 71 % of the
                // time (bf16 rows 93 %), the rest is the hand-over per 128 channels.  112 registers are 24 bytes short of what it
                // holds: some 120 bytes spill (0.3 % of its instructions).
                const int half = (t.rows + 31) / 32 * 16, r = rank * half + quarter * 32 + lane, groups = p.K / 128;
                const bool mine = quarter * 32 + lane < half && r < t.rows;
                const int64_t row = t.row + r;
                const float* from = p.x_scale + row * groups;
                float sum[64];
#pragma unroll
                for (int i = 0; i < 64; ++i) sum[i] = 0.0f;
                float next = mine ? ld_plain(from) : 0.0f;
                bool ok = true;
                for (int g = 0; g < groups; ++g) {
                    const float2 scale = make_float2(next, next);
                    if (mine && g + 1 < groups) next = ld_plain(from + g + 1);
                    ok = warp_wait<CG>(&sh.acc_full[acc], acc_phase, &sh, p.status);
                    if (!ok) break;
                    tc_fence_after();
                    const uint32_t d = tmem + ((uint32_t)(quarter * 32) << 16) + acc * 256 + group * 64;
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        float v[32];
                        tmem_ld32(d + h * 32, v);
                        if (h == 1) {   // all of them have been read: the products may go on
                            tc_fence_before();
                            __syncwarp();
                            if (lane == 0) mbar_arrive_pair_relaxed(first_of_pair(&sh.acc_empty[acc]));
                        }
#pragma unroll
                        for (int i = 0; i < 32; i += 2) fma_two(sum + h * 32 + i, v + i, scale);
                    }
                    if (++acc == p.accs) {
                        acc = 0;
                        acc_phase ^= 1;
                    }
                }
                if (group_or(1 + group, 128, !ok)) break;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int f = t.f0 + group * 32 + i * 8;
                    if (f >= p.F || !mine) continue;
                    float *g = sum + i * 16, *u = g + 8;
                    if (p.pre) {
                        st_vec(p.pre + row * 2 * p.F + f, pack8(g));
                        st_vec(p.pre + (row * 2 + 1) * p.F + f, pack8(u));
                    }
                    act_values<8>(g, p.act);
#pragma unroll
                    for (int j = 0; j < 8; ++j) g[j] *= u[j];
                    st_vec(p.out + row * p.F + f, pack8(g));
                }
                continue;
            } else if constexpr (kScaled) {
                // Rows with scales: the sum over every 128 channels is multiplied with the row's scale of them and added up here, in
                // 32 bits -- the e4m3 values are bf16 exactly, their products with the scales would be rounded once more.
                float sum[4][16];
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 16; ++j) sum[i][j] = 0.0f;
                group_sync(1 + group, 128);   // (the last tile's results have left the room)
                float* scales = reinterpret_cast<float*>(tiles);
                const int me = threadIdx.x - kFirstResult * 32 - group * 128, groups = p.K / 128;
                const int mine = (me / 8 * 2 + group) * 8 + me % 8;   // the row whose scales this thread fetches
                const bool fetches = me < 32 && mine < t.rows;
                const float* from = p.x_scale + (int64_t)(t.row + mine) * groups;
                float next = fetches ? ld_plain(from) : 0.0f;
                bool ok = true;
                for (int g = 0; g < groups; ++g) {
                    float* here = scales + (g & 1) * 32;
                    if (me < 32) here[me] = next;
                    if (fetches && g + 1 < groups) next = ld_plain(from + g + 1);
                    ok = warp_wait<CG>(&sh.acc_full[acc], acc_phase, &sh, p.status);
                    ok = !group_or(1 + group, 128, !ok);   // (also: all scales are there)
                    if (!ok) break;
                    tc_fence_after();
                    const uint32_t d = tmem + ((uint32_t)(quarter * 32) << 16) + acc * kHalves * p.most;
                    const bool done = g == groups - 1;
#pragma unroll
                    for (int i0 = 0; i0 < 4; i0 += 2) {   // (two pieces' columns are there whether rows use them or not)
                        const int c = (2 * i0 + group) * 8;
                        float v[2][16];
                        if (c < t.rows) tmem_ld_pieces(d + c, d + p.most + c, v);
                        if (i0 == 2 && !done) {   // all of them have been read: the products may go on
                            tc_fence_before();
                            __syncwarp();
                            if (lane == 0) mbar_arrive(&sh.acc_empty[acc]);
                        }
                        if (c >= t.rows) continue;
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const float2 s = *reinterpret_cast<const float2*>(here + (i0 + i) * 8 + 2 * (lane & 3));
#pragma unroll
                            for (int q = 0; q < 16; q += 2) fma_two(sum[i0 + i] + q, v[i] + q, s);
                        }
                    }
                    if (done) {   // the whole sums take the place of the last group's
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int c = (2 * i + group) * 8;
                            if (c < t.rows) tmem_st_piece(d + c, d + p.most + c, sum[i]);
                        }
                    } else if (++acc == p.accs) {
                        acc = 0;
                        acc_phase ^= 1;
                    }
                }
                if (!ok) break;
                group_sync(1 + group, 128);   // (the scales' room is the results')
            } else if (!empty) {
                const bool ok = warp_wait<CG>(&sh.acc_full[acc], acc_phase, &sh, p.status);
                // (warps that meet at barriers below leave together)
                if (MODE == kWeightsGrad ? !ok : group_or(1 + group, 128, !ok)) break;
                tc_fence_after();
            }
            const uint32_t d = tmem + ((uint32_t)(quarter * 32) << 16) + acc * kHalves * p.most;
            bool held = !empty;   // the accumulator is given back once its last columns have been read
            auto give_back = [&](bool when) {
                if (!held || !when) return;
                held = false;
                tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    if constexpr (CG == 1) mbar_arrive(&sh.acc_empty[acc]);
                    else mbar_arrive_pair_relaxed(first_of_pair(&sh.acc_empty[acc]));
                }
            };
            if constexpr (MODE == kWeightsGrad) {
                for (int h = 0; h < kHalves; ++h) {
                    const int f = t.f0 + (h + rank) * 128 + quarter * 32;
                    for (int c = group * 128; c < group * 128 + 128; c += 64) {
                        if (f >= p.F || t.fb0 + c >= p.FB) break;
                        float v[64];
                        if (empty) {
#pragma unroll
                            for (int j = 0; j < 64; ++j) v[j] = 0.0f;
                        } else {
                            tmem_ld64(d + h * p.most + c, v);
                        }
                        give_back(c == group * 128 + 64 && (h == kHalves - 1 || f + 128 >= p.F));
                        if (lane == 0) bulk_wait_read<0>();   // (the tile's last copy has read it)
                        __syncwarp();
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            // (16-byte pieces in the order of the 128-byte swizzle: conflict-free)
                            *reinterpret_cast<uint4*>(tiles + lane * 128 + ((i ^ (lane & 7)) << 4)) = pack8(v + i * 8);
                        fence_proxy_async_smem();
                        __syncwarp();
                        if (lane == 0) {
                            tile_store(&map_c, t.fb0 + c, f, t.e, smem_u32(tiles));
                            bulk_commit();
                        }
                    }
                }
            } else {
                // one CTA and the gated block: gate and up of a feature in the same lane, in two accumulators, eight rows at a time; a
                // pair: eight lanes gate, the next eight lanes up of the same features, so that a lane finishes every second row
                constexpr int kRows = gated(MODE) && CG == 1 ? 8 : 16;
                constexpr int kWidth = gated(MODE) && CG == 2 ? 64 : 128, kPitch = kWidth == 64 ? kNarrow : kWide;
                constexpr int kVecs = kWidth / 8, kPasses = kRows * kVecs / 128;
                const int me = threadIdx.x - kFirstResult * 32 - group * 128;   // thread of the column group
                const int halves = gated(MODE) || p.span == 128 ? 1 : kHalves;
                for (int h = 0; h < halves; ++h) {
                    const int f0 = t.f0 + (gated(MODE) ? rank * kWidth : (h + rank) * 128);
                    if (f0 >= p.F) break;
                    const int col = gated(MODE) && CG == 2 ? quarter * 16 + (lane >> 4) * 8 + (lane & 7) : quarter * 32 + lane;
                    // whole rows' pieces, 16 bytes per thread: rows and features of this thread's vectors
                    const int vec_f = f0 + me % kVecs * 8, vec_row = me / kVecs;
                    const bool vec_in = vec_f < p.F;
                    auto put_out = [&](uint16_t* to, int64_t pitch, const uint8_t* from, int c) {
#pragma unroll
                        for (int i = 0; i < kPasses; ++i) {
                            const int r = vec_row + i * (128 / kVecs);
                            if (vec_in && c + r < t.rows)
                                st_vec(to + (t.row + c + r) * pitch + vec_f, *reinterpret_cast<const uint4*>(from + r * kPitch + me % kVecs * 16));
                        }
                    };
                    const float bias = MODE != kLinear ? 0.0f : h == 0 ? extras.bias[0] : extras.bias[1];
                    for (int c = group * kRows; c < t.rows; c += kGroups * kRows) {
                        const bool last = c + kGroups * kRows >= t.rows && (h == halves - 1 || f0 + 128 >= p.F);
                        uint8_t* tile = tiles + flip * kTile;
                        float v[16];
                        if constexpr (gated(MODE) && CG == 1) tmem_ld8x2(d + c, d + p.most + c, v, v + 8);
                        else tmem_ld16(d + h * p.most + c, v);
                        give_back(last);
                        if constexpr (gated(MODE)) {
                            float g[8], u[8];
                            const bool up = lane & 8;
#pragma unroll
                            for (int i = 0; i < 8; ++i) {
                                if constexpr (CG == 1) {
                                    g[i] = v[i];
                                    u[i] = v[8 + i];
                                } else {
                                    const float other = __shfl_xor_sync(0xffffffffu, up ? v[2 * i] : v[2 * i + 1], 8);
                                    g[i] = up ? other : v[2 * i];
                                    u[i] = up ? v[2 * i + 1] : other;
                                }
                            }
                            uint8_t* at = tile + (CG == 1 ? 0 : up * kPitch) + col * 2;
                            constexpr int kStep = (CG == 1 ? 1 : 2) * kPitch;
                            if (p.pre) {
#pragma unroll
                                for (int i = 0; i < 8; ++i) {
                                    put_bf16(at + i * kStep + kTile, g[i]);
                                    put_bf16(at + i * kStep + 2 * kTile, u[i]);
                                }
                            }
                            act_values<8>(g, p.act);
#pragma unroll
                            for (int i = 0; i < 8; ++i) put_bf16(at + i * kStep, g[i] * u[i]);
                        } else {
                            uint8_t* at = tile + col * 2;
                            if constexpr (MODE == kLinear) {
#pragma unroll
                                for (int i = 0; i < 16; ++i) v[i] += bias;
                                if (p.pre) {
#pragma unroll
                                    for (int i = 0; i < 16; ++i) put_bf16(at + i * kPitch + kTile, v[i]);
                                }
                                act_values<16>(v, p.act);
                                if (p.row_scale) {
#pragma unroll
                                    for (int i = 0; i < 16; ++i) v[i] *= __shfl_sync(0xffffffffu, extras.scale, i);
                                }
                                if (p.residual) {
                                    // through the tile, where every thread finds the values of its own feature
#pragma unroll
                                    for (int i = 0; i < kPasses; ++i)
                                        *reinterpret_cast<uint4*>(tile + (vec_row + i * (128 / kVecs)) * kPitch + me % kVecs * 16) = extras.rows[i];
                                    group_sync(1 + group, 128);
#pragma unroll
                                    for (int i = 0; i < 16; ++i)
                                        v[i] += __uint_as_float((uint32_t) * reinterpret_cast<const uint16_t*>(at + i * kPitch) << 16);
                                }
                                extras.next(p, t, rank);
                            }
#pragma unroll
                            for (int i = 0; i < 16; ++i) put_bf16(at + i * kPitch, v[i]);
                        }
                        group_sync(1 + group, 128);
                        put_out(p.out, p.F, tile, c);
                        if (p.pre) {
                            put_out(p.pre, gated(MODE) ? 2 * p.F : p.F, tile + kTile, c);
                            if (gated(MODE)) put_out(p.pre + p.F, 2 * p.F, tile + 2 * kTile, c);
                        }
                        // (with two tiles in turn the other one's readers have met at a barrier since)
                        if (p.pre || p.tiles == 1) group_sync(1 + group, 128);
                        else flip ^= 1;
                    }
                }
            }
            give_back(true);
            if (!empty && ++acc == p.accs) {
                acc = 0;
                acc_phase ^= 1;
            }
        }
        if constexpr (MODE == kWeightsGrad) bulk_wait_all<0>();
    } else {
    if constexpr (kSplits) registers_down<kFewRegisters>();
    // The loads and the products are each one thread's loop: with the whole warp in it (votes and elections in every step) a product's
    // step took 60 cycles longer, of 512.
    const bool lead = elect_one();
    const uint32_t ring0 = smem_u32(ring);
    const uint32_t a_bytes = kHalves == 2 && !gated(MODE) && p.span == 128 ? kHalfBytes : kHalves * kHalfBytes;
    if (warp == 0) {
        // ------------------------------------------------------------------ loads
        int s = 0, used = 0, ends = 0;
        unsigned phase = 0;
        bool ok = true;
        auto next_stage = [&] {
            ++used;
            if (++s == p.stages) {
                s = 0;
                phase ^= 1;
            }
        };
        for (int id = unit; ok && walk.find(id, t); id += units) {
            const int K = MODE == kWeightsGrad ? t.rows : p.K;
            const bool two = kHalves == 2 && (gated(MODE) || (p.span == 256 && t.f0 + 128 < p.F));
            const int f0 = t.f0 + rank * (gated(MODE) ? 64 : 128), fb0 = t.fb0 + rank * 128;
            // (in a pair each CTA brings one half of the rows, or of x's features)
            const int mine = CG == 1 ? t.rows : (t.rows + 31) / 32 * 16, row0 = t.row + rank * mine;
            // (boxes of 64 and of 16 rows: a copy costs the loading thread some 55 cycles, eight copies of 16 rows nearly the whole step)
            const int small = MODE == kWeightsGrad ? 0 : (mine + 15) / 16 % 4, large = MODE == kWeightsGrad ? 4 / CG : (mine + 15) / 64;
            const unsigned bytes = (two ? 2 : 1) * kHalfBytes + large * 8192 + small * 2048;
            if (lead) {
                for (int plane = 0; ok && plane < (MODE == kWeightsGrad ? p.planes : 1); ++plane)
                    for (int k0 = 0; k0 < K; k0 += kStepK) {
                        ok = thread_wait<CG>(&sh.empty[s], phase ^ 1, &sh, p.status);
                        if (!ok) break;
                        const uint32_t a = ring0 + s * p.stage_bytes, b = a + a_bytes;
                        uint32_t bar = CG == 1 ? smem_u32(&sh.full[s]) : first_of_pair(&sh.full[s]);
                        if (kMends && K - k0 < kStepK) {   // each CTA counts its own last rows, which have to be mended
                            uint64_t* end = &sh.ends[ends++ % kMaxRing];
                            bar = smem_u32(end);
                            mbar_arrive_expect_tx(end, bytes);
                        } else if (rank == 0) {
                            mbar_arrive_expect_tx(&sh.full[s], CG * bytes);
                        }
                        if constexpr (gated(MODE) && CG == 1) {
                            tile_load<CG>(a, &map_a, k0, f0, 2 * t.e, bar);
                            tile_load<CG>(a + kHalfBytes, &map_a, k0, f0, 2 * t.e + 1, bar);
                        } else if constexpr (gated(MODE)) {
                            tile_load5_pair(a, &map_a, k0, 0, 0, f0 / 8, t.e, bar);
                        } else if constexpr (MODE == kLinear) {
                            tile_load<CG>(a, &map_a, k0, f0, t.e, bar);
                            if (two) tile_load<CG>(a + kHalfBytes, &map_a, k0, f0 + 128, t.e, bar);
                        } else {
                            const int y = MODE == kRowsGrad ? k0 : t.row + k0, z = MODE == kRowsGrad ? t.e : 0;
                            tile_load<CG>(a, &map_a, f0, y, z, bar);
                            tile_load<CG>(a + 8192, &map_a, f0 + 64, y, z, bar);
                            if (two) {
                                tile_load<CG>(a + 16384, &map_a, f0 + 128, y, z, bar);
                                tile_load<CG>(a + 24576, &map_a, f0 + 192, y, z, bar);
                            }
                        }
                        if constexpr (MODE == kWeightsGrad) {
#pragma unroll
                            for (int j = 0; j < 4 / CG; ++j) tile_load<CG>(b + j * 8192, &map_b, fb0 + 64 * j, t.row + k0, plane, bar);
                        } else {
                            for (int j = 0; j < large; ++j) tile_load<CG>(b + j * 8192, &map_b, k0, row0 + j * 64, 0, bar);
                            for (int j = 0; j < small; ++j)
                                tile_load<CG>(b + large * 8192 + j * 2048, &map_c, k0, row0 + large * 64 + j * 16, 0, bar);
                        }
                        next_stage();
                    }
            }
            ok = __all_sync(0xffffffffu, ok);
        }
        if (lead) {
            if (CG == 2 && ok)   // the products' last arrivals come to this CTA's barriers: it may not leave before them
                for (int i = 0; ok && i < p.stages && i < used; ++i) {
                    s = s ? s - 1 : p.stages - 1;
                    if (s == p.stages - 1) phase ^= 1;
                    ok = thread_wait<CG>(&sh.empty[s], phase, &sh, p.status);
                }
            else if (!ok && rank == 0)
                // nothing may still be on its way into shared memory when the CTA leaves: the last copy of every stage (a pair leaves
                // together, and the first CTA's barriers count for both)
                for (int i = 0; i < p.stages && i < used; ++i) {
                    s = s ? s - 1 : p.stages - 1;
                    if (s == p.stages - 1) phase ^= 1;
                    mbar_wait(&sh.full[s], phase, nullptr);
                }
        }
        __syncwarp();
    } else if (warp == 1) {
        // ------------------------------------------------------------------ products
        int s = 0, acc = 0;
        unsigned phase = 0, acc_phase = 0;
        bool ok = true;
        // (the first stage's operands; the address is the low end of a descriptor, and all of shared memory fits there)
        const uint64_t a0 = kAcross ? operand(ring0, 8192, 1024) : operand(ring0, 16, 1024);
        const uint64_t b0 = MODE == kWeightsGrad ? operand(ring0 + a_bytes, 8192, 1024) : operand(ring0 + a_bytes, 16, 1024);
        constexpr int kPartA = (kAcross ? 2048 : 32) >> 4, kPartB = (MODE == kWeightsGrad ? 2048 : 32) >> 4;   // 16 of the contraction
        for (int id = unit; rank == 0 && ok && walk.find(id, t); id += units) {
            const int K = MODE == kWeightsGrad ? t.rows : p.K;
            const bool two = kHalves == 2 && (gated(MODE) || (p.span == 256 && t.f0 + 128 < p.F));
            const int n = MODE == kWeightsGrad || kRowsFirst ? 256 : (t.rows + 16 * CG - 1) / (16 * CG) * (16 * CG);
            const uint32_t idesc = instruction(128 * CG, n, kAcross, MODE == kWeightsGrad);
            if (lead && K > 0) {
                uint32_t d = 0;
                bool add = false;
                // rows with scales: every group of 128 channels is a sum of its own, two steps
                auto open = [&] {
                    ok = thread_wait<CG>(&sh.acc_empty[acc], acc_phase ^ 1, &sh, p.status);
                    tc_fence_after();
                    d = tmem + acc * kHalves * p.most;
                    add = false;
                };
                auto close = [&] {
                    mma_commit<CG>(&sh.acc_full[acc]);
                    if (++acc == p.accs) {
                        acc = 0;
                        acc_phase ^= 1;
                    }
                };
                auto part = [&](uint64_t da, uint64_t db) {
                    if (kRowsFirst) mma_f16<CG>(d, db, da, idesc, add);
                    else mma_f16<CG>(d, da, db, idesc, add);
                    if (two) mma_f16<CG>(d + p.most, da + (kHalfBytes >> 4), db, idesc, add);
                    add = true;
                };
                if (!kScaled) open();
                for (int plane = 0; ok && plane < (MODE == kWeightsGrad ? p.planes : 1); ++plane)
                    for (int left = K; left > 0; left -= kStepK) {
                        if (kScaled && (left & 64) == 0) open();   // (the contraction is a multiple of 128)
                        if (kScaled && !ok) break;
                        ok = thread_wait<CG>(&sh.full[s], phase, &sh, p.status);
                        if (!ok) break;
                        tc_fence_after();
                        const uint64_t da = a0 + (uint32_t)(s * p.stage_bytes >> 4), db = b0 + (uint32_t)(s * p.stage_bytes >> 4);
                        if (left >= kStepK) {
#pragma unroll
                            for (int j = 0; j < 4; ++j) part(da + j * kPartA, db + j * kPartB);
                        } else {
                            for (int j = 0; j * 16 < left; ++j) part(da + j * kPartA, db + j * kPartB);
                        }
                        mma_commit<CG>(&sh.empty[s]);
                        if (kScaled && (left & 64) != 0) close();
                        if (++s == p.stages) {
                            s = 0;
                            phase ^= 1;
                        }
                    }
                if (!kScaled && ok) close();
            }
            ok = __all_sync(0xffffffffu, ok);
        }
        if (!ok) {   // no product may still be running when the tensor memory is given back
            if (lead) mma_commit<CG>(&sh.drained);
            __syncwarp();
            mbar_wait(&sh.drained, 0, nullptr);
        }
    } else if (kMends && warp == 2) {
        // ------------------------------------------------------------------ last rows of a segment in the weights' gradient
        // Each CTA clears what is behind them in its own operands; of a pair the second tells the first, and the first completes the
        // stage that its products wait for.  (Done for every step, the arrival at the other CTA alone took more than twice a step's time.)
        int s = 0, ends = 0;
        bool ok = true;
        for (int id = unit; ok && walk.find(id, t); id += units) {
            const int left = t.rows % kStepK;
            for (int plane = 0; ok && plane < p.planes; ++plane) {
                s += t.rows / kStepK;
                if (!left) continue;
                const int at = s++ % p.stages, end = ends % kMaxRing;
                const unsigned phase = ends++ / kMaxRing & 1;
                ok = warp_wait<CG>(&sh.ends[end], phase, &sh, p.status);
                if (!ok) break;
                clear_rows(ring + (size_t)at * p.stage_bytes, kHalves * 2 + 4 / CG, left, lane);
                if (CG == 2 && rank == 0) ok = warp_wait<CG>(&sh.cleared[end], phase, &sh, p.status);
                if (!ok) break;
                if (lane == 0) {
                    if (rank == 0) mbar_arrive(&sh.full[at]);
                    else mbar_arrive_pair(first_of_pair(&sh.cleared[end]));
                }
            }
            s %= p.stages;
        }
    }
    }
    tc_fence_before();
    __syncwarp();
    if constexpr (CG == 1) __syncthreads();
    else pair_sync();
    tc_fence_after();
    if (warp == 1) tmem_free<CG>(tmem, kColumns);
}

// ------------------------------------------------------------------------------------------ passes over the rows

constexpr int kRowThreads = 256;

// Rows quantised by an FP8 dispatch as bf16.  Forward: the e4m3 values alone, which bf16 holds exactly (their scales are applied to the
// sums).  Weights' gradient, whose sum runs over rows with different scales: value times scale as the sum of two bf16 numbers,
// the second in the second half of the scratch (off by 2^-17 of the value; one bf16 would be off by 2^-9).  A warp per row, eight
// channels per lane: 8-byte loads, 16-byte stores, six of each on their way.
constexpr int kWidenAhead = 6;
template <bool SPLIT>
__global__ void __launch_bounds__(kRowThreads) widen_kernel(const uint8_t* q, const float* scale, uint16_t* out, int64_t plane, int H,
                                                           Segments seg) {
    griddep_wait();
    const int lane = threadIdx.x & 31, warps = kRowThreads / 32;
    int first, rows;
    for (int e = blockIdx.y; e < seg.E; e += gridDim.y) {
        segment(seg, e, first, rows);
        for (int r = blockIdx.x * warps + (threadIdx.x >> 5); r < rows; r += gridDim.x * warps) {
            const int64_t row = first + r;
            const uint8_t* from = q + row * H;
            for (int c0 = lane * 8; c0 < H; c0 += 256 * kWidenAhead) {
                uint2 in[kWidenAhead];
                float s[kWidenAhead];
#pragma unroll
                for (int i = 0; i < kWidenAhead; ++i) {
                    const int c = c0 + i * 256;
                    if (c < H) {
                        in[i] = *reinterpret_cast<const uint2*>(from + c);
                        if (SPLIT) s[i] = ld_plain(scale + row * (H / 128) + c / 128);
                    }
                }
#pragma unroll
                for (int i = 0; i < kWidenAhead; ++i) {
                    const int c = c0 + i * 256;
                    if (c >= H) break;
                    float f[8];
                    const uint32_t w[2] = {in[i].x, in[i].y};
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w[j >> 1] >> (16 * (j & 1))), __NV_E4M3);
                        const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&h));
                        f[2 * j] = SPLIT ? v.x * s[i] : v.x;
                        f[2 * j + 1] = SPLIT ? v.y * s[i] : v.y;
                    }
                    const uint4 high = pack8(f);
                    st_vec(out + row * H + c, high);
                    if (SPLIT) {
                        float back[8];
                        unpack8(high, back);
#pragma unroll
                        for (int j = 0; j < 8; ++j) f[j] -= back[j];
                        st_vec(out + plane + row * H + c, pack8(f));
                    }
                }
            }
        }
    }
}

// dg = dh u act'(g), du = dh act(g); pre and grad_pre may be the same array.
__global__ void __launch_bounds__(kRowThreads) gated_grad_kernel(const uint16_t* grad, const uint16_t* pre, uint16_t* grad_pre, int I,
                                                                int act, Segments seg) {
    griddep_wait();
    int first, rows;
    for (int e = blockIdx.y; e < seg.E; e += gridDim.y) {
        segment(seg, e, first, rows);
        for (int r = blockIdx.x; r < rows; r += gridDim.x) {
            const int64_t row = first + r;
            for (int c = threadIdx.x * 8; c < I; c += kRowThreads * 8) {
                float dh[8], g[8], u[8], value[8], slope[8];
                unpack8(ld_vec(grad + row * I + c), dh);
                unpack8(ld_vec(pre + row * 2 * I + c), g);
                unpack8(ld_vec(pre + (row * 2 + 1) * I + c), u);
                act_both8(g, act, value, slope);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    g[i] = dh[i] * u[i] * slope[i];
                    u[i] = dh[i] * value[i];
                }
                st_vec(grad_pre + row * 2 * I + c, pack8(g));
                st_vec(grad_pre + (row * 2 + 1) * I + c, pack8(u));
            }
        }
    }
}

// What the linear product's gradients need of every row, in one pass: dz = scale grad act'(z) as bf16 (grad_pre), the row
// weight's gradient <grad, act(z)> (grad_scale) and, of dz as it is before it is rounded, the sums over the rows (partial); each or
// none.  A block takes one of gridDim.x slices of an expert's rows and up to 256 * 8 * P columns, whose sums its threads keep in
// registers; bias_grad_kernel joins the slices in order.
// 24000 rows of 4096, floor 91 us: 155; as two kernels, one by rows and one by columns, 344.
constexpr int kSumRows = 8;   // rows whose sums across the block are joined together
template <int P>
__global__ void __launch_bounds__(kRowThreads) linear_grad_kernel(const uint16_t* grad, const uint16_t* pre, const float* row_scale,
                                                                 uint16_t* grad_pre, float* grad_scale, float* partial, int N, int act,
                                                                 Segments seg) {
    __shared__ float part[kSumRows][kRowThreads / 32];
    griddep_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, col0 = blockIdx.z * (P * kRowThreads * 8) + threadIdx.x * 8;
    int first, rows;
    for (int e = blockIdx.y; e < seg.E; e += gridDim.y) {
        segment(seg, e, first, rows);
        const int r0 = (int)((int64_t)rows * blockIdx.x / gridDim.x), r1 = (int)((int64_t)rows * (blockIdx.x + 1) / gridDim.x);
        float sums[P][8];
#pragma unroll
        for (int q = 0; q < P; ++q)
#pragma unroll
            for (int i = 0; i < 8; ++i) sums[q][i] = 0.0f;
        for (int r = r0; r < r1; r += kSumRows) {
            const int n = min(kSumRows, r1 - r);
            for (int j = 0; j < n; ++j) {
                const int64_t row = first + r + j;
                const float scale = row_scale ? ld_plain(row_scale + row) : 1.0f;
                uint4 in[P], at[P];
#pragma unroll
                for (int q = 0; q < P; ++q) {
                    const int c = col0 + q * (kRowThreads * 8);
                    in[q] = at[q] = make_uint4(0, 0, 0, 0);
                    if (c < N) {
                        in[q] = ld_vec(grad + row * N + c);
                        if (pre) at[q] = ld_vec(pre + row * N + c);
                    }
                }
                float dot = 0.0f;
#pragma unroll
                for (int q = 0; q < P; ++q) {
                    const int c = col0 + q * (kRowThreads * 8);
                    if (c >= N) break;
                    float dy[8], z[8], value[8], slope[8];
                    unpack8(in[q], dy);
                    unpack8(at[q], z);
                    act_both8(z, act, value, slope);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        dot += dy[i] * value[i];
                        dy[i] *= slope[i] * scale;
                        sums[q][i] += dy[i];
                    }
                    if (grad_pre) st_vec(grad_pre + row * N + c, pack8(dy));
                }
                if (!grad_scale) continue;
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, o);
                if (lane == 0) part[j][warp] = dot;
            }
            if (!grad_scale) continue;
            __syncthreads();
            if (threadIdx.x < n) {
                float all = 0.0f;
#pragma unroll
                for (int w = 0; w < kRowThreads / 32; ++w) all += part[threadIdx.x][w];
                grad_scale[first + r + threadIdx.x] = all;
            }
            __syncthreads();
        }
        if (!partial) continue;
#pragma unroll
        for (int q = 0; q < P; ++q) {
            const int c = col0 + q * (kRowThreads * 8);
            if (c >= N) break;
            float4* to = reinterpret_cast<float4*>(partial + ((int64_t)e * gridDim.x + blockIdx.x) * N + c);
            to[0] = make_float4(sums[q][0], sums[q][1], sums[q][2], sums[q][3]);
            to[1] = make_float4(sums[q][4], sums[q][5], sums[q][6], sums[q][7]);
        }
    }
}

// The slices' sums, joined in order and rounded.
__global__ void __launch_bounds__(kRowThreads) bias_grad_kernel(const float* partial, uint16_t* grad_bias, int slices, int N, int E) {
    griddep_wait();
    const int c = blockIdx.x * kRowThreads + threadIdx.x;
    if (c >= N) return;
    for (int e = blockIdx.y; e < E; e += gridDim.y) {
        float all = 0.0f;
        for (int i = 0; i < slices; ++i) all += ld_plain(partial + ((int64_t)e * slices + i) * N + c);
        const __nv_bfloat16 v = __float2bfloat16_rn(all);
        grad_bias[(int64_t)e * N + c] = *reinterpret_cast<const uint16_t*>(&v);
    }
}

// ------------------------------------------------------------------------------------------ host

typedef CUresult (*EncodeFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                             const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeFn encoder() {
    static std::atomic<void*> fn{nullptr};
    void* f = fn.load(std::memory_order_acquire);
    if (!f) {
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found) != cudaSuccess ||
            found != cudaDriverEntryPointSuccess)
            return nullptr;
        fn.store(f, std::memory_order_release);
    }
    return reinterpret_cast<EncodeFn>(f);
}

// Weights of the gated block for pairs, [E, 2, I, H] with I in eights: the box is 64 features' halves, eight rows of the gate's
// matrix and eight of the other's in turn, so that both products of a feature end up in the same warp's lanes.
bool make_gated_map(CUtensorMap* map, const void* base, uint64_t H, uint64_t I, uint64_t E) {
    const EncodeFn encode = encoder();
    if (!encode) return false;
    const cuuint64_t dims[5] = {H, 8, 2, I / 8, E}, strides[4] = {H * 2, I * H * 2, 8 * H * 2, 2 * I * H * 2};
    const cuuint32_t box[5] = {64, 8, 2, 8, 1}, steps[5] = {1, 1, 1, 1, 1};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, const_cast<void*>(base), dims, strides, box, steps,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// bf16 [planes, rows, cols], boxes of `box_rows` x 64, 128-byte swizzle; what lies outside reads as zero.
bool make_map(CUtensorMap* map, const void* base, uint64_t cols, uint64_t rows, uint64_t planes, unsigned box_rows) {
    const EncodeFn encode = encoder();
    if (!encode) return false;
    const cuuint64_t dims[3] = {cols, rows, planes}, strides[2] = {cols * 2, cols * rows * 2};
    const cuuint32_t box[3] = {64, box_rows, 1}, steps[3] = {1, 1, 1};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, steps,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

struct DeviceFacts {
    int sms = 0, smem = 0;
};
cudaError_t device_facts(DeviceFacts* f) {
    static std::atomic<uint64_t> known[kAttrDevices];   // what a device is does not change: SMs and shared memory, packed
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const uint64_t v = dev < kAttrDevices ? known[dev].load(std::memory_order_relaxed) : 0;
    if (v) {
        f->sms = (int)(v >> 32);
        f->smem = (int)(v & 0xffffffffu);
        return cudaSuccess;
    }
    e = cudaDeviceGetAttribute(&f->sms, cudaDevAttrMultiProcessorCount, dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&f->smem, cudaDevAttrMaxSharedMemoryPerBlockOptin, dev);
    if (e == cudaSuccess && dev < kAttrDevices) known[dev].store(((uint64_t)f->sms << 32) | (uint32_t)f->smem, std::memory_order_relaxed);
    return e;
}

template <int MODE, int CG>
cudaError_t launch_product(const CUtensorMap& a, const CUtensorMap& b, const CUtensorMap& c, Product p, cudaStream_t st) {
    DeviceFacts dev;
    cudaError_t e = device_facts(&dev);
    if (e != cudaSuccess) return e;
    constexpr int kHalves = CG == 1 ? 2 : 1;
    p.span = gated(MODE) ? 128 : 256;
    // Single CTAs: narrow tiles where there is an SM for each of them (one tile of rows per expert).  Narrow against wide, 4096 x 2048 and
    // 2048 x 2048 weights, 16 rows each, linear (the rows' gradient alike): 4 experts (64 narrow tiles) 19.0 and 23.5 us, 8 of 2048 x 2048
    // (128) 15.1 and 16.3; with more of them than SMs a few get two, as long as a wide one: 10 experts (160) 43.6 and 37.0, 12 of 2048 x 2048
    // (192) 24.9 and 21.4, 16 (256) 26.7 and 25.8, 32 (512) 48.6 and 45.1, 32 of 2048 x 7168 (1792) 146 and 143.
    if (CG == 1 && (MODE == kLinear || MODE == kRowsGrad) && (int64_t)p.seg.E * ((p.F + 127) / 128) <= dev.sms) p.span = 128;
    p.stage_bytes = (p.span == 128 && !gated(MODE) ? 1 : kHalves) * kHalfBytes + p.most / CG * 128;
    p.accs = 2 * kHalves * p.most <= kColumns ? 2 : 1;
    // a tile of results per column group, and one for each array of saved products (the gated block in pairs has room for two in turn)
    p.tiles = p.pre ? (gated(MODE) ? 3 : 2) : gated(MODE) ? 2 : 1;
    const int tiles = result_groups(MODE, CG) * (MODE == kWeightsGrad ? 1 : p.tiles) * tile_bytes(MODE, CG);
    const int room = dev.smem - 1024 - (int)sizeof(Shared) - tiles;
    p.stages = room / p.stage_bytes;
    if (p.stages > kMaxRing) p.stages = kMaxRing;
    if (p.stages < 2) return cudaErrorInvalidConfiguration;
    const int smem = p.stages * p.stage_bytes + tiles + 1024;
    static std::atomic<int> granted[kAttrDevices];
    e = allow_dynamic_smem(reinterpret_cast<const void*>(expert_kernel<MODE, CG>), smem, granted);
    if (e != cudaSuccess) return e;
    return launch_overlapped(expert_kernel<MODE, CG>, dev.sms / CG * CG, gemm_threads(MODE, CG), (size_t)smem, st, false, CG, a, b, c, p);
}

// The segments of a call are not known to the host, their capacity is.
int64_t rows_each(const ubep_expert_rows_t& r) { return (int64_t)r.num_ranks * r.rows_per_rank_cap / r.num_experts; }
// Pairs of CTAs where there are rows enough to multiply; single CTAs, with more of the weights under way, where reading those is all
// there is to do.  Single against pairs, 32 experts of 4096 x 2048, rows each: gated 64: 172 and 176 us, 96: 195 and 182, 128: 202 and
// 186; linear 64: 90 and 92, 96: 144 and 96; FP8 rows 32: 181 and 231, 64: 191 and 238, 128: 266 and 261; weights' gradient 32: 104 and 112,
// 64: 98 and 110, 96: 124 and 132, 128: 142 and 113; the rows' gradient 32: 88.7 and 85.9, 96: 132 and 95.
bool in_pairs(const ubep_expert_rows_t& r) { return rows_each(r) > 64; }
// Rows per tile.  Small pieces leave room for more stages and a second accumulator.
int rows_per_tile(const ubep_expert_rows_t& r) { return in_pairs(r) ? 256 : 64; }

uint64_t all_rows(const ubep_expert_rows_t& r) { return (uint64_t)r.num_ranks * r.rows_per_rank_cap; }
// Rows of all regions, [R * cap, width], in boxes of 64 and of 16 rows.
bool make_rows_maps(CUtensorMap* large, CUtensorMap* small, const void* rows, int width, const ubep_expert_rows_t& r) {
    return make_map(large, rows, width, all_rows(r), 1, 64) && make_map(small, rows, width, all_rows(r), 1, 16);
}

dim3 row_grid(const ubep_expert_rows_t& r, const DeviceFacts& dev) {
    const int per = (dev.sms * 16 + r.num_experts - 1) / r.num_experts;
    return dim3((unsigned)(per < r.rows_per_rank_cap ? per : r.rows_per_rank_cap), (unsigned)(r.num_experts < 65535 ? r.num_experts : 65535));
}

Segments segments_of(const ubep_expert_rows_t& r) {
    return Segments{r.offset, r.count, r.num_experts, r.num_experts / r.num_ranks, r.rows_per_rank_cap};
}

// FP8 rows as bf16 in the scratch.
template <bool SPLIT>
cudaError_t widen(const ubep_expert_rows_t& r, const void* x, const float* x_scale, void* scratch, int H, cudaStream_t st, int* launches) {
    DeviceFacts dev;
    cudaError_t e = device_facts(&dev);
    if (e != cudaSuccess) return e;
    dim3 grid = row_grid(r, dev);
    grid.x = (grid.x + kRowThreads / 32 - 1) / (kRowThreads / 32);
    ++*launches;
    return launch_overlapped(widen_kernel<SPLIT>, grid, kRowThreads, 0, st, false, 1, static_cast<const uint8_t*>(x), x_scale,
                             static_cast<uint16_t*>(scratch), (int64_t)all_rows(r) * H, H, segments_of(r));
}

// dx[row, k] = sum_n dz[row, n] w[e, n, k]
cudaError_t rows_grad(const ubep_expert_rows_t& r, const void* dz, const void* w, int K, int N, void* grad_x, cudaStream_t st) {
    Product p{};
    p.seg = segments_of(r);
    p.F = K;
    p.K = N;
    p.most = rows_per_tile(r);
    p.out = static_cast<uint16_t*>(grad_x);
    p.status = r.status;
    CUtensorMap a, b, c;
    const bool pairs = in_pairs(r);
    if (!make_map(&a, w, K, N, r.num_experts, 64) || !make_rows_maps(&b, &c, dz, N, r)) return cudaErrorInvalidValue;
    return pairs ? launch_product<kRowsGrad, 2>(a, b, c, p, st) : launch_product<kRowsGrad, 1>(a, b, c, p, st);
}

// dw[e, n, k] = sum_row dz[row, n] x[row, k]
cudaError_t weights_grad(const ubep_expert_rows_t& r, const void* dz, const void* x, int planes, int K, int N, void* grad_w,
                         cudaStream_t st) {
    Product p{};
    p.seg = segments_of(r);
    p.F = N;
    p.FB = K;
    p.most = 256;
    p.planes = planes;
    p.out = static_cast<uint16_t*>(grad_w);
    p.status = r.status;
    CUtensorMap a, b, out;
    if (!make_map(&a, dz, N, all_rows(r), 1, 64) || !make_map(&b, x, K, all_rows(r), planes, 64) || !make_map(&out, grad_w, K, N, r.num_experts, 32))
        return cudaErrorInvalidValue;
    return in_pairs(r) ? launch_product<kWeightsGrad, 2>(a, b, out, p, st) : launch_product<kWeightsGrad, 1>(a, b, out, p, st);
}

}  // namespace

cudaError_t launch_expert_gated(const ubep_expert_rows_t& r, const void* x, const float* x_scale, const void* w, int H, int I, int act,
                                void* h, void* pre, void* scratch, cudaStream_t st, int* launches) {
    const void* rows = x_scale ? scratch : x;
    cudaError_t e = x_scale ? widen<false>(r, x, x_scale, scratch, H, st, launches) : cudaSuccess;
    if (e != cudaSuccess) return e;
    Product p{};
    p.x_scale = x_scale;
    p.seg = segments_of(r);
    p.F = I;
    p.K = H;
    p.most = rows_per_tile(r);
    p.act = act;
    p.out = static_cast<uint16_t*>(h);
    p.pre = static_cast<uint16_t*>(pre);
    p.status = r.status;
    CUtensorMap a, b, c;
    const bool pairs = in_pairs(r);
    if (!(pairs ? make_gated_map(&a, w, H, I, r.num_experts) : make_map(&a, w, H, I, 2 * (uint64_t)r.num_experts, 128)) ||
        !make_rows_maps(&b, &c, rows, H, r))
        return cudaErrorInvalidValue;
    if (x_scale)
        e = pairs ? launch_product<kGatedScaled, 2>(a, b, c, p, st) : launch_product<kGatedScaled, 1>(a, b, c, p, st);
    else
        e = pairs ? launch_product<kGated, 2>(a, b, c, p, st) : launch_product<kGated, 1>(a, b, c, p, st);
    if (e == cudaSuccess) ++*launches;
    return e;
}

cudaError_t launch_expert_gated_backward(const ubep_expert_rows_t& r, const void* x, const float* x_scale, const void* w, const void* pre,
                                         const void* grad_h, int H, int I, int act, void* grad_pre, void* grad_x, void* grad_w,
                                         void* scratch, cudaStream_t st, int* launches) {
    cudaError_t e = grad_w && x_scale ? widen<true>(r, x, x_scale, scratch, H, st, launches) : cudaSuccess;
    if (e != cudaSuccess) return e;
    DeviceFacts dev;
    e = device_facts(&dev);
    if (e != cudaSuccess) return e;
    gated_grad_kernel<<<row_grid(r, dev), kRowThreads, 0, st>>>(static_cast<const uint16_t*>(grad_h), static_cast<const uint16_t*>(pre),
                                                               static_cast<uint16_t*>(grad_pre), I, act, segments_of(r));
    e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    ++*launches;
    if (grad_x) {
        e = rows_grad(r, grad_pre, w, H, 2 * I, grad_x, st);
        if (e != cudaSuccess) return e;
        ++*launches;
    }
    if (grad_w) {
        e = weights_grad(r, grad_pre, x_scale ? scratch : x, x_scale ? 2 : 1, H, 2 * I, grad_w, st);
        if (e != cudaSuccess) return e;
        ++*launches;
    }
    return cudaSuccess;
}

cudaError_t launch_expert_linear(const ubep_expert_rows_t& r, const void* x, const void* w, const void* bias, const float* row_scale,
                                 const void* residual, int K, int N, int act, void* y, void* pre, cudaStream_t st, int* launches) {
    Product p{};
    p.seg = segments_of(r);
    p.F = N;
    p.K = K;
    p.most = rows_per_tile(r);
    p.act = act;
    p.out = static_cast<uint16_t*>(y);
    p.pre = static_cast<uint16_t*>(pre);
    p.bias = static_cast<const uint16_t*>(bias);
    p.residual = static_cast<const uint16_t*>(residual);
    p.row_scale = row_scale;
    p.status = r.status;
    CUtensorMap a, b, c;
    const bool pairs = in_pairs(r);
    if (!make_map(&a, w, K, N, r.num_experts, 128) || !make_rows_maps(&b, &c, x, K, r)) return cudaErrorInvalidValue;
    const cudaError_t e = pairs ? launch_product<kLinear, 2>(a, b, c, p, st) : launch_product<kLinear, 1>(a, b, c, p, st);
    if (e == cudaSuccess) ++*launches;
    return e;
}

cudaError_t launch_expert_linear_backward(const ubep_expert_rows_t& r, const void* x, const void* w, const void* pre,
                                          const float* row_scale, const void* grad_y, int K, int N, int act, void* grad_pre,
                                          void* grad_x, void* grad_w, void* grad_bias, float* grad_scale, float* scratch,
                                          cudaStream_t st, int* launches) {
    cudaError_t e = cudaSuccess;
    const void* dz = grad_y;
    const bool changes = act || row_scale;
    if (changes || grad_bias) {
        // slices of each expert's rows: a thousand blocks in all, as many partial sums as the scratch has room for
        const int slices = r.num_experts < UBEP_EXPERT_PARTIALS ? UBEP_EXPERT_PARTIALS / r.num_experts : 1;
        dim3 grid((unsigned)slices, (unsigned)(r.num_experts < 65535 ? r.num_experts : 65535));
        const bool dots = grad_scale != nullptr;
        const int vecs = (N / 8 + kRowThreads - 1) / kRowThreads;
        // (a row weight's gradient is a sum over the whole row, so one block has to see all of it; without one the columns may be split)
        if (vecs > 4 && !dots) grid.z = (unsigned)((vecs + 3) / 4);
        auto go = [&](auto kern) {
            return launch_overlapped(kern, grid, kRowThreads, 0, st, false, 1, static_cast<const uint16_t*>(grad_y),
                                     changes ? static_cast<const uint16_t*>(pre) : (const uint16_t*)nullptr, row_scale,
                                     changes && (grad_x || grad_w) ? static_cast<uint16_t*>(grad_pre) : (uint16_t*)nullptr, grad_scale,
                                     grad_bias ? scratch : (float*)nullptr, N, act, segments_of(r));
        };
        e = vecs <= 1 ? go(linear_grad_kernel<1>) : vecs <= 2 ? go(linear_grad_kernel<2>) : vecs <= 4 || !dots ? go(linear_grad_kernel<4>) :
            vecs <= 8 ? go(linear_grad_kernel<8>) : cudaErrorInvalidValue;
        if (e != cudaSuccess) return e;
        ++*launches;
        if (changes) dz = grad_pre;
        if (grad_bias) {
            const dim3 joins((unsigned)((N + kRowThreads - 1) / kRowThreads), grid.y);
            e = launch_overlapped(bias_grad_kernel, joins, kRowThreads, 0, st, false, 1, (const float*)scratch,
                                  static_cast<uint16_t*>(grad_bias), slices, N, r.num_experts);
            if (e != cudaSuccess) return e;
            ++*launches;
        }
    }
    if (grad_x) {
        e = rows_grad(r, dz, w, K, N, grad_x, st);
        if (e != cudaSuccess) return e;
        ++*launches;
    }
    if (grad_w) {
        e = weights_grad(r, dz, x, 1, K, N, grad_w, st);
        if (e != cudaSuccess) return e;
        ++*launches;
    }
    return cudaSuccess;
}

}  // namespace ubep
