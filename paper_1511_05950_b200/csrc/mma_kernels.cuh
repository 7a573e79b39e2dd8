// Matrix products on the fifth-generation tensor cores: D = A B^T tile by tile, a persistent kernel of CTA pairs.
//
// A pair of CTAs takes a tile of 256 x 256 (tcgen05.mma, cta_group::2): each holds 128 rows of A and 128 of B for every 64 steps of the contraction,
// in a ring of stages that one thread a CTA fills with TMA loads (128-byte swizzle), and 128 rows of the sums in its tensor memory,
// twice, so that the epilogue of one tile runs under the products of the next.  Warps: 0 loads, 1 issues the products (of the pair's first CTA), 2 owns
// the tensor memory, 4 to 11 are the epilogue (a warp reaches the 32 lanes of its number modulo 4; two warps share them, half the columns each).
//
// Either operand may lie with its contraction dimension contiguous (rows of A, "K-major") or with its other one (A given as its transpose,
// "MN-major"): the loads bring blocks of 64 x 64 as they lie, and the descriptors tell the tensor cores.
//
// Waits are bounded.  One that runs out makes the rest of what its CTA writes NaN; it waits for nothing after that, apart from copies in flight (with the same limit).
#pragma once

#include "units.cuh"

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math_constants.h>
#include <stdint.h>

namespace softsync {

constexpr int kTile = 256, kHalf = 128, kStep = 64;          // tile, rows of an operand in a CTA, contraction steps of a stage
constexpr int kStages = 6;
constexpr int kStageBytes = 2 * kHalf * kStep * 2;
constexpr int kMmaThreads = 384, kEpilogueWarp = 4, kEpilogueWarps = 8;
constexpr int kMmaShared = kStages * kStageBytes + 1024;      // the ring, aligned to the swizzle's 1024 bytes
constexpr int kMmaWaitLimit = 1 << 20;                         // polls of up to a microsecond

// ---- instructions ------------------------------------------------------------------------------------------------------
__device__ __forceinline__ unsigned mma_smem(const void *p) { return static_cast<unsigned>(__cvta_generic_to_shared(p)); }
__device__ __forceinline__ unsigned pair_rank()
{
    unsigned r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ unsigned leaders(unsigned addr)    // the same place in the pair's first CTA
{
    unsigned r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(addr));
    return r;
}
__device__ __forceinline__ void pair_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void bar_init(unsigned bar, unsigned count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" :: "r"(bar), "r"(count) : "memory"); }
__device__ __forceinline__ void bar_expect(unsigned bar, unsigned bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" :: "r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void bar_arrive_leader(unsigned bar)
{
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" :: "r"(leaders(bar)) : "memory");
}
__device__ __forceinline__ bool bar_wait(unsigned bar, unsigned parity)
{
    for (int tries = 0; tries < kMmaWaitLimit; ++tries) {
        unsigned ok;
        asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2, %3;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                     : "=r"(ok) : "r"(bar), "r"(parity), "r"(1000u) : "memory");
        if (ok) return true;
    }
    return false;
}
__device__ __forceinline__ void tile_load(unsigned dst, const CUtensorMap *map, int x, int y, unsigned leader_bar)
{
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 :: "r"(dst), "l"(map), "r"(x), "r"(y), "r"(leader_bar) : "memory");
}
__device__ __forceinline__ void mma_pair(unsigned d, uint64_t a, uint64_t b, unsigned idesc, unsigned accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 :: "r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void commit_pair(unsigned bar)      // arrives at both CTAs' barrier once the products issued so far are done
{
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 :: "r"(bar), "h"(static_cast<uint16_t>(3)) : "memory");
}
__device__ __forceinline__ void tmem_load32(unsigned addr, float (&v)[32])
{
    unsigned *r = reinterpret_cast<unsigned *>(v);
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]),
                   "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]),
                   "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
                 : "r"(addr) : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ float mma_ex2(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// Shared-memory descriptors, 128-byte swizzle.  K-major: rows of 128 bytes, groups of eight 1024 apart; 16 contraction steps are 32 bytes on.
// MN-major: blocks of 64 x 64, a contraction step a row of 128 bytes, groups of eight steps 1024 apart (stride), blocks 8192 apart
// (leading); 16 steps are 2048 bytes on.
template <bool MN> __device__ __forceinline__ uint64_t operand_descriptor(unsigned addr)
{
    constexpr uint64_t leading = MN ? 8192 >> 4 : 1, stride = 1024 >> 4;
    return (static_cast<uint64_t>(addr) >> 4 & 0x3fff) | leading << 16 | stride << 32 | uint64_t{1} << 46 | uint64_t{2} << 61;
}
template <bool MN> constexpr int kDescriptorStep = MN ? 2048 >> 4 : 32 >> 4;
// bf16 operands, fp32 sums, 256 x 256
template <bool MN_A, bool MN_B>
constexpr unsigned kInstruction = 1u << 4 | 1u << 7 | 1u << 10 | (MN_A ? 1u << 15 : 0u) | (MN_B ? 1u << 16 : 0u) | (kTile / 8u) << 17 | (kTile / 16u) << 24;

// ---- what a product is -------------------------------------------------------------------------------------------------
struct MmaPlan {
    int m, n, k;                          // extents; where `live` is given it replaces m (live_is_k 0) or k (1)
    const int *live;
    int live_is_k;
    int splits;                           // parts that the contraction is split into, each with sums of its own
    int group;                            // row tiles whose turns come before the next column tile's
};

struct TileAt { int m, n, split, first, steps; };            // tile indices, split, and its stages of the contraction

struct TileWalk {
    int tiles_m, tiles_n, all_steps, splits, group;
    long long count;
    __device__ __forceinline__ TileWalk(const MmaPlan &p)
    {
        const int live = p.live ? *p.live : 0, m = p.live && !p.live_is_k ? live : p.m, k = p.live && p.live_is_k ? live : p.k;
        tiles_m = (m + kTile - 1) / kTile;
        tiles_n = (p.n + kTile - 1) / kTile;
        all_steps = (k + kStep - 1) / kStep;
        splits = p.splits;
        group = p.group;
        count = static_cast<long long>(tiles_m) * tiles_n * splits;
    }
    __device__ __forceinline__ TileAt at(long long t) const
    {
        TileAt r;
        const long long tiles = static_cast<long long>(tiles_m) * tiles_n;
        r.split = static_cast<int>(t / tiles);
        const long long in = t - r.split * tiles;
        const long long band = static_cast<long long>(group) * tiles_n;
        const int b = static_cast<int>(in / band), high = min(group, tiles_m - b * group);
        const int at = static_cast<int>(in - b * band);
        r.n = at / high;
        r.m = b * group + at % high;
        const int per = (all_steps + splits - 1) / splits;
        r.first = min(all_steps, r.split * per);
        r.steps = min(all_steps, r.first + per) - r.first;
        return r;
    }
};

// ---- epilogues: each is called by the 32 lanes of a warp, a row a lane, 32 columns at a time -----------------------------------
// Maximum and sum of exponentials of a row's 128 columns, and the token's product.
struct StatsEpilogue {
    const int *order;                     // the rows that take part, or null: all
    const long long *tokens;
    int rows, vocab;
    const int *live;
    float scale;                          // log2(e) / T
    float2 *parts;                        // [column half][row]: maximum of the products, sum of 2^(scale (x - maximum))
    long long part_stride;
    float *picked;                        // the token's product

    int row, tok;
    bool valid;
    float top, sum;
    __device__ __forceinline__ void begin(int r, int)
    {
        row = r;
        valid = r < (live ? *live : rows);
        const long long t = valid ? tokens[order ? order[r] : r] : -1;
        tok = t >= 0 && t < vocab ? static_cast<int>(t) : -1;
        top = -CUDART_INF_F;
        sum = 0.f;
    }
    __device__ __forceinline__ void take(float (&x)[32], int col)
    {
        if (col >= vocab) return;
        if (col + 32 > vocab) {
#pragma unroll
            for (int k = 0; k < 32; ++k) if (col + k >= vocab) x[k] = -CUDART_INF_F;
        }
        const unsigned at = static_cast<unsigned>(tok - col);
        if (__any_sync(kAllLanes, at < 32u)) {
            float z = 0.f;
#pragma unroll
            for (int k = 0; k < 32; ++k) z = at == static_cast<unsigned>(k) ? x[k] : z;
            if (at < 32u && valid) picked[row] = z;
        }
        float m = top;
#pragma unroll
        for (int k = 0; k < 32; ++k) m = fmaxf(m, x[k]);
        const float shift = m == -CUDART_INF_F ? 0.f : m * scale;
        float s[4] = {sum * mma_ex2(top * scale - shift), 0.f, 0.f, 0.f};
        if (top == -CUDART_INF_F) s[0] = 0.f;
#pragma unroll
        for (int k = 0; k < 32; ++k) s[k & 3] += mma_ex2(fmaf(x[k], scale, -shift));
        sum = (s[0] + s[1]) + (s[2] + s[3]);
        top = m;
    }
    __device__ __forceinline__ void end(int col, int)
    {
        if (valid && col < vocab) parts[static_cast<long long>(col / kHalf) * part_stride + row] = make_float2(top, sum);
    }
};

// G = a (p - 1[j = token]) of a piece of the vocabulary, rounded to bf16.
struct GradEpilogue {
    const int *order;
    const long long *tokens;
    const float *lse, *coef;              // of all rows; coef null: 1
    float sign;                           // of coef
    int rows, vocab;
    const int *live;
    float scale;
    int first, width;                     // the piece: columns [first, first + width)
    __nv_bfloat16 *g;
    long long g_stride;

    int row, tok, write;
    float a, shift;
    __device__ __forceinline__ void begin(int r, int)
    {
        const int n = live ? *live : rows;
        row = r;
        write = r < (n + kStep - 1) / kStep * kStep;        // rows up to a whole stage of the next product: zeros
        a = 0.f; shift = 0.f; tok = -1;
        if (r < n) {
            const int at = order ? order[r] : r;
            const long long t = tokens[at];
            tok = t >= first && t < first + width ? static_cast<int>(t - first) : -1;
            a = coef ? sign * coef[at] : 1.f;
            shift = lse[at] * 1.4426950408889634f;
        }
    }
    __device__ __forceinline__ void take(float (&x)[32], int col)
    {
        if (col >= width) return;
        const unsigned at = static_cast<unsigned>(tok - col);
        const bool picked = __any_sync(kAllLanes, at < 32u);
#pragma unroll
        for (int k = 0; k < 32; ++k) x[k] = mma_ex2(fmaf(x[k], scale, -shift));
        if (picked) {
#pragma unroll
            for (int k = 0; k < 32; ++k) x[k] -= at == static_cast<unsigned>(k) ? 1.f : 0.f;
        }
        if (!write) return;
        uint4 *to = reinterpret_cast<uint4 *>(g + row * g_stride + col);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            float *v = x + 8 * k;
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = a == 0.f ? 0.f : a * v[j];
            if (col + 8 * k < width)
                to[k] = make_uint4(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7]));
        }
    }
    __device__ __forceinline__ void end(int, int) {}
};

// The product itself: alpha D (times a gain for each column), or fp32 sums of a split for a later kernel.
struct StoreEpilogue {
    int rows, cols;
    float alpha;
    const float *alpha_dev;               // may be null
    const void *gain;                     // may be null
    int gain_bf16;
    void *out;                            // bf16 or fp32, or null: sums to `part`
    int out_bf16, vectors;
    long long stride;
    float *part;
    long long part_stride, part_rows;     // elements of a row, and of a split
    int add;                              // to what is there

    int row;
    float factor;
    float *to;
    __device__ __forceinline__ void begin(int r, int split)
    {
        row = r;
        factor = alpha_dev ? alpha * *alpha_dev : alpha;
        if (part) to = part + split * part_rows + r * part_stride;
    }
    __device__ __forceinline__ void take(float (&x)[32], int col)
    {
        if (row >= rows || col >= cols) return;
        if (!out) {                                       // padded to whole vectors
            float4 *p = reinterpret_cast<float4 *>(to + col);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                if (col + 4 * k >= part_stride) break;
                float4 v = make_float4(x[4 * k], x[4 * k + 1], x[4 * k + 2], x[4 * k + 3]);
                if (add) { const float4 o = p[k]; v.x += o.x; v.y += o.y; v.z += o.z; v.w += o.w; }
                p[k] = v;
            }
            return;
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int c = col + 8 * k, left = cols - c;
            if (left <= 0) break;
            const bool whole = vectors && left >= kUnit;
            Unit u;
#pragma unroll
            for (int j = 0; j < kUnit; ++j) u.v[j] = x[8 * k + j] * factor;
            if (gain) {
                const Unit w = load_gain(gain, gain_bf16, c, left, whole);
#pragma unroll
                for (int j = 0; j < kUnit; ++j) u.v[j] *= w.v[j];
            }
            if (out_bf16) store_unit(static_cast<__nv_bfloat16 *>(out) + row * stride + c, u, left, whole);
            else store_unit(static_cast<float *>(out) + row * stride + c, u, left, whole);
        }
    }
    __device__ __forceinline__ void end(int, int) {}
};

// ---- the kernel --------------------------------------------------------------------------------------------------------
template <typename Epilogue, bool MN_A, bool MN_B>
__global__ void __cluster_dims__(2) __launch_bounds__(kMmaThreads, 1) mma_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                                                              const __grid_constant__ MmaPlan plan, const __grid_constant__ Epilogue given)
{
    extern __shared__ unsigned char raw_ring[];
    __shared__ __align__(8) unsigned long long full[kStages], empty[kStages], ready[2], drained[2];
    __shared__ unsigned tmem_base;
    const unsigned ring = (mma_smem(raw_ring) + 1023u) & ~1023u;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const unsigned rank = pair_rank();
    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) { bar_init(mma_smem(&full[s]), 1); bar_init(mma_smem(&empty[s]), 1); }
        for (int b = 0; b < 2; ++b) { bar_init(mma_smem(&ready[b]), 1); bar_init(mma_smem(&drained[b]), 2 * kEpilogueWarps); }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 2) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" :: "r"(mma_smem(&tmem_base)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    pair_sync();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const unsigned tmem = tmem_base;
    const TileWalk walk(plan);
    const long long start = blockIdx.x >> 1, pairs = gridDim.x >> 1;

    if (warp == 0) {
        if (lane == 0) {
            unsigned turn = 0;                             // stages filled so far
            bool late = false;
            for (long long t = start; t < walk.count && !late; t += pairs) {
                const TileAt at = walk.at(t);
                const int ya = at.m * kTile + static_cast<int>(rank) * kHalf, yb = at.n * kTile + static_cast<int>(rank) * kHalf;
                for (int s = 0; s < at.steps; ++s, ++turn) {
                    const unsigned slot = turn % kStages, round = turn / kStages;
                    if (round && !bar_wait(mma_smem(&empty[slot]), (round - 1) & 1)) { late = true; break; }
                    const unsigned bar = leaders(mma_smem(&full[slot])), a = ring + slot * kStageBytes, b = a + kStageBytes / 2;
                    if (rank == 0) bar_expect(mma_smem(&full[slot]), 2 * kStageBytes);
                    const int x = (at.first + s) * kStep;
                    if constexpr (MN_A) { tile_load(a, &map_a, ya, x, bar); tile_load(a + 8192, &map_a, ya + 64, x, bar); }
                    else tile_load(a, &map_a, x, ya, bar);
                    if constexpr (MN_B) { tile_load(b, &map_b, yb, x, bar); tile_load(b + 8192, &map_b, yb + 64, x, bar); }
                    else tile_load(b, &map_b, x, yb, bar);
                }
            }
            // every copy has arrived, and every stage's release, before either CTA may leave
            for (unsigned k = turn > kStages ? turn - kStages : 0; k < turn; ++k) {
                late = late || !bar_wait(mma_smem(&empty[k % kStages]), (k / kStages) & 1);
                if (late && rank == 0) bar_wait(mma_smem(&full[k % kStages]), (k / kStages) & 1);
            }
        }
    } else if (warp == 1) {
        if (lane == 0 && rank == 0) {
            unsigned turn = 0, tile = 0;
            bool late = false;
            for (long long t = start; t < walk.count && !late; t += pairs) {
                const TileAt at = walk.at(t);
                if (!at.steps) continue;
                const unsigned buffer = tile & 1, use = tile >> 1;
                ++tile;
                if (use && !bar_wait(mma_smem(&drained[buffer]), (use - 1) & 1)) { late = true; break; }
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                for (int s = 0; s < at.steps; ++s, ++turn) {
                    const unsigned slot = turn % kStages;
                    if (!bar_wait(mma_smem(&full[slot]), (turn / kStages) & 1)) { late = true; break; }
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint64_t a = operand_descriptor<MN_A>(ring + slot * kStageBytes), b = operand_descriptor<MN_B>(ring + slot * kStageBytes + kStageBytes / 2);
#pragma unroll
                    for (int k = 0; k < kStep / 16; ++k)
                        mma_pair(tmem + buffer * kTile, a + k * kDescriptorStep<MN_A>, b + k * kDescriptorStep<MN_B>, kInstruction<MN_A, MN_B>, s || k);
                    commit_pair(mma_smem(&empty[slot]));
                }
                if (!late) commit_pair(mma_smem(&ready[buffer]));
            }
        }
    } else if (warp >= kEpilogueWarp) {
        Epilogue ep = given;
        const int quarter = warp & 3, half = (warp - kEpilogueWarp) >> 2;
        unsigned tile = 0;
        bool late = false;
        for (long long t = start; t < walk.count; t += pairs) {
            const TileAt at = walk.at(t);
            const unsigned buffer = tile & 1, use = tile >> 1;
            if (at.steps) {
                ++tile;
                late = late || !bar_wait(mma_smem(&ready[buffer]), use & 1);
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            }
            const int col = at.n * kTile + half * kHalf;
            ep.begin(at.m * kTile + static_cast<int>(rank) * kHalf + quarter * 32 + lane, at.split);
#pragma unroll 1
            for (int c = 0; c < kHalf; c += 32) {
                float x[32];
                __syncwarp();
                if (at.steps) {
                    tmem_load32(tmem + (static_cast<unsigned>(quarter * 32) << 16) + buffer * kTile + half * kHalf + c, x);
                } else {
#pragma unroll
                    for (int k = 0; k < 32; ++k) x[k] = 0.f;
                }
                if (late) {
#pragma unroll
                    for (int k = 0; k < 32; ++k) x[k] = CUDART_NAN_F;
                }
                ep.take(x, col + c);
            }
            ep.end(col, at.split);
            __syncwarp();
            if (at.steps) {
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                if (lane == 0) bar_arrive_leader(mma_smem(&drained[buffer]));
            }
        }
    }
    __syncwarp();
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    pair_sync();                                           // nobody leaves while the other's barriers or products may still be used
    if (warp == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" :: "r"(tmem) : "memory");
}

}  // namespace softsync
