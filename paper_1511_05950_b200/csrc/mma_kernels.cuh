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
// What bounds it: the tensor cores, busy 92 to 97 % of the cycles in large products, and through them the power limit, which takes the clock from 1.96 to
// 1.40-1.55 GHz (1450 to 1640 TFLOP/s in a launch alone, 1250 to 1310 in seconds of them).  256 x 256 is the largest tile that leaves the sums a second
// place; it takes 64 bytes of L2 a cycle and SM.
//
// Waits are bounded.  One that runs out makes the rest of what its CTA writes NaN; it waits for nothing after that, apart from copies in flight (with the same limit).
#pragma once

#include "units.cuh"

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math_constants.h>
#include <stdint.h>
#include <type_traits>

namespace softsync {

constexpr int kTile = 256, kHalf = 128, kStep = 64;          // tile, rows of an operand in a CTA, contraction steps of a stage
constexpr int kOperandBytes = kHalf * kStep * 2, kStageBytes = 2 * kOperandBytes;
constexpr int kEpilogueWarp = 4, kEpilogueWarps = 8, kMmaThreads = 32 * (kEpilogueWarp + kEpilogueWarps);
constexpr int kStages = 6;
constexpr int kDeskBytes = 4096;                               // where an epilogue warp turns a row a lane into neighbouring lanes of a row
constexpr int kDesks = kStages * kStageBytes, kMmaShared = kDesks + kEpilogueWarps * kDeskBytes + 1024;       // aligned to the swizzle's 1024 bytes
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
// One lane of a warp that runs as a whole: what it alone does keeps its operands in the warp's own registers.  Under a branch on the lane's number they were moved there
// one by one, and the products of a stage took longer to issue than to compute.
__device__ __forceinline__ bool elected()
{
    unsigned r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r != 0;
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
// At the pair's first CTA.  Relaxed: a release in the cluster's scope waits for everything that the SM has under way (1600 cycles, where a stage takes 512), and what is
// put in order here, reads of tensor memory, has fences of its own.
__device__ __forceinline__ void bar_arrive_leader(unsigned bar)
{
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" :: "r"(leaders(bar)) : "memory");
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
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];\n\t"
                 "tcgen05.wait::ld.sync.aligned;"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
                 : "r"(addr) : "memory");
}
__device__ __forceinline__ void tmem_load16(unsigned addr, float (&v)[16])
{
    unsigned *r = reinterpret_cast<unsigned *>(v);
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n\t"
                 "tcgen05.wait::ld.sync.aligned;"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(addr) : "memory");
}
__device__ __forceinline__ void tmem_store16(unsigned addr, const float (&v)[16])
{
    const unsigned *r = reinterpret_cast<const unsigned *>(v);
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
                 :: "r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
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
    int sum_stages;                       // whose sums are added up in tensor memory, where the epilogue leaves it open
    const int *live;
    int live_is_k;
    int slots;                            // pairs that work at once, where the last tiles may be split along the contraction; else 0
    int group;                            // row tiles whose turns come before the next column tile's
    int splits;                           // of the last tiles, where the host knows (no `live`)
};
// How the operands lie: MN-major or K-major.
template <bool A, bool B> struct Lying { static constexpr bool mn_a = A, mn_b = B; };

// Into how many parts the last `rest` tiles (fewer than slots) are split along their `steps`, so that they fill the GPU.  In steps of 0.4 us: a round
// takes its steps and about 6 for filling and draining the pipeline; the parts are summed by a kernel of its own (8, and 0.2 for each part's 256 KB
// written and read).  Measured: 8192 rows, 256 x 256 (one tile of 128 steps) 45 us whole, 23.6 in 4 parts, 19.4 in 12, 19.1 in 24, 19.9 in 37; 8192 x 2048 (34 tiles left over) 192 whole
// and 193 in two parts, where the power limit gives the fewer SMs a higher clock.
constexpr int kMostParts = 3;             // times slots: room in the workspace
constexpr int kLeastSplit = 16, kLeastPart = 4;                  // stages of a tile that is split, and of a part
constexpr int kSplitChoices = 11;
__host__ __device__ inline int split_choice(int j)
{
    constexpr int tried[kSplitChoices] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 37, 74};
    return tried[j];
}
__host__ __device__ inline int split_cost(int s, int rest, int steps, int slots)
{
    if (s == 1) return 5 * (steps + 6);
    if (steps < kLeastSplit || s * kLeastPart > steps || rest * s > kMostParts * slots) return 0x7fffffff;
    return 5 * ((rest * s + slots - 1) / slots * ((steps + s - 1) / s + 6) + 8) + rest * s;
}
inline int split_count(int rest, int steps, int slots)
{
    int best = 0;
    for (int j = 1; j < kSplitChoices; ++j)
        if (split_cost(split_choice(j), rest, steps, slots) < split_cost(split_choice(best), rest, steps, slots)) best = j;
    return split_choice(best);
}
// The same by a warp, a choice a lane (one by one they took 0.4 us): the first of the cheapest.
__device__ __forceinline__ int warp_split_count(int rest, int steps, int slots)
{
    const int lane = threadIdx.x & 31, j = lane < kSplitChoices ? lane : 0;
    constexpr unsigned long long packed = 1ull | 2ull << 7 | 3ull << 14 | 4ull << 21 | 6ull << 28 | 8ull << 35 | 12ull << 42 | 16ull << 49 | 24ull << 56;
    const int s = j < 9 ? static_cast<int>(packed >> (7 * j) & 127) : j == 9 ? 37 : 74;
    const unsigned cost = static_cast<unsigned>(split_cost(s, rest, steps, slots)), least = __reduce_min_sync(kAllLanes, cost);
    return __shfl_sync(kAllLanes, s, __ffs(static_cast<int>(__ballot_sync(kAllLanes, cost == least))) - 1);
}

struct TileAt { int m, n, part, first, steps; };             // tile indices, number of the part (-1: the whole tile), and its stages of the contraction

struct TileWalk {
    int tiles_m, tiles_n, all_steps, splits, group, whole, count;        // fewer than 2^31 items: the host sees to that
    __device__ __forceinline__ explicit TileWalk(const MmaPlan &p)          // by whole warps
    {
        const int live = p.live ? *p.live : 0, m = p.live && !p.live_is_k ? live : p.m, k = p.live && p.live_is_k ? live : p.k;
        tiles_m = (m + kTile - 1) / kTile;
        tiles_n = (p.n + kTile - 1) / kTile;
        all_steps = (k + kStep - 1) / kStep;
        group = p.group;
        whole = count = tiles_m * tiles_n;
        splits = 1;
        if (!p.slots) return;
        const int rest = static_cast<int>(static_cast<unsigned>(count) % static_cast<unsigned>(p.slots));
        if (!rest || (splits = p.live ? warp_split_count(rest, all_steps, p.slots) : p.splits) == 1) return;
        whole = count - rest;
        count = whole + rest * splits;
    }
    __device__ __forceinline__ void place(unsigned tile, int &m, int &n) const
    {
        if (tiles_m <= group) {
            n = static_cast<int>(tile / static_cast<unsigned>(tiles_m));
            m = static_cast<int>(tile) - n * tiles_m;
            return;
        }
        const unsigned band = static_cast<unsigned>(group) * static_cast<unsigned>(tiles_n), b = tile / band, at = tile - b * band;
        const unsigned high = static_cast<unsigned>(min(group, tiles_m - static_cast<int>(b) * group));
        n = static_cast<int>(at / high);
        m = static_cast<int>(b * static_cast<unsigned>(group) + (at - static_cast<unsigned>(n) * high));
    }
    __device__ __forceinline__ TileAt at(int t) const
    {
        TileAt r;
        r.part = -1; r.first = 0; r.steps = all_steps;
        if (t >= whole) {
            r.part = t - whole;
            const int per = (all_steps + splits - 1) / splits, tile = r.part / splits, split = r.part - tile * splits;
            r.first = min(all_steps, split * per);
            r.steps = min(all_steps, r.first + per) - r.first;
            t = whole + tile;
        }
        place(static_cast<unsigned>(t), r.m, r.n);
        return r;
    }
};

// ---- an epilogue warp's desk ---------------------------------------------------------------------------------------------
// Tensor memory gives a lane one row; stored like that, 16 bytes of 32 different rows at a time, a tile's 64 KB took 4096 trips of the load-store
// unit (2.1 us).  So rows go through shared memory, and neighbouring lanes store neighbouring vectors.  Sixteenths of 128 (of a row of 64 bytes: quarters) change
// places with the row's number, so that eight lanes never meet in a bank.
__device__ __forceinline__ void desk_put(unsigned at, uint4 v)
{
    asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" :: "r"(at), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ uint4 desk_get(unsigned at)
{
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ unsigned wide_place(int row, int vector) { return row * 128 + ((vector ^ (row & 7)) << 4); }
__device__ __forceinline__ unsigned narrow_place(int row, int vector) { return row * 64 + ((vector ^ ((row >> 1) & 3)) << 4); }

// ---- epilogues: each is called by the 32 lanes of a warp, a row a lane ------------------------------------------------------
// 16 bits of an exponential between 0 and 1: 6 of exponent, 10 of fraction, and no sign.  Half a step is 2^-11 of the value, down to 2^-62: a rare
// entry's share is as exact as a likely one's, which it would not be in fp16.  They are bits 13 to 28 of the float times 2^-64 (its exponent
// less 64), rounded.
__device__ __forceinline__ unsigned share_bits(float a, float b)
{
    const unsigned x = static_cast<unsigned>(max(__float_as_int(a) - (0x20000000 - 0x1000), 0)), y = static_cast<unsigned>(max(__float_as_int(b) - (0x20000000 - 0x1000), 0));
    return __byte_perm(x >> 13, y << 3, 0x7610);
}
__device__ __forceinline__ float2 shares_below(unsigned w)       // times 2^-64
{
    return make_float2(__uint_as_float((w & 0xffffu) << 13), __uint_as_float(w >> 3 & 0x1fffe000u));
}

// The tensor cores cut the running sum to 24 bits at every step, towards zero: over a width of 4096 that took 2e-6 of a product (256 steps of 16) whose terms have either sign, and
// 1e-5 where all have one.  So sums are taken out of tensor memory every kSumStages stages and added up in registers, rounded to nearest: 4e-7.  Taking them keeps the tensor cores from their
// sums for a while (a contraction of 8192 in sums of 1024: 7 % of its time, 240 us for 224), so results of 16 bits, whose own rounding is 2e-3, have sums of 4096: 1e-5 at most.
constexpr int kSumStages = 16, kSumStages16 = 64;

// Maximum and sum of exponentials of a row's 128 columns, and the token's product; of the piece of the vocabulary that is kept, the exponentials
// themselves, relative to that maximum, in 16 bits.
struct StatsEpilogue {
    static constexpr int kSums = kSumStages;
    static constexpr bool kAllColumns = true;                  // take: 128 columns at once, or 32
    const int *order;                     // the rows that take part, or null: all
    const long long *tokens;
    int rows, vocab;
    const int *live;
    float scale;                          // log2(e) / T
    float2 *parts;                        // [128 columns][row]: maximum of the products, sum of 2^(scale (x - maximum))
    long long part_stride;
    float *picked;                        // the token's product
    uint16_t *kept;                       // of columns from `first` on; may be null
    long long kept_stride;
    int first;
    unsigned *done;                       // counter of the next kernel, set to zero

    __device__ __forceinline__ void take(float (&x)[kHalf], int row, int col, bool late, unsigned desk) const
    {
        if (col >= vocab) return;                              // the same for the whole warp
        const bool valid = row < (live ? *live : rows);
        const long long t = valid ? tokens[order ? order[row] : row] : -1;
        if (col + kHalf > vocab) {
#pragma unroll
            for (int k = 0; k < kHalf; ++k) if (col + k >= vocab) x[k] = -CUDART_INF_F;
        }
        const bool mine = t >= col && t < col + kHalf && t < vocab;
        if (__any_sync(kAllLanes, mine)) {
            const int at = static_cast<int>(t - col);
            float z = 0.f;
#pragma unroll
            for (int k = 0; k < kHalf; ++k) z = at == k ? x[k] : z;
            if (mine) picked[row] = z;
        }
        if (late) x[0] = CUDART_NAN_F;
        float m[4] = {x[0], x[1], x[2], x[3]};
#pragma unroll
        for (int k = 4; k < kHalf; ++k) m[k & 3] = fmaxf(m[k & 3], x[k]);
        const float top = fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3])), from = top == -CUDART_INF_F ? 0.f : top;
        float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < kHalf; ++k) { x[k] = mma_ex2((x[k] - from) * scale); s[k & 3] += x[k]; }
        if (valid) parts[static_cast<long long>(col / kHalf) * part_stride + row] = make_float2(top, (s[0] + s[1]) + (s[2] + s[3]));
        if (!kept || col < first) return;
        const int lane = threadIdx.x & 31, row0 = row - lane;
        const unsigned there = __ballot_sync(kAllLanes, valid);
#pragma unroll
        for (int c = 0; c < kHalf; c += 64) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float *v = x + c + 8 * k;
                desk_put(desk + wide_place(lane, k), make_uint4(share_bits(v[0], v[1]), share_bits(v[2], v[3]), share_bits(v[4], v[5]), share_bits(v[6], v[7])));
            }
            __syncwarp();
#pragma unroll
            for (int r = lane >> 3; r < 32; r += 4) {
                const uint4 v = desk_get(desk + wide_place(r, lane & 7));
                if (there >> r & 1) *reinterpret_cast<uint4 *>(kept + (row0 + r) * kept_stride + (col - first) + c + 8 * (lane & 7)) = v;
            }
            __syncwarp();
        }
    }
};

// G = a (p - 1[j = token]) of a piece of the vocabulary, rounded to bf16.  Products are added up as for the statistics, so that they are the very values that lse is made of: taken out once,
// they left p of a confident row (product 100, width 4096) at 0.999 where it is one.
//
// p = 2^(scale (x - maximum) - log2 sum) from the statistics of the row, whose rounding is that of small numbers where p is near one.  From lse alone, p = 2^(log2(e) (x / T - lse)): the
// difference first, for the same reason, so that what is left there is lse's own rounding.
struct GradEpilogue {
    static constexpr int kSums = kSumStages;
    static constexpr bool kAllColumns = false;
    const int *order;
    const long long *tokens;
    const float2 *norms;                  // of the rows that take part, or null: from lse
    const float *lse, *coef, *coef_scale; // of all rows; coef, and what it is multiplied by, null: 1
    float sign;                           // of coef
    int rows, vocab;
    const int *live;
    float scale, last;                    // p = 2^(last (scale (x - norm.x) - norm.y)): log2(e) / T and 1, or 1 / T and log2(e)
    int first, width;                     // the piece: columns [first, first + width)
    __nv_bfloat16 *g;
    long long g_stride;

    int row, tok, valid, write;
    float a;
    float2 norm;
    __device__ __forceinline__ void begin(int r, int)
    {
        const int n = live ? *live : rows;
        row = r;
        valid = r < n;
        write = r < (n + kStep - 1) / kStep * kStep;        // rows up to a whole stage of the next product: zeros
        a = 0.f; norm = make_float2(0.f, 0.f); tok = -1;
        if (valid) {
            const int at = order ? order[r] : r;
            const long long t = tokens[at];
            tok = t >= first && t < first + width ? static_cast<int>(t - first) : -1;
            a = coef ? sign * coef[at] * *coef_scale : 1.f;
            norm = norms ? norms[r] : make_float2(0.f, lse[at]);
            if (t < 0 || t >= vocab) norm.y = CUDART_NAN_F;
        }
    }
    __device__ __forceinline__ void take(float (&x)[32], int col, unsigned desk)
    {
        if (col >= width) return;
        const unsigned at = static_cast<unsigned>(tok - col);
        const bool picked = __any_sync(kAllLanes, at < 32u);
#pragma unroll
        for (int k = 0; k < 32; ++k) x[k] = mma_ex2(fmaf(x[k] - norm.x, scale, -norm.y) * last);
        if (picked) {
#pragma unroll
            for (int k = 0; k < 32; ++k) x[k] -= at == static_cast<unsigned>(k) ? 1.f : 0.f;
        }
#pragma unroll
        for (int k = 0; k < 32; ++k) x[k] = valid ? a * x[k] : 0.f;
        const int lane = threadIdx.x & 31, row0 = row - lane, k = lane & 3;
        const unsigned there = __ballot_sync(kAllLanes, write);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float *v = x + 8 * j;
            desk_put(desk + narrow_place(lane, j), make_uint4(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7])));
        }
        __syncwarp();
#pragma unroll
        for (int r = lane >> 2; r < 32; r += 8) {
            const uint4 v = desk_get(desk + narrow_place(r, k));
            if ((there >> r & 1) && col + 8 * k < width) *reinterpret_cast<uint4 *>(g + (row0 + r) * g_stride + col + 8 * k) = v;
        }
        __syncwarp();
    }
};

// Where a product goes: alpha (D + sum) times a gain for each column, rounded once; or D (+ sum) in fp32, for another product to be added.
struct StoreTarget {
    int rows, cols;
    const int *live;                      // rows that there are, or null
    const int *order;                     // where they go, or null
    float alpha;
    const float *alpha_dev;               // may be null
    const void *gain;                     // may be null
    int gain_bf16;
    void *out;                            // bf16 or fp32; null: to `sum`
    int out_bf16, vectors;
    long long stride;
    float *sum;
    long long sum_stride;                 // whole vectors
    int add;                              // what `sum` holds
    float *parts;                         // 256 x 256 sums of each part of a split tile

    __device__ __forceinline__ int count() const { return live ? *live : rows; }
    __device__ __forceinline__ float factor() const { return alpha_dev ? alpha * *alpha_dev : alpha; }
    __device__ __forceinline__ void add_sum(int row, int col, Unit &u) const
    {
        const float4 *s = reinterpret_cast<const float4 *>(sum + static_cast<long long>(row) * sum_stride + col);
        const float4 a = s[0], b = s[1];
        u.v[0] += a.x; u.v[1] += a.y; u.v[2] += a.z; u.v[3] += a.w; u.v[4] += b.x; u.v[5] += b.y; u.v[6] += b.z; u.v[7] += b.w;
    }
    __device__ __forceinline__ void write(void *row, int col, int left, bool whole, Unit &u, const Unit &w, float factor) const
    {
#pragma unroll
        for (int j = 0; j < kUnit; ++j) u.v[j] *= factor;
        if (gain) {
#pragma unroll
            for (int j = 0; j < kUnit; ++j) u.v[j] *= w.v[j];
        }
        if (out_bf16) store_unit(static_cast<__nv_bfloat16 *>(row) + col, u, left, whole);
        else store_unit(static_cast<float *>(row) + col, u, left, whole);
    }
    // A row's unit of sums, to where it belongs.
    __device__ __forceinline__ void store(int row, int col, Unit &u) const
    {
        const int left = cols - col;
        if (left <= 0) return;
        if (add) add_sum(row, col, u);
        if (!out) {
            store_unit(sum + static_cast<long long>(row) * sum_stride + col, u, kUnit, true);
            return;
        }
        const bool whole = vectors && left >= kUnit;
        Unit w;
        if (gain) w = load_gain(gain, gain_bf16, col, left, whole);
        write(static_cast<unsigned char *>(out) + static_cast<long long>(order ? order[row] : row) * stride * (out_bf16 ? 2 : 4), col, left, whole, u, w, factor());
    }
};
struct StoreEpilogue {
    static constexpr int kSums = 0;
    static constexpr bool kAllColumns = false;
    StoreTarget target;

    // This lane stores eight columns of four rows (8 j + lane / 4) of every 32 x 32 sums: their places (null: none), found once a tile.  Where rows allow no vectors it
    // stores one column of all rows, whose places the lanes hold (-1: none).
    int row0, place;
    float factor;
    float *part;
    unsigned char *to[4];
    __device__ __forceinline__ void begin(int r, int p)
    {
        const int lane = threadIdx.x & 31, count = target.count();
        row0 = r - lane;
        factor = target.factor();
        part = p >= 0 ? target.parts + (static_cast<long long>(p) * kTile + row0 % kTile) * kTile : nullptr;
        place = -1;
        if (r < count) place = target.order ? target.order[r] : r;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int row = row0 + 8 * j + (lane >> 2);
            to[j] = nullptr;
            if (row >= count) continue;
            if (target.out) to[j] = static_cast<unsigned char *>(target.out) + static_cast<long long>(target.order ? target.order[row] : row) * target.stride * (target.out_bf16 ? 2 : 4);
            else to[j] = reinterpret_cast<unsigned char *>(target.sum + static_cast<long long>(row) * target.sum_stride);
        }
    }
    __device__ __forceinline__ void take(float (&x)[32], int col, unsigned desk)
    {
        if (col >= target.cols) return;
        const int lane = threadIdx.x & 31, unit = lane & 3, at = col + kUnit * unit, left = target.cols - at;
#pragma unroll
        for (int k = 0; k < 8; ++k)
            desk_put(desk + wide_place(lane, k), make_uint4(__float_as_uint(x[4 * k]), __float_as_uint(x[4 * k + 1]), __float_as_uint(x[4 * k + 2]), __float_as_uint(x[4 * k + 3])));
        if (target.out && !target.vectors && !part) {
            const int c = col + lane;
            float w = factor;
            if (target.gain && c < target.cols) w *= target.gain_bf16 ? unit_value(static_cast<const __nv_bfloat16 *>(target.gain) + c) : static_cast<const float *>(target.gain)[c];
            __syncwarp();
#pragma unroll 1
            for (int row = 0; row < 32; row += 8) {        // eight rows' values under way at once
                float v[8];
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v[k]) : "r"(desk + wide_place(row + k, lane >> 2) + 4 * (lane & 3)) : "memory");
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const int at_row = __shfl_sync(kAllLanes, place, row + k);
                    if (at_row < 0 || c >= target.cols) continue;
                    if (target.add) v[k] += target.sum[static_cast<long long>(row0 + row + k) * target.sum_stride + c];
                    const long long to_value = at_row * target.stride + c;
                    if (target.out_bf16) static_cast<__nv_bfloat16 *>(target.out)[to_value] = __float2bfloat16_rn(v[k] * w);
                    else static_cast<float *>(target.out)[to_value] = v[k] * w;
                }
            }
            __syncwarp();
            return;
        }
        const bool whole = target.vectors && left >= kUnit;
        Unit gain;
        if (target.gain && left > 0) gain = load_gain(target.gain, target.gain_bf16, at, left, whole);
        __syncwarp();
        uint4 v[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[2 * j] = desk_get(desk + wide_place(j * 8 + (lane >> 2), 2 * unit));
            v[2 * j + 1] = desk_get(desk + wide_place(j * 8 + (lane >> 2), 2 * unit + 1));
        }
        __syncwarp();
        if (left <= 0) return;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (!to[j]) continue;
            if (part) {
                uint4 *p = reinterpret_cast<uint4 *>(part + (j * 8 + (lane >> 2)) * kTile + at % kTile);
                p[0] = v[2 * j];
                p[1] = v[2 * j + 1];
                continue;
            }
            Unit u{{__uint_as_float(v[2 * j].x), __uint_as_float(v[2 * j].y), __uint_as_float(v[2 * j].z), __uint_as_float(v[2 * j].w), __uint_as_float(v[2 * j + 1].x),
                    __uint_as_float(v[2 * j + 1].y), __uint_as_float(v[2 * j + 1].z), __uint_as_float(v[2 * j + 1].w)}};
            if (target.add) target.add_sum(row0 + j * 8 + (lane >> 2), at, u);
            if (target.out) target.write(to[j], at, left, whole, u, gain, factor);
            else store_unit(reinterpret_cast<float *>(to[j]) + at, u, kUnit, true);
        }
    }
};

// One product of a launch: operands, extents, and what becomes of it.  Its size counts: 64 bytes more made every launch 0.6 us longer.
template <typename Epilogue>
struct alignas(64) MmaJob {
    CUtensorMap a, b;
    MmaPlan plan;
    Epilogue epilogue;
};

// The split tiles' parts added up, of up to two products.  Up to eight warps share a row's parts (all of whose loads are under way at once), a lane takes eight
// columns; the warps' sums are added in order.
struct SplitSums {
    MmaPlan plan[2];
    StoreTarget target[2];
    int blocks;                           // of the first product
};
__global__ void __launch_bounds__(256) split_sum_kernel(const __grid_constant__ SplitSums in)
{
    __shared__ float sums[8][32][kUnit + 1];
    wait_for_earlier();
    let_next_start();
    const int job = static_cast<int>(blockIdx.x) >= in.blocks, block = static_cast<int>(blockIdx.x) - (job ? in.blocks : 0);
    const int blocks = job ? static_cast<int>(gridDim.x) - in.blocks : in.blocks;
    const StoreTarget &target = in.target[job];
    const TileWalk walk(in.plan[job]);
    if (walk.splits == 1) return;
    int share = 1;                        // warps of a row
    while (share < 8 && share < walk.splits) share *= 2;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, of = warp & (share - 1), rows = 8 / share, count = target.count();
    for (int first = block * rows; first < (walk.count - walk.whole) / walk.splits * kTile; first += blocks * rows) {          // rows of split tiles
        const int rest = first / kTile, r = first % kTile + warp / share;
        int m, n;
        walk.place(static_cast<unsigned>(walk.whole + rest), m, n);
        const int row = m * kTile + r, col = n * kTile + lane * kUnit;
        Unit u{};
        if (row < count) {
            const float *p = target.parts + (static_cast<long long>(rest) * walk.splits * kTile + r) * kTile + lane * kUnit;
#pragma unroll 8
            for (int s = of; s < walk.splits; s += share) {
                const float4 *q = reinterpret_cast<const float4 *>(p + static_cast<long long>(s) * kTile * kTile);
                const float4 a = __ldcs(q), b = __ldcs(q + 1);
                u.v[0] += a.x; u.v[1] += a.y; u.v[2] += a.z; u.v[3] += a.w; u.v[4] += b.x; u.v[5] += b.y; u.v[6] += b.z; u.v[7] += b.w;
            }
        }
        if (of) {
#pragma unroll
            for (int k = 0; k < kUnit; ++k) sums[warp][lane][k] = u.v[k];
        }
        __syncthreads();
        if (!of && row < count) {
            for (int w = 1; w < share; ++w) {
#pragma unroll
                for (int k = 0; k < kUnit; ++k) u.v[k] += sums[warp + w][lane][k];
            }
            target.store(row, col, u);
        }
        __syncthreads();                  // sums are written again
    }
}

// ---- the kernel --------------------------------------------------------------------------------------------------------
// What the warps of a CTA know of its barriers, and how far they are.
struct MmaState {
    unsigned long long full[kStages], empty[kStages], ready[2], drained[2];
};

// The epilogue's side of the sums in tensor memory: waits for the next ones; gives a place back.
__device__ __forceinline__ unsigned sums_arrived(MmaState &bars, unsigned &sums, bool &late)
{
    const unsigned buffer = sums & 1;
    late = late || !bar_wait(mma_smem(&bars.ready[buffer]), (sums >> 1) & 1);
    ++sums;
    __syncwarp();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    return buffer;
}
__device__ __forceinline__ void sums_taken(MmaState &bars, unsigned buffer)
{
    __syncwarp();
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    if ((threadIdx.x & 31) == 0) bar_arrive_leader(mma_smem(&bars.drained[buffer]));
}
// The sums of `steps` stages, of `each` stages one by one, added up in registers.
__device__ __forceinline__ void add_sums(MmaState &bars, unsigned lanes, int steps, int each, float (&x)[kHalf], unsigned &sums, bool &late)
{
#pragma unroll
    for (int k = 0; k < kHalf; ++k) x[k] = 0.f;
#pragma unroll 1
    for (int s = 0; s < steps; s += each) {
        const unsigned buffer = sums_arrived(bars, sums, late);
#pragma unroll
        for (int c = 0; c < kHalf; c += 16) {
            float y[16];
            tmem_load16(lanes + buffer * kTile + c, y);
#pragma unroll
            for (int k = 0; k < 16; ++k) x[c + k] += y[k];
        }
        sums_taken(bars, buffer);
    }
}
// The same where the epilogue wants them in tensor memory, 32 columns at a time: all but the last are added to the last where it lies.  (With them in registers the epilogue's loop had to be
// unrolled, and its code took 2 us to fetch: 200 rows, 768 x 256, 9.7 us, then 11.9.)
__device__ __forceinline__ void join_sums(MmaState &bars, unsigned lanes, int steps, int each, unsigned &sums, bool &late)
{
    float x[kHalf];
    add_sums(bars, lanes, steps - each, each, x, sums, late);
    const unsigned last = lanes + sums_arrived(bars, sums, late) * kTile;
#pragma unroll
    for (int c = 0; c < kHalf; c += 16) {
        float y[16];
        tmem_load16(last + c, y);
#pragma unroll
        for (int k = 0; k < 16; ++k) y[k] += x[c + k];
        tmem_store16(last + c, y);
    }
    asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}

// One job's tiles, by every warp in its role.  turn, sums: stages and sums so far; late: a wait ran out; start: this pair's first tile.
// LONG: a tile or part may have more than one sum.
template <typename Epilogue, typename L, bool LONG>
__device__ __forceinline__ void run_job(const MmaJob<Epilogue> &job, MmaState &bars, unsigned ring, unsigned tmem, unsigned rank, int pairs, int &start, unsigned &turn, unsigned &sums, bool &late)
{
    const int warp = __shfl_sync(kAllLanes, static_cast<int>(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    const TileWalk walk(job.plan);
    const int each = !LONG ? 1 << 30 : Epilogue::kSums ? Epilogue::kSums : job.plan.sum_stages;
    if (warp == 0) {
        for (int t = start; t < walk.count && !late; t += pairs) {
            const TileAt at = walk.at(t);
            const int ya = at.m * kTile + static_cast<int>(rank) * kHalf, yb = at.n * kTile + static_cast<int>(rank) * kHalf;
            for (int s = 0; s < at.steps; ++s, ++turn) {
                const unsigned slot = turn % kStages, round = turn / kStages;
                const int x = (at.first + s) * kStep;
                if (round && !bar_wait(mma_smem(&bars.empty[slot]), (round - 1) & 1)) { late = true; break; }
                if (elected()) {
                    const unsigned bar = leaders(mma_smem(&bars.full[slot])), a = ring + slot * kStageBytes, b = a + kOperandBytes;
                    if (rank == 0) bar_expect(mma_smem(&bars.full[slot]), 2 * kStageBytes);
                    if constexpr (L::mn_a) { tile_load(a, &job.a, ya, x, bar); tile_load(a + 8192, &job.a, ya + 64, x, bar); }
                    else tile_load(a, &job.a, x, ya, bar);
                    if constexpr (L::mn_b) { tile_load(b, &job.b, yb, x, bar); tile_load(b + 8192, &job.b, yb + 64, x, bar); }
                    else tile_load(b, &job.b, x, yb, bar);
                }
                __syncwarp();
            }
        }
    } else if (warp == 1) {
        for (int t = start; rank == 0 && t < walk.count && !late; t += pairs) {
            const TileAt at = walk.at(t);
            unsigned buffer = 0;
            for (int s = 0; s < at.steps; ++s, ++turn) {
                const int in = LONG ? static_cast<int>(static_cast<unsigned>(s) % static_cast<unsigned>(each)) : s;
                if (in == 0) {
                    if (s && elected()) commit_pair(mma_smem(&bars.ready[buffer]));
                    buffer = sums & 1;
                    const unsigned use = sums >> 1;
                    ++sums;
                    if (use && !bar_wait(mma_smem(&bars.drained[buffer]), (use - 1) & 1)) { late = true; break; }
                }
                const unsigned slot = turn % kStages;
                if (!bar_wait(mma_smem(&bars.full[slot]), (turn / kStages) & 1)) { late = true; break; }
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint64_t a = operand_descriptor<L::mn_a>(ring + slot * kStageBytes), b = operand_descriptor<L::mn_b>(ring + slot * kStageBytes + kOperandBytes);
                if (elected()) {
#pragma unroll
                    for (int k = 0; k < kStep / 16; ++k)
                        mma_pair(tmem + buffer * kTile, a + k * kDescriptorStep<L::mn_a>, b + k * kDescriptorStep<L::mn_b>, kInstruction<L::mn_a, L::mn_b>, in || k);
                    commit_pair(mma_smem(&bars.empty[slot]));
                }
                __syncwarp();
            }
            if (!late && at.steps && elected()) commit_pair(mma_smem(&bars.ready[buffer]));
            __syncwarp();
        }
    } else if (warp >= kEpilogueWarp) {
        Epilogue ep = job.epilogue;
        const int quarter = warp & 3, half = (warp - kEpilogueWarp) >> 2;
        const unsigned lanes = tmem + (static_cast<unsigned>(quarter * 32) << 16) + half * kHalf, desk = ring + kDesks + (warp - kEpilogueWarp) * kDeskBytes;
        if constexpr (Epilogue::kAllColumns) if (blockIdx.x == 0 && threadIdx.x == 32 * kEpilogueWarp && ep.done) *ep.done = 0;
        for (int t = start; t < walk.count; t += pairs) {
            const TileAt at = walk.at(t);
            const int col = at.n * kTile + half * kHalf, row = at.m * kTile + static_cast<int>(rank) * kHalf + quarter * 32 + lane;
            if constexpr (Epilogue::kAllColumns) {
                float x[kHalf];
                add_sums(bars, lanes, at.steps, each, x, sums, late);
                ep.take(x, row, col, late, desk);
            } else {
                if (LONG && at.steps > each) join_sums(bars, lanes, at.steps, each, sums, late);
                else if (at.steps) sums_arrived(bars, sums, late);
                const unsigned buffer = (sums - 1) & 1;
                ep.begin(row, at.part);
#pragma unroll 1
                for (int c = 0; c < kHalf; c += 32) {
                    float v[32];
                    __syncwarp();
                    if (at.steps) {
                        tmem_load32(lanes + buffer * kTile + c, v);
                    } else {
#pragma unroll
                        for (int k = 0; k < 32; ++k) v[k] = 0.f;
                    }
                    if (late) {
#pragma unroll
                        for (int k = 0; k < 32; ++k) v[k] = CUDART_NAN_F;
                    }
                    ep.take(v, col + c, desk);
                }
                if (at.steps) sums_taken(bars, buffer);
            }
        }
    }
    __syncwarp();                                      // the next walk is a whole warp's
    start = (start + pairs - walk.count % pairs) % pairs;           // turns go on where they are
}

// Of two jobs (M not void) the second's tiles follow the first's.  Without LONG it has 128 registers instead of 168, and kernels before and after it on the stream have room to prepare themselves beside it
// (weight gradient of 200 rows, 768 x 256: 9.6 us, 10.9 with it).
template <typename Epilogue, typename L, typename M, bool LONG>
__global__ void __cluster_dims__(2) __launch_bounds__(kMmaThreads, 1) mma_kernel(const __grid_constant__ MmaJob<Epilogue> first, const __grid_constant__ MmaJob<Epilogue> second)
{
    extern __shared__ unsigned char raw_ring[];
    __shared__ __align__(8) MmaState bars;
    __shared__ unsigned tmem_base;
    const unsigned ring = (mma_smem(raw_ring) + 1023u) & ~1023u;
    const int warp = __shfl_sync(kAllLanes, static_cast<int>(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    const unsigned rank = pair_rank();
    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) { bar_init(mma_smem(&bars.full[s]), 1); bar_init(mma_smem(&bars.empty[s]), 1); }
        for (int b = 0; b < 2; ++b) { bar_init(mma_smem(&bars.ready[b]), 1); bar_init(mma_smem(&bars.drained[b]), 2 * kEpilogueWarps); }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("prefetch.tensormap [%0];" :: "l"(&first.a) : "memory");
        asm volatile("prefetch.tensormap [%0];" :: "l"(&first.b) : "memory");
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
    wait_for_earlier();
    let_next_start();
    const int pairs = static_cast<int>(gridDim.x >> 1);
    int start = static_cast<int>(blockIdx.x >> 1);
    unsigned turn = 0, sums = 0;                           // stages and sums so far, of both products
    bool late = false;
    run_job<Epilogue, L, LONG>(first, bars, ring, tmem, rank, pairs, start, turn, sums, late);
    if constexpr (!std::is_void_v<M>) run_job<Epilogue, M, LONG>(second, bars, ring, tmem, rank, pairs, start, turn, sums, late);
    if (warp == 0 && lane == 0)                            // every copy has arrived, and every stage's release, before either CTA may leave
        for (unsigned k = turn > kStages ? turn - kStages : 0; k < turn; ++k) {
            late = late || !bar_wait(mma_smem(&bars.empty[k % kStages]), (k / kStages) & 1);
            if (late && rank == 0) bar_wait(mma_smem(&bars.full[k % kStages]), (k / kStages) & 1);
        }
    __syncwarp();
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    pair_sync();                                           // nobody leaves while the other's barriers or products may still be used
    if (warp == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" :: "r"(tmem) : "memory");
}

}  // namespace softsync
