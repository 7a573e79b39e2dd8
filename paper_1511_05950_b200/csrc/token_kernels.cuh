// Kernels over rows of logits: softmax statistics of a row, the terms of the losses, gradients.
//
// A row's statistics are its maximum m (in the logits' own units), the sum s of 2^((x - m) c) with c = log2(e) / T, and the sum t of
// that times (x - m) c, from which log probability, log normaliser and entropy follow:
//     lse = m / T + ln 2 log2(s),    H = ln 2 (log2(s) - t / s),    p_j = 2^((x_j - m) c - log2(s)).
//
// A row is cut into 16-byte vectors at 16-byte addresses; where a row starts or ends inside one (an odd vocabulary), that vector's
// elements are handled one by one, so nothing outside the row is read or written.
//
// What bounds these kernels: HBM (bf16: 2 bytes an element for the statistics, 4 for statistics and gradient), with the
// exponential unit close behind: it gives 16 results a clock and SM, and at 7 TB/s 12 of them are wanted in either case.  So a
// row is read ONCE and stays in registers between its statistics and its gradient, split over a cluster of up to eight
// blocks where one block's registers do not hold it; the blocks exchange three numbers each through distributed shared memory.
#pragma once

#include "update_kernels.cuh"

#include <math_constants.h>

namespace softsync {

constexpr float kLn2 = 0.6931471805599453f;
constexpr float kLowest = -3.402823466e38f;
constexpr float kFloor = -1e30f;          // logits below this have p = 0 beside an ordinary maximum

// Whether no product of a logit above the floor with c overflows and every logit below the floor has p = 0 beside the maximum m.
__device__ __forceinline__ bool ordinary(float m, float c) { return fabsf(m) < 1e29f && c < 1e7f && c > 1e-20f; }

struct RowsIn {
    const unsigned char *data;
    long long rows, vocab, stride;        // stride in elements
    const long long *tokens;
    const float *weights;                 // nullptr: ones
    float scale;                          // c = log2(e) / T
    float inv_temperature;
};

// What a row leaves for a later gradient pass.
struct RowStat { float max, log2_sum; };

// ---- instructions ----------------------------------------------------------------------------------------------------
__device__ __forceinline__ float max_nan(float a, float b)             // NaN if either is
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ unsigned max_nan_bf16x2(unsigned a, unsigned b)
{
    unsigned r;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ unsigned max_bf16x2(unsigned a, unsigned b) // the other one if one is NaN
{
    unsigned r;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ float ex2(float x)                           // 2^x, results below the smallest normal are zero
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float warp_max(float x)
{
    float r;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float warp_sum(float x)
{
    for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c)
{
    unsigned long long r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(*reinterpret_cast<unsigned long long *>(&a)),
        "l"(*reinterpret_cast<unsigned long long *>(&b)), "l"(*reinterpret_cast<unsigned long long *>(&c)));
    return *reinterpret_cast<float2 *>(&r);
}
__device__ __forceinline__ float2 add2(float2 a, float2 b)
{
    unsigned long long r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(*reinterpret_cast<unsigned long long *>(&a)), "l"(*reinterpret_cast<unsigned long long *>(&b)));
    return *reinterpret_cast<float2 *>(&r);
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b)
{
    unsigned long long r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(*reinterpret_cast<unsigned long long *>(&a)), "l"(*reinterpret_cast<unsigned long long *>(&b)));
    return *reinterpret_cast<float2 *>(&r);
}

// ---- 16-byte vectors of a row ------------------------------------------------------------------------------------------
template <typename GT> __host__ __device__ constexpr int logit_bytes() { return sizeof(Raw<GT, 1>); }
template <typename GT> __host__ __device__ constexpr int per_vector() { return 16 / logit_bytes<GT>(); }

__device__ __forceinline__ float logit_at(const GradFp32 *, const unsigned char *row, long long j) { return reinterpret_cast<const float *>(row)[j]; }
__device__ __forceinline__ float logit_at(const GradBf16 *, const unsigned char *row, long long j)
{ return __uint_as_float(static_cast<unsigned>(reinterpret_cast<const unsigned short *>(row)[j]) << 16); }

// A row as vectors: vector q holds the elements [q * per_vector - phase, ...) of the row.
template <typename GT>
struct RowVectors {
    const unsigned char *row;
    int phase, vocab, count;
    __device__ __forceinline__ RowVectors(const unsigned char *r, int v) : row(r), vocab(v)
    {
        phase = static_cast<int>(reinterpret_cast<uintptr_t>(r) & 15) / logit_bytes<GT>();
        count = (phase + v + per_vector<GT>() - 1) / per_vector<GT>();
    }
    __device__ __forceinline__ int first(int q) const { return q * per_vector<GT>() - phase; }
    __device__ __forceinline__ bool whole(int q) const { return first(q) >= 0 && first(q) + per_vector<GT>() <= vocab; }
};

__device__ __forceinline__ uint4 load_vector16(const void *p)
{
    uint4 r;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(p));
    return r;
}

// Vector q, minus infinity where it reaches beyond the row.
template <typename GT>
__device__ __forceinline__ uint4 load_row_vector(const RowVectors<GT> &v, int q)
{
    const int j = v.first(q);
    if (v.whole(q)) return load_vector16(v.row + static_cast<long long>(j) * logit_bytes<GT>());
    uint4 r;
    unsigned *w = &r.x;
    if constexpr (logit_bytes<GT>() == 4) {
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] = j + k >= 0 && j + k < v.vocab ? reinterpret_cast<const unsigned *>(v.row)[j + k] : 0xff800000u;
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const unsigned short *h = reinterpret_cast<const unsigned short *>(v.row);
            const unsigned lo = j + 2 * k >= 0 && j + 2 * k < v.vocab ? h[j + 2 * k] : 0xff80u;
            const unsigned hi = j + 2 * k + 1 >= 0 && j + 2 * k + 1 < v.vocab ? h[j + 2 * k + 1] : 0xff80u;
            w[k] = lo | hi << 16;
        }
    }
    return r;
}

// Writes vector q's values g to the row at dst; `same` says that dst has the source row's place within 16 bytes.
template <typename GT>
__device__ __forceinline__ void store_row_vector(const RowVectors<GT> &v, int q, unsigned char *dst, bool same, const float (&g)[per_vector<GT>()])
{
    const int j = v.first(q);
    if (same && v.whole(q)) {
        uint4 r;
        if constexpr (logit_bytes<GT>() == 4) r = make_uint4(__float_as_uint(g[0]), __float_as_uint(g[1]), __float_as_uint(g[2]), __float_as_uint(g[3]));
        else r = make_uint4(pack_bf16x2(g[0], g[1]), pack_bf16x2(g[2], g[3]), pack_bf16x2(g[4], g[5]), pack_bf16x2(g[6], g[7]));
        __stcs(reinterpret_cast<uint4 *>(dst + static_cast<long long>(j) * logit_bytes<GT>()), r);
        return;
    }
#pragma unroll
    for (int k = 0; k < per_vector<GT>(); ++k)
        if (j + k >= 0 && j + k < v.vocab) {
            if constexpr (logit_bytes<GT>() == 4) reinterpret_cast<float *>(dst)[j + k] = g[k];
            else reinterpret_cast<unsigned short *>(dst)[j + k] = __bfloat16_as_ushort(__float2bfloat16_rn(g[k]));
        }
}

// Zeros over a whole row (its part of `parts`), by the row's own alignment.
template <typename GT>
__device__ __forceinline__ void zero_row(unsigned char *dst, int vocab, int part, int parts)
{
    const RowVectors<GT> v(dst, vocab);
    const float zero[per_vector<GT>()] = {};
    for (int q = part * static_cast<int>(blockDim.x) + threadIdx.x; q < v.count; q += parts * blockDim.x) store_row_vector(v, q, dst, true, zero);
}

// The elements of word k of a vector, as fp32.
__device__ __forceinline__ float2 unpack_bf16(unsigned w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }

// Largest element of the vectors, NaN left aside.
template <typename GT, int NV>
__device__ __forceinline__ float vectors_max(const uint4 (&x)[NV])
{
    if constexpr (logit_bytes<GT>() == 4) {
        float m = -CUDART_INF_F;
#pragma unroll
        for (int v = 0; v < NV; ++v)
            m = fmaxf(m, fmaxf(fmaxf(__uint_as_float(x[v].x), __uint_as_float(x[v].y)), fmaxf(__uint_as_float(x[v].z), __uint_as_float(x[v].w))));
        return m;
    } else {
        unsigned m = 0xff80ff80u;
#pragma unroll
        for (int v = 0; v < NV; ++v) m = max_bf16x2(m, max_bf16x2(max_bf16x2(x[v].x, x[v].y), max_bf16x2(x[v].z, x[v].w)));
        const float2 f = unpack_bf16(m);
        return fmaxf(f.x, f.y);
    }
}

// Two elements of a vector with everything below the floor raised to it: minus infinity times p = 0 would be NaN.
template <typename GT>
__device__ __forceinline__ float2 floored_pair(const uint4 &x, int k)
{
    const unsigned *w = &x.x;
    if constexpr (logit_bytes<GT>() == 4)
        return make_float2(max_nan(__uint_as_float(w[2 * k]), kFloor), max_nan(__uint_as_float(w[2 * k + 1]), kFloor));
    else
        return unpack_bf16(max_nan_bf16x2(w[k], 0xf149f149u));          // -9.95e29 in bf16
}
template <typename GT>
__device__ __forceinline__ float2 plain_pair(const uint4 &x, int k)
{
    const unsigned *w = &x.x;
    if constexpr (logit_bytes<GT>() == 4) return make_float2(__uint_as_float(w[2 * k]), __uint_as_float(w[2 * k + 1]));
    else return unpack_bf16(w[k]);
}

// Adds the vectors' exponentials relative to the maximum m to s, and (ENTROPY) times their exponents to t.  The difference to the
// maximum is taken before it is scaled: the maximum's own exponent is exactly zero, and a row that a mask of the type's lowest value
// leaves nothing of stays finite (its softmax is uniform).  Beside an ordinary maximum pairs go through packed instructions and the floor
// stands in for minus infinity; else every exponent is held above -1000.
template <typename GT, int NV, bool ENTROPY>
__device__ __forceinline__ void row_exponentials(const uint4 (&x)[NV], float m, float c, float &s, float &t)
{
    if (ordinary(m, c)) {
        const float2 c2 = make_float2(c, c), m2 = make_float2(-m, -m);
        float2 s2 = make_float2(0.f, 0.f), t2 = s2;
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int k = 0; k < per_vector<GT>() / 2; ++k) {
                const float2 d = mul2(add2(ENTROPY ? floored_pair<GT>(x[v], k) : plain_pair<GT>(x[v], k), m2), c2);
                const float2 e = make_float2(ex2(d.x), ex2(d.y));
                s2 = add2(s2, e);
                if constexpr (ENTROPY) t2 = fma2(e, d, t2);
            }
        s += s2.x + s2.y;
        if constexpr (ENTROPY) t += t2.x + t2.y;
    } else {
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int k = 0; k < per_vector<GT>() / 2; ++k) {
                const float2 y = plain_pair<GT>(x[v], k);
                const float a = max_nan((y.x - m) * c, -1000.f), b = max_nan((y.y - m) * c, -1000.f);
                const float e = ex2(a), f = ex2(b);
                s += e + f;
                if constexpr (ENTROPY) t += e * a + f * b;
            }
    }
}

// What multiplies the exponentials of a part with maximum m in a whole with maximum `top`.
__device__ __forceinline__ float part_factor(float m, float top, float c, float &d)
{
    d = fmaxf((m - top) * c, -1000.f);
    return ex2(d);
}

// Per-row factors of the gradient: dz_j = a (1[j = token] - p_j) + b p_j (log p_j + H).
struct RowCoef { float a, b; };

// Gradient of one vector.  With d = (x - m) c - log2 s:  p = 2^d,  g = p (b ln 2 d + (b H - a)).
template <typename GT, bool ENTROPY>
__device__ __forceinline__ void vector_gradient(const uint4 &x, float m, float log2_sum, float c, RowCoef k, float entropy, float (&g)[per_vector<GT>()])
{
    const float add = ENTROPY ? fmaf(k.b, entropy, -k.a) : -k.a, mult = k.b * kLn2;
    if (ordinary(m, c)) {
        const float2 c2 = make_float2(c, c), mm = make_float2(-m, -m), l2 = make_float2(-log2_sum, -log2_sum), a2 = make_float2(add, add), m2 = make_float2(mult, mult);
#pragma unroll
        for (int j = 0; j < per_vector<GT>() / 2; ++j) {
            const float2 d = fma2(add2(ENTROPY ? floored_pair<GT>(x, j) : plain_pair<GT>(x, j), mm), c2, l2);
            const float2 p = make_float2(ex2(d.x), ex2(d.y));
            const float2 r = mul2(p, ENTROPY ? fma2(m2, d, a2) : a2);
            g[2 * j] = r.x;
            g[2 * j + 1] = r.y;
        }
    } else {
#pragma unroll
        for (int j = 0; j < per_vector<GT>(); ++j) {
            const float2 y = plain_pair<GT>(x, j / 2);
            const float d = max_nan(((j & 1 ? y.y : y.x) - m) * c, -1000.f) - log2_sum;
            g[j] = ex2(d) * (ENTROPY ? fmaf(mult, d, add) : add);
        }
    }
}

// ---- clusters ------------------------------------------------------------------------------------------------------------
__device__ __forceinline__ unsigned cluster_rank() { unsigned r; asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ unsigned cluster_size() { unsigned r; asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ void store_to_rank(const void *mine, unsigned rank, float x)
{
    unsigned addr;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(addr) : "r"(smem_addr(mine)), "r"(rank));
    asm volatile("st.shared::cluster.f32 [%0], %1;" :: "r"(addr), "f"(x) : "memory");
}

constexpr int kMaxCluster = 8;

struct RowShared {
    float warp[3][32];                    // each warp's m, s, t
    float part[3][kMaxCluster];           // each block's m, s, t, written by the blocks
    float row[5];                         // m, log2 s, entropy, a, b: what every thread needs for the gradient
    float terms[5];                       // the row's share of the policy loss's sums
};

// The row's m, s, t from the warps' of all its blocks, in every lane of warp 0 (the other warps get nothing).  All threads of
// all blocks call it; between its two halves of the cluster barrier the blocks write into one another's shared memory.
// cluster_arrive() has been called once before, so that no block writes before its peer has started.
__device__ __forceinline__ void join_row(RowShared &sh, float c, float &m, float &s, float &t)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const unsigned blocks = cluster_size();
    s = warp_sum(s);
    t = warp_sum(t);
    if (lane == 0) { sh.warp[0][warp] = m; sh.warp[1][warp] = s; sh.warp[2][warp] = t; }
    __syncthreads();
    if (warp == 0) {
        m = lane < warps ? sh.warp[0][lane] : kLowest;
        s = lane < warps ? sh.warp[1][lane] : 0.f;
        t = lane < warps ? sh.warp[2][lane] : 0.f;
        const float top = warp_max(m);
        float d;
        const float f = part_factor(m, top, c, d);
        t = warp_sum(f * fmaf(s, d, t));
        s = warp_sum(f * s);
        m = top;
    }
    if (blocks == 1) return;
    cluster_wait();                                       // every block of the row has started
    if (warp == 0 && lane < static_cast<int>(blocks)) {
        const unsigned me = cluster_rank();
        store_to_rank(&sh.part[0][me], lane, m);
        store_to_rank(&sh.part[1][me], lane, s);
        store_to_rank(&sh.part[2][me], lane, t);
    }
    cluster_arrive();
    cluster_wait();
    if (warp == 0) {
        m = lane < static_cast<int>(blocks) ? sh.part[0][lane] : kLowest;
        s = lane < static_cast<int>(blocks) ? sh.part[1][lane] : 0.f;
        t = lane < static_cast<int>(blocks) ? sh.part[2][lane] : 0.f;
        const float top = warp_max(m);
        float d;
        const float f = part_factor(m, top, c, d);
        t = warp_sum(f * fmaf(s, d, t));
        s = warp_sum(f * s);
        m = top;
    }
}

// ---- statistics of a row, in batches -----------------------------------------------------------------------------------------
struct StatsOut {
    float *logp, *lse, *entropy;          // lse, entropy may be null
    RowStat *stat;                        // may be null
    RowCoef *coef;                        // set to zero for the kernel that follows (may be null), and so is
    unsigned *counter;
};

// One cluster per row; each thread holds NV vectors of a batch at a time.  A batch's maximum is taken over the whole warp before
// any exponential, so that the running sums are rescaled once a batch and by the same factor in every lane.
template <typename GT, int NV, bool ENTROPY>
__global__ void __launch_bounds__(512) row_stats_kernel(const __grid_constant__ RowsIn in, const __grid_constant__ StatsOut out)
{
    __shared__ RowShared sh;
    const int blocks = cluster_size(), rank = cluster_rank();
    const long long r = blockIdx.x / static_cast<unsigned>(blocks);
    if (rank == 0 && threadIdx.x == 0) {
        if (out.coef) out.coef[r] = RowCoef{0.f, 0.f};
        if (out.counter && r == 0) *out.counter = 0;
    }
    if (in.weights && in.weights[r] == 0.f) {              // the whole cluster leaves
        if (rank == 0 && threadIdx.x == 0) {
            out.logp[r] = 0.f;
            if (out.lse) out.lse[r] = 0.f;
            if (out.entropy) out.entropy[r] = 0.f;
        }
        return;
    }
    if (blocks > 1) cluster_arrive();
    const unsigned char *row = in.data + r * in.stride * logit_bytes<GT>();
    const RowVectors<GT> v(row, static_cast<int>(in.vocab));
    long long tok = -1;
    float x_tok = CUDART_NAN_F;
    if (threadIdx.x == 0) {
        tok = in.tokens[r];
        if (tok >= 0 && tok < in.vocab) x_tok = logit_at(static_cast<const GT *>(nullptr), row, tok);
    }
    const int threads = blockDim.x;
    float m = kLowest, s = 0.f, t = 0.f;
    for (int base = rank * NV * threads; base < v.count; base += blocks * NV * threads) {
        uint4 x[NV];
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int q = base + k * threads + threadIdx.x;
            x[k] = q < v.count ? load_row_vector(v, q) : (logit_bytes<GT>() == 4 ? make_uint4(0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u)
                                                                                 : make_uint4(0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u));
        }
        const float top = fmaxf(warp_max(vectors_max<GT, NV>(x)), m);
        if (top > m) {
            float d;
            const float f = part_factor(m, top, in.scale, d);
            t = f * fmaf(s, d, t);
            s *= f;
            m = top;
        }
        row_exponentials<GT, NV, ENTROPY>(x, m, in.scale, s, t);
    }
    join_row(sh, in.scale, m, s, t);
    if (rank || threadIdx.x) return;
    const float l2 = log2f(s);
    out.logp[r] = (x_tok - m) * in.inv_temperature - kLn2 * l2;
    if (out.lse) out.lse[r] = m * in.inv_temperature + kLn2 * l2;
    if (ENTROPY && out.entropy) out.entropy[r] = kLn2 * (l2 - t / s);
    if (out.stat) out.stat[r] = RowStat{m, l2};
}

// ---- gradient from statistics -----------------------------------------------------------------------------------------------
constexpr int kGradThreads = 256, kGradVectors = 4;

// One block per segment of a row, rows from the last to the first: the statistics pass went the other way, so the rows it read
// last, which the L2 still holds, come first.
template <typename GT, bool ENTROPY>
__global__ void __launch_bounds__(kGradThreads) row_grad_kernel(const __grid_constant__ RowsIn in, const RowStat *stat, const RowCoef *coef,
                                                                const float *entropy, unsigned char *out, long long out_stride, int segments)
{
    const long long r = in.rows - 1 - blockIdx.x / static_cast<unsigned>(segments);
    const int segment = blockIdx.x % static_cast<unsigned>(segments);
    const unsigned char *row = in.data + r * in.stride * logit_bytes<GT>();
    unsigned char *dst = out + r * out_stride * logit_bytes<GT>();
    const RowCoef k = coef[r];
    if ((in.weights && in.weights[r] == 0.f) || (k.a == 0.f && k.b == 0.f)) {        // nothing to read: the gradient is zero
        zero_row<GT>(dst, static_cast<int>(in.vocab), segment, segments);
        return;
    }
    const RowVectors<GT> v(row, static_cast<int>(in.vocab));
    uint4 x[kGradVectors];
    const int base = segment * kGradVectors * kGradThreads + threadIdx.x;
#pragma unroll
    for (int i = 0; i < kGradVectors; ++i)
        if (base + i * kGradThreads < v.count) x[i] = load_row_vector(v, base + i * kGradThreads);
    const RowStat st = stat[r];
    const float h = ENTROPY ? entropy[r] : 0.f;
    const long long tok = in.tokens[r];
    const bool same = ((reinterpret_cast<uintptr_t>(row) ^ reinterpret_cast<uintptr_t>(dst)) & 15) == 0;
#pragma unroll
    for (int i = 0; i < kGradVectors; ++i) {
        const int q = base + i * kGradThreads;
        if (q >= v.count) break;
        float g[per_vector<GT>()];
        vector_gradient<GT, ENTROPY>(x[i], st.max, st.log2_sum, in.scale, k, h, g);
        const long long at = tok - v.first(q);
        if (at >= 0 && at < per_vector<GT>())
#pragma unroll
            for (int j = 0; j < per_vector<GT>(); ++j)
                if (j == at) g[j] += k.a;
        store_row_vector(v, q, dst, same, g);
    }
}

// ---- the policy loss -----------------------------------------------------------------------------------------------------
struct PolicyIn {
    const float *old_logp, *advantages, *ref_logp;
    float low, high, kl_coef, entropy_coef;            // low = 1 - clip_low, high = 1 + clip_high
};

// One token's terms: {loss, clipped term, KL, entropy, clipped} and the slope dl / dlogp.
struct PolicyTerms { float v[5], slope; };
__device__ __forceinline__ PolicyTerms policy_terms(const PolicyIn &in, float adv, float old_logp, float ref_logp, float logp, float entropy)
{
    const float ratio = expf(logp - old_logp);
    const float free_ = ratio * adv, held = fminf(max_nan(ratio, in.low), in.high) * adv;
    const bool clipped = free_ > held;
    PolicyTerms o;
    o.v[1] = clipped ? -held : -free_;
    o.slope = clipped ? 0.f : -free_;
    o.v[2] = 0.f;
    if (in.ref_logp) {
        const float d = ref_logp - logp, e = expm1f(d);
        o.v[2] = e - d;
        o.slope -= in.kl_coef * e;
    }
    o.v[0] = o.v[1] + in.kl_coef * o.v[2] - in.entropy_coef * entropy;
    o.v[3] = entropy;
    o.v[4] = clipped ? 1.f : 0.f;
    return o;
}

constexpr int kTermThreads = 1024;
constexpr int kRowGroup = 64;             // rows whose terms one warp adds up

struct Totals {                           // written by policy_totals_kernel, or reset by it
    double inv_weight;                    // 1 / sum of the weights, 0 where that is 0
    unsigned groups_done;
};

// Sum over the block, the same bits in every thread.
__device__ __forceinline__ double block_total(double x, double *scratch)
{
    for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = x;
    __syncthreads();
    double y = 0;
    for (int k = 0; k < static_cast<int>(blockDim.x >> 5); ++k) y += scratch[k];
    return y;
}

// The sum of the weights, and zeros in the counters.  The row kernel is launched as a dependent that may start at once: it
// needs neither before it has read its row.
static __global__ void __launch_bounds__(kTermThreads) policy_totals_kernel(const float *weights, long long rows, Totals *totals, unsigned *group_count, int groups)
{
    __shared__ double scratch[kTermThreads / 32];
    griddep_launch_dependents();
    for (int k = threadIdx.x; k < groups; k += blockDim.x) group_count[k] = 0;
    double sum = 0;
    if (weights)
        for (long long r = threadIdx.x; r < rows; r += blockDim.x) sum += weights[r];
    sum = weights ? block_total(sum, scratch) : static_cast<double>(rows);
    if (threadIdx.x == 0) {
        totals->inv_weight = sum != 0.0 ? 1.0 / sum : 0.0;
        totals->groups_done = 0;
    }
}

struct TermsOut {
    Totals *totals;
    unsigned *group_count;                // rows of each group that are done
    float (*terms)[5];                    // each row's share of the five sums
    double (*group_sum)[5];
    float *stats;
};

// Called by one whole warp once per row, with the row's terms already times its share (zeros for a row of weight zero).  The warp that
// completes a group of kRowGroup rows adds the group up, the one that completes the last group adds the groups up: always the same
// additions, whichever warp does them.
__device__ __forceinline__ void count_row(const TermsOut &out, long long rows, long long r, const float (&v)[5])
{
    const int lane = threadIdx.x & 31;
    const long long group = r / kRowGroup, groups = (rows + kRowGroup - 1) / kRowGroup;
    const long long first = group * kRowGroup;
    const unsigned size = static_cast<unsigned>(min(static_cast<long long>(kRowGroup), rows - first));
    unsigned before = 0;
    if (lane == 0) {
#pragma unroll
        for (int q = 0; q < 5; ++q) __stcg(&out.terms[r][q], v[q]);
        __threadfence();
        before = atomicAdd(out.group_count + group, 1u);
    }
    if (__shfl_sync(0xffffffffu, before, 0) + 1 != size) return;
    __threadfence();
    double sum[5] = {};
    for (unsigned k = lane; k < size; k += 32)
#pragma unroll
        for (int q = 0; q < 5; ++q) sum[q] += __ldcg(&out.terms[first + k][q]);
#pragma unroll
    for (int q = 0; q < 5; ++q)
        for (int o = 16; o; o >>= 1) sum[q] += __shfl_xor_sync(0xffffffffu, sum[q], o);
    if (lane == 0) {
#pragma unroll
        for (int q = 0; q < 5; ++q) __stcg(&out.group_sum[group][q], sum[q]);
        __threadfence();
        before = atomicAdd(&out.totals->groups_done, 1u);
    }
    if (__shfl_sync(0xffffffffu, before, 0) + 1 != groups) return;
    __threadfence();
    double all[5] = {};
    for (long long k = lane; k < groups; k += 32)
#pragma unroll
        for (int q = 0; q < 5; ++q) all[q] += __ldcg(&out.group_sum[k][q]);
#pragma unroll
    for (int q = 0; q < 5; ++q)
        for (int o = 16; o; o >>= 1) all[q] += __shfl_xor_sync(0xffffffffu, all[q], o);
    if (lane == 0)
#pragma unroll
        for (int q = 0; q < 5; ++q) out.stats[q] = static_cast<float>(all[q]);
}

// Statistics, loss terms and gradient (out: null for none) of a row from one read: the row's vectors stay in the registers of its
// cluster, at most NV a thread.
template <typename GT, int NV, bool ENTROPY_GRAD>
__global__ void __launch_bounds__(1024) policy_row_kernel(const __grid_constant__ RowsIn in, const __grid_constant__ PolicyIn pin,
                                                          const __grid_constant__ TermsOut terms, float *logp, float *entropy,
                                                          unsigned char *out, long long out_stride)
{
    __shared__ RowShared sh;
    const int blocks = cluster_size(), rank = cluster_rank();
    const long long r = blockIdx.x / static_cast<unsigned>(blocks);
    unsigned char *dst = out + r * out_stride * logit_bytes<GT>();
    const float w = in.weights ? in.weights[r] : 1.f;
    if (w == 0.f) {                                        // the whole cluster takes this way
        if (rank == 0 && threadIdx.x < 32) {
            if (threadIdx.x == 0) { logp[r] = 0.f; entropy[r] = 0.f; }
            griddep_wait();
            const float none[5] = {};
            count_row(terms, in.rows, r, none);
        }
        if (out) zero_row<GT>(dst, static_cast<int>(in.vocab), rank, blocks);
        return;
    }
    if (blocks > 1) cluster_arrive();
    const unsigned char *row = in.data + r * in.stride * logit_bytes<GT>();
    const RowVectors<GT> v(row, static_cast<int>(in.vocab));
    const int threads = blockDim.x, base = rank * NV * threads + threadIdx.x;
    uint4 x[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int q = base + k * threads;
        x[k] = q < v.count ? load_row_vector(v, q) : (logit_bytes<GT>() == 4 ? make_uint4(0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u)
                                                                             : make_uint4(0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u));
    }
    const long long tok = in.tokens[r];
    float x_tok = CUDART_NAN_F, adv = 0.f, old_logp = 0.f, ref_logp = 0.f;
    if (threadIdx.x < 32) {
        if (tok >= 0 && tok < in.vocab) x_tok = logit_at(static_cast<const GT *>(nullptr), row, tok);
        adv = pin.advantages[r];
        old_logp = pin.old_logp[r];
        if (pin.ref_logp) ref_logp = pin.ref_logp[r];
    }
    float m = fmaxf(warp_max(vectors_max<GT, NV>(x)), kLowest), s = 0.f, t = 0.f;
    row_exponentials<GT, NV, true>(x, m, in.scale, s, t);
    join_row(sh, in.scale, m, s, t);
    if (threadIdx.x < 32) {
        const float l2 = log2f(s), h = kLn2 * (l2 - t / s);
        const float lp = (x_tok - m) * in.inv_temperature - kLn2 * l2;
        const PolicyTerms o = policy_terms(pin, adv, old_logp, ref_logp, lp, h);
        griddep_wait();
        const float share = static_cast<float>(w * __ldcg(&terms.totals->inv_weight));
        if (threadIdx.x == 0) {
            sh.row[0] = m; sh.row[1] = l2; sh.row[2] = h;
            sh.row[3] = o.slope * share * in.inv_temperature;
            sh.row[4] = pin.entropy_coef * share * in.inv_temperature;
        }
        if (rank == 0 && threadIdx.x == 0) {
            logp[r] = lp;
            entropy[r] = h;
#pragma unroll
            for (int q = 0; q < 5; ++q) sh.terms[q] = o.v[q] * share;
        }
    }
    __syncthreads();
    const RowCoef coef{sh.row[3], sh.row[4]};
    m = sh.row[0];
    const float l2 = sh.row[1], h = sh.row[2];
    const bool same = ((reinterpret_cast<uintptr_t>(row) ^ reinterpret_cast<uintptr_t>(dst)) & 15) == 0;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int q = base + k * threads;
        if (q >= v.count || !out) break;
        float g[per_vector<GT>()];
        vector_gradient<GT, ENTROPY_GRAD>(x[k], m, l2, in.scale, coef, h, g);
        const long long at = tok - v.first(q);
        if (at >= 0 && at < per_vector<GT>())
#pragma unroll
            for (int j = 0; j < per_vector<GT>(); ++j)
                if (j == at) g[j] += coef.a;
        store_row_vector(v, q, dst, same, g);
    }
    if (rank == 0 && threadIdx.x < 32) {
        const float each[5] = {sh.terms[0], sh.terms[1], sh.terms[2], sh.terms[3], sh.terms[4]};
        count_row(terms, in.rows, r, each);
    }
}

// The terms alone, from statistics already there: no gradient wanted, or rows too long to stay on chip.
static __global__ void __launch_bounds__(256) policy_terms_kernel(const __grid_constant__ RowsIn rows, const __grid_constant__ PolicyIn in,
                                                                  const __grid_constant__ TermsOut terms, const float *logp, const float *entropy, RowCoef *coef)
{
    const long long r = (static_cast<long long>(blockIdx.x) * blockDim.x + threadIdx.x) >> 5;      // one warp a row
    if (r >= rows.rows) return;
    const float w = rows.weights ? rows.weights[r] : 1.f;
    float each[5] = {};
    RowCoef k{0.f, 0.f};
    if (w != 0.f) {
        const PolicyTerms o = policy_terms(in, in.advantages[r], in.old_logp[r], in.ref_logp ? in.ref_logp[r] : 0.f, logp[r], entropy[r]);
        const float share = static_cast<float>(w * terms.totals->inv_weight);
        k.a = o.slope * share * rows.inv_temperature;
        k.b = in.entropy_coef * share * rows.inv_temperature;
        for (int q = 0; q < 5; ++q) each[q] = o.v[q] * share;
    }
    if (coef && (threadIdx.x & 31) == 0) coef[r] = k;
    count_row(terms, rows.rows, r, each);
}

// ---- the preference loss -----------------------------------------------------------------------------------------------------
struct PreferenceIn {
    const long long *offsets;
    const float *ref_logp;
    long long pairs;
    float beta, smoothing;
};

// The row ranges come from the device: whatever they hold, no row outside [0, rows) is touched.
__device__ __forceinline__ void sequence_rows(const PreferenceIn &in, long long k, long long rows, long long &lo, long long &hi)
{
    lo = min(max(in.offsets[k], 0ll), rows);
    hi = min(max(in.offsets[k + 1], lo), rows);
}

constexpr int kPairThreads = 256;

// One block per pair; the block that ends last adds the pairs' terms up in their order.  `done` is zero before and after.
static __global__ void __launch_bounds__(kPairThreads) preference_terms_kernel(const __grid_constant__ RowsIn rows, const __grid_constant__ PreferenceIn in,
                                                                               const float *logp, float *seq_logp, RowCoef *coef, double (*each)[3],
                                                                               unsigned *done, float *stats)
{
    __shared__ double scratch[kPairThreads / 32];
    __shared__ bool finish;
    const long long i = blockIdx.x;
    double pi[2];
    for (int side = 0; side < 2; ++side) {
        long long lo, hi;
        sequence_rows(in, 2 * i + side, rows.rows, lo, hi);
        double s = 0;
        for (long long r = lo + threadIdx.x; r < hi; r += blockDim.x) {
            const float w = rows.weights ? rows.weights[r] : 1.f;
            if (w != 0.f) s += static_cast<double>(w) * logp[r];
        }
        s = block_total(s, scratch);
        if (threadIdx.x == 0) seq_logp[2 * i + side] = static_cast<float>(s);
        pi[side] = s - in.ref_logp[2 * i + side];
    }
    const double margin = in.beta * (pi[0] - pi[1]);
    const double slope = (1.0 / (1.0 + exp(-margin)) - (1.0 - in.smoothing)) * in.beta / static_cast<double>(in.pairs);
    if (coef)
        for (int side = 0; side < 2; ++side) {
            long long lo, hi;
            sequence_rows(in, 2 * i + side, rows.rows, lo, hi);
            for (long long r = lo + threadIdx.x; r < hi; r += blockDim.x) {
                const float w = rows.weights ? rows.weights[r] : 1.f;
                coef[r] = RowCoef{w != 0.f ? static_cast<float>((side ? -slope : slope) * w) * rows.inv_temperature : 0.f, 0.f};
            }
        }
    if (threadIdx.x == 0) {
        const double up = log1p(exp(-fabs(margin)));                       // log(1 + e^-|x|)
        const double loss = (1.0 - in.smoothing) * (up + fmax(-margin, 0.0)) + in.smoothing * (up + fmax(margin, 0.0));
        __stcg(&each[i][0], isnan(margin) ? margin : loss);
        __stcg(&each[i][1], margin > 0.0 ? 1.0 : 0.0);
        __stcg(&each[i][2], margin);
        __threadfence();
        finish = atomicInc(done, gridDim.x - 1) == gridDim.x - 1;
    }
    __syncthreads();
    if (!finish) return;
    __threadfence();
    double sum[3] = {};
    for (long long k = threadIdx.x; k < in.pairs; k += blockDim.x)
#pragma unroll
        for (int q = 0; q < 3; ++q) sum[q] += __ldcg(&each[k][q]);
    for (int q = 0; q < 3; ++q) {
        const double s = block_total(sum[q], scratch);
        if (threadIdx.x == 0) stats[q] = static_cast<float>(s / static_cast<double>(in.pairs));
    }
}

}  // namespace softsync
