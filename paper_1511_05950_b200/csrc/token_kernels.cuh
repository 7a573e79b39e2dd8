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
// exponential unit close behind: it gives 16 results a clock and SM, and at 7 TB/s 12 of them are wanted in either case.
#pragma once

#include "packed.cuh"
#include "update_kernels.cuh"

#include <math_constants.h>

namespace softsync {

constexpr float kLn2 = 0.6931471805599453f;
constexpr float kLowest = -3.402823466e38f;
constexpr float kFloor = -1e30f;          // logits below this have p = 0 beside an ordinary maximum
constexpr unsigned kFloorBits = 0xf149f149u;
constexpr float kFloorBf16 = -0x1.92p99f; // the same in bf16, twice in kFloorBits

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
// ---- 16-byte vectors of a row ------------------------------------------------------------------------------------------
template <typename GT> __host__ __device__ constexpr int logit_bytes() { return sizeof(Raw<GT, 1>); }
template <typename GT> __host__ __device__ constexpr int per_vector() { return 16 / logit_bytes<GT>(); }

__device__ __forceinline__ float logit_at(const GradFp32 *, const unsigned char *row, long long j) { return reinterpret_cast<const float *>(row)[j]; }
__device__ __forceinline__ float logit_at(const GradBf16 *, const unsigned char *row, long long j)
{ return __uint_as_float(static_cast<unsigned>(reinterpret_cast<const unsigned short *>(row)[j]) << 16); }

// A row as vectors: vector q holds the elements [q * per_vector - phase, ...) of the row; those in [inner, full) lie inside it.
template <typename GT>
struct RowVectors {
    const unsigned char *row;
    int phase, vocab, inner, full, count;
    __device__ __forceinline__ RowVectors(const unsigned char *r, int v) : row(r), vocab(v)
    {
        phase = static_cast<int>(reinterpret_cast<uintptr_t>(r) & 15) / logit_bytes<GT>();
        inner = phase ? 1 : 0;
        full = (phase + v) / per_vector<GT>();
        count = (phase + v + per_vector<GT>() - 1) / per_vector<GT>();
    }
    __device__ __forceinline__ int first(int q) const { return q * per_vector<GT>() - phase; }
    __device__ __forceinline__ bool whole(int q) const { return q >= inner && q < full; }
    __device__ __forceinline__ bool ragged() const { return phase != 0 || count != full; }
    __device__ __forceinline__ const unsigned char *at(int q) const { return row - phase * logit_bytes<GT>() + static_cast<long long>(q) * 16; }
};

__device__ __forceinline__ uint4 load_vector16(const void *p)
{
    uint4 r;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(p));
    return r;
}

template <typename GT>
__device__ __forceinline__ uint4 no_vector()               // minus infinity throughout
{
    constexpr unsigned w = logit_bytes<GT>() == 4 ? 0xff800000u : 0xff80ff80u;
    return make_uint4(w, w, w, w);
}


// A vector that reaches beyond the row, element by element; minus infinity out there.
template <typename GT>
__device__ __forceinline__ uint4 load_ragged_vector(const unsigned char *row, int j, int vocab)
{
    uint4 r;
    unsigned *w = &r.x;
    if constexpr (logit_bytes<GT>() == 4) {
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] = j + k >= 0 && j + k < vocab ? reinterpret_cast<const unsigned *>(row)[j + k] : 0xff800000u;
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const unsigned short *h = reinterpret_cast<const unsigned short *>(row);
            const unsigned lo = j + 2 * k >= 0 && j + 2 * k < vocab ? h[j + 2 * k] : 0xff80u;
            const unsigned hi = j + 2 * k + 1 >= 0 && j + 2 * k + 1 < vocab ? h[j + 2 * k + 1] : 0xff80u;
            w[k] = lo | hi << 16;
        }
    }
    return r;
}

// The vectors q0, q0 + T, ... of a row; minus infinity beyond its end.
template <typename GT, int T, int NV>
__device__ __forceinline__ void load_vectors(uint4 (&x)[NV], const RowVectors<GT> &v, int q0)
{
    const unsigned char *p = v.at(q0);
#pragma unroll
    for (int k = 0; k < NV; ++k)
        if (v.whole(q0 + k * T)) x[k] = load_vector16(p + k * T * 16);
        else x[k] = no_vector<GT>();
    if (!v.ragged()) return;
    const int d = v.full - q0;
    if (v.count != v.full && d >= 0 && d < NV * T && d % T == 0) {
        const uint4 end = load_ragged_vector<GT>(v.row, v.first(v.full), v.vocab);
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (d == k * T) x[k] = end;
    }
    if (v.phase && q0 == 0) x[0] = load_ragged_vector<GT>(v.row, -v.phase, v.vocab);
}

template <typename GT>
__device__ __forceinline__ uint4 pack_vector(const float (&g)[per_vector<GT>()])
{
    if constexpr (logit_bytes<GT>() == 4) return make_uint4(__float_as_uint(g[0]), __float_as_uint(g[1]), __float_as_uint(g[2]), __float_as_uint(g[3]));
    else return make_uint4(pack_bf16x2(g[0], g[1]), pack_bf16x2(g[2], g[3]), pack_bf16x2(g[4], g[5]), pack_bf16x2(g[6], g[7]));
}
// A vector's elements one by one, at the row's ends.
template <typename GT>
__device__ __forceinline__ void store_single(unsigned char *dst, int j, int vocab, uint4 packed)
{
    const unsigned *w = &packed.x;
#pragma unroll
    for (int k = 0; k < per_vector<GT>(); ++k)
        if (j + k >= 0 && j + k < vocab) {
            if constexpr (logit_bytes<GT>() == 4) reinterpret_cast<unsigned *>(dst)[j + k] = w[k];
            else reinterpret_cast<unsigned short *>(dst)[j + k] = static_cast<unsigned short>(w[k / 2] >> (16 * (k & 1)));
        }
}
template <typename GT>
__device__ __forceinline__ void store_logit(unsigned char *dst, long long j, float x)
{
    if constexpr (logit_bytes<GT>() == 4) reinterpret_cast<float *>(dst)[j] = x;
    else reinterpret_cast<unsigned short *>(dst)[j] = __bfloat16_as_ushort(__float2bfloat16_rn(x));
}

// Zeros over a whole row by `threads` threads, this one number `me`, by the row's own alignment.
template <typename GT>
__device__ __forceinline__ void zero_row(unsigned char *dst, int vocab, int me, int threads)
{
    const RowVectors<GT> v(dst, vocab);
    const uint4 zero = make_uint4(0, 0, 0, 0);
    for (int q = me; q < v.count; q += threads) {
        if (v.whole(q)) __stcs(reinterpret_cast<uint4 *>(dst + static_cast<long long>(v.first(q)) * logit_bytes<GT>()), zero);
        else store_single<GT>(dst, v.first(q), vocab, zero);
    }
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
        return unpack_bf16(max_nan_bf16x2(w[k], kFloorBits));
}
template <typename GT>
__device__ __forceinline__ float2 plain_pair(const uint4 &x, int k)
{
    const unsigned *w = &x.x;
    if constexpr (logit_bytes<GT>() == 4) return make_float2(__uint_as_float(w[2 * k]), __uint_as_float(w[2 * k + 1]));
    else return unpack_bf16(w[k]);
}

// The vectors' sum of exponentials relative to m and (ENTROPY) of exponentials times exponents, added to s and t.  The difference to m
// is taken before it is scaled: m's own exponent is exactly zero, and a row that a mask of the type's lowest value leaves nothing
// of stays finite (its softmax is uniform).  FLOOR: minus infinity, whose p = 0 times its exponent would be NaN, is held at kFloor.
template <typename GT, int NV, bool ENTROPY, bool FLOOR>
__device__ __forceinline__ void packed_exponentials(const uint4 (&x)[NV], float m, float c, float &s, float &t)
{
    const float2 c2 = make_float2(c, c), m2 = make_float2(-m, -m);
    float2 s2 = make_float2(0.f, 0.f), t2 = s2;
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int k = 0; k < per_vector<GT>() / 2; ++k) {
            const float2 d = mul2(add2(FLOOR ? floored_pair<GT>(x[v], k) : plain_pair<GT>(x[v], k), m2), c2);
            const float2 e = make_float2(ex2(d.x), ex2(d.y));
            s2 = add2(s2, e);
            if constexpr (ENTROPY) t2 = fma2(e, d, t2);
        }
    s += s2.x + s2.y;
    if constexpr (ENTROPY) t += t2.x + t2.y;
}
// Any m, NaN and infinities included: every exponent is held above -1000.
template <typename GT, int NV, bool ENTROPY>
__device__ __forceinline__ void single_exponentials(const uint4 (&x)[NV], float m, float c, float &s, float &t)
{
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

// Takes the vectors into a warp's running sums s, t relative to its m (kLowest to begin with).  Any value of the row serves as m as
// long as nothing above it is far above it, so the maximum is looked for in the first vectors alone; those that follow are added without
// looking, and only where that meets an infinity or a NaN, or a sum past kNearSum, is the maximum looked for again and the sums moved to
// it.  (Looking everywhere costs half an instruction an element, the floor another half.)  An exponent of up to 10 is rounded to 2^-22 at
// most; without the bound a confident token 60 above the first vectors took its row's log probability 4e-6 off, from there 1e-6.
constexpr float kNearSum = 1024.f;
template <typename GT, int NV, bool ENTROPY>
__device__ __forceinline__ void add_vectors(const uint4 (&x)[NV], float c, float &m, float &s, float &t)
{
    if (ordinary(m, c)) {
        float s2 = 0.f, t2 = 0.f;
        packed_exponentials<GT, NV, ENTROPY, false>(x, m, c, s2, t2);
        if (__all_sync(0xffffffffu, s2 < kNearSum && (!ENTROPY || fabsf(t2) < 1e30f))) {
            s += s2;
            if constexpr (ENTROPY) t += t2;
            return;
        }
    }
    const float top = fmaxf(warp_max(vectors_max<GT, NV>(x)), m);
    if (top > m) {
        const float d = fmaxf((m - top) * c, -1000.f), f = ex2(d);
        t = f * fmaf(s, d, t);
        s *= f;
        m = top;
    }
    if (ordinary(m, c)) packed_exponentials<GT, NV, ENTROPY, true>(x, m, c, s, t);
    else single_exponentials<GT, NV, ENTROPY>(x, m, c, s, t);
}

// log2 of a row's sum; NaN, and with it all the row's results, where nothing has a probability (a row of minus infinities) and where
// the token has no logit (NaN in its place).
__device__ __forceinline__ float log2_or_nan(float s, float x_tok) { return s > 0.f && x_tok == x_tok ? log2f(s) : CUDART_NAN_F; }

// What multiplies the exponentials of a part with maximum m in a whole with maximum `top`.
__device__ __forceinline__ float part_factor(float m, float top, float c, float &d)
{
    d = fmaxf((m - top) * c, -1000.f);
    return ex2(d);
}

// Per-row factors of the gradient: dz_j = a (1[j = token] - p_j) + b p_j (log p_j + H).
struct RowCoef { float a, b; };

// What the gradient of a row's elements needs.  With d = (x - m) c - log2 s:  p = 2^d,  g = p (b ln 2 d + (b H - a)).  For bf16 the
// exponent is x c + shift, one instruction less, where the shift is small: its rounding is an error of the exponent that a whole row
// shares, below 1024 at most 2^-15, 1 % of the rounding of a bf16 result (2^-9).  Beyond (large logits, a finite mask over everything, a small
// temperature) the difference to m is taken first, as for fp32: a row of -1e9 had its p 2^34 times too large from the shift.  The rows of
// a well-behaved model never come there: logits of 32 at a temperature of 1 make a shift of 50.
constexpr float kShiftLimit = 1024.f;
struct RowGradient {
    float c, add, mult, one, off, base;                    // the exponent is (x - off) c + base
    bool regular, shifted;                                 // the maximum is ordinary; off is zero: the same for the whole row
    template <typename GT>
    __device__ __forceinline__ RowGradient(const GT *, float m, float l2, float c_, RowCoef k, float entropy)
        : c(c_), add(fmaf(k.b, entropy, -k.a)), mult(k.b * kLn2), one(k.a), regular(ordinary(m, c_))
    {
        const float shift = -fmaf(m, c, l2);
        shifted = logit_bytes<GT>() == 2 && regular && fabsf(shift) < kShiftLimit;
        off = shifted ? 0.f : m;
        base = shifted ? shift : -l2;
    }

    // any maximum, beside an ordinary one with the bits of the vector form; the token's own entry has `one` to be added
    template <typename GT, bool ENTROPY>
    __device__ __forceinline__ float single(float x) const
    {
        constexpr float floor = logit_bytes<GT>() == 4 ? kFloor : kFloorBf16;
        const float y = ENTROPY ? max_nan(x, floor) : x;
        const float d = regular ? fmaf(y - off, c, base) : max_nan((x - off) * c, -1000.f) + base;
        return __fmul_rn(ex2(d), ENTROPY ? fmaf(mult, d, add) : add);
    }
    // beside an ordinary maximum; SHIFT: shifted
    template <typename GT, bool ENTROPY, bool SHIFT>
    __device__ __forceinline__ uint4 vector(const uint4 &x) const
    {
        const float2 c2 = make_float2(c, c), m2 = make_float2(-off, -off), l2 = make_float2(base, base);
        const float2 a2 = make_float2(add, add), b2 = make_float2(mult, mult);
        float g[per_vector<GT>()];
#pragma unroll
        for (int j = 0; j < per_vector<GT>() / 2; ++j) {
            const float2 y = ENTROPY ? floored_pair<GT>(x, j) : plain_pair<GT>(x, j);
            const float2 d = fma2(SHIFT ? y : add2(y, m2), c2, l2);
            const float2 r = mul2(make_float2(ex2(d.x), ex2(d.y)), ENTROPY ? fma2(b2, d, a2) : a2);
            g[2 * j] = r.x;
            g[2 * j + 1] = r.y;
        }
        return pack_vector<GT>(g);
    }
    template <typename GT, bool ENTROPY>
    __device__ __forceinline__ uint4 vector_of(const uint4 &x) const
    {
        if constexpr (logit_bytes<GT>() == 2)
            if (shifted) return vector<GT, ENTROPY, true>(x);
        return vector<GT, ENTROPY, false>(x);
    }
};

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
    float row[6];                         // m, log2 s, entropy, a, b, token's logit: what every thread needs for the gradient
};

// m, s, t of 32 parts, one a lane, become those of the whole in every lane.
__device__ __forceinline__ void join_lanes(float c, float &m, float &s, float &t)
{
    const float top = warp_max(m);
    float d;
    const float f = part_factor(m, top, c, d);
    t = warp_sum(f * fmaf(s, d, t));
    s = warp_sum(f * s);
    m = top;
}

// The block's m, s, t from its warps' (each warp: the same m, and s and t to be summed over its lanes), in every lane of warp 0;
// the other warps get nothing.
__device__ __forceinline__ void join_warps(RowShared &sh, float c, float &m, float &s, float &t)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    s = warp_sum(s);
    t = warp_sum(t);
    if (lane == 0) { sh.warp[0][warp] = m; sh.warp[1][warp] = s; sh.warp[2][warp] = t; }
    __syncthreads();
    if (warp == 0) {
        m = lane < warps ? sh.warp[0][lane] : kLowest;
        s = lane < warps ? sh.warp[1][lane] : 0.f;
        t = lane < warps ? sh.warp[2][lane] : 0.f;
        join_lanes(c, m, s, t);
    }
}

// The same over all blocks of a cluster, which write into one another's shared memory and meet at the cluster's barrier.  The blocks have
// met once before, so that none writes before its peer has started.
__device__ __forceinline__ void join_cluster(RowShared &sh, float c, float &m, float &s, float &t)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const unsigned blocks = cluster_size();
    join_warps(sh, c, m, s, t);
    if (blocks == 1) return;
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
        join_lanes(c, m, s, t);
    }
}

// ---- statistics of a row, in batches -----------------------------------------------------------------------------------------
struct StatsOut {
    float *logp, *lse, *entropy;          // lse, entropy may be null
    RowStat *stat;                        // may be null
    RowCoef *coef;                        // set to zero for the kernel that follows (may be null)
};

// One cluster per row; each thread holds NV vectors of a batch at a time.  A batch's maximum is taken over the whole warp before
// any exponential, so that the running sums are rescaled once a batch and by the same factor in every lane.
//
// One read of the logits bounds it, and behind it the exponential unit and the issue (64 % of its slots).  8192 x 131072 bf16, an
// eighth of the rows without a weight and so not read: 310 to 335 us, 5.6 to 6.1 TB/s with the entropy.  32 x 50257 bf16: 6.6 us, of which
// the launch and two trips to memory are the most; a row is spread over a cluster there, as many blocks as have work.
template <typename GT, int T, int NV, bool ENTROPY>
__global__ void __launch_bounds__(T, 1536 / T) row_stats_kernel(const __grid_constant__ RowsIn in, const __grid_constant__ StatsOut out)
{
    __shared__ RowShared sh;
    const int blocks = cluster_size(), rank = cluster_rank();
    const long long r = blockIdx.x / static_cast<unsigned>(blocks);
    griddep_launch_dependents();
    if (rank == 0 && threadIdx.x == 0 && out.coef) out.coef[r] = RowCoef{0.f, 0.f};
    if (in.weights && in.weights[r] == 0.f) {              // the whole cluster leaves
        if (rank == 0 && threadIdx.x == 0) {
            out.logp[r] = 0.f;
            if (out.lse) out.lse[r] = 0.f;
            if (out.entropy) out.entropy[r] = 0.f;
        }
        return;
    }
    if (blocks > 1) { cluster_arrive(); cluster_wait(); }
    const unsigned char *row = in.data + r * in.stride * logit_bytes<GT>();
    const RowVectors<GT> v(row, static_cast<int>(in.vocab));
    long long tok = -1;
    float x_tok = CUDART_NAN_F;
    if (threadIdx.x == 0) {
        tok = in.tokens[r];
        if (tok >= 0 && tok < in.vocab) x_tok = logit_at(static_cast<const GT *>(nullptr), row, tok);
    }
    float m = kLowest, s = 0.f, t = 0.f;
    for (int base = rank * NV * T; base < v.count; base += blocks * NV * T) {
        uint4 x[NV];
        load_vectors<GT, T, NV>(x, v, base + threadIdx.x);
        add_vectors<GT, NV, ENTROPY>(x, in.scale, m, s, t);
    }
    join_cluster(sh, in.scale, m, s, t);
    if (rank || threadIdx.x) return;
    const float l2 = log2_or_nan(s, x_tok);
    out.logp[r] = (x_tok - m) * in.inv_temperature - kLn2 * l2;
    if (out.lse) out.lse[r] = m * in.inv_temperature + kLn2 * l2;
    if (ENTROPY && out.entropy) out.entropy[r] = kLn2 * (l2 - t / s);
    if (out.stat) out.stat[r] = RowStat{m, l2};
}

// Terms of the pairs of a preference loss, to be added up (stats may be null: nothing to do).
struct PairTail {
    const double (*each)[3];
    long long pairs;
    float *stats;
};

// By one warp, in the pairs' order.
__device__ __forceinline__ void finish_pairs(const PairTail &tail)
{
    double sum[3] = {};
    for (long long k = threadIdx.x; k < tail.pairs; k += 32)
#pragma unroll
        for (int q = 0; q < 3; ++q) sum[q] += __ldcg(&tail.each[k][q]);
#pragma unroll
    for (int q = 0; q < 3; ++q)
        for (int o = 16; o; o >>= 1) sum[q] += __shfl_xor_sync(0xffffffffu, sum[q], o);
    if (threadIdx.x == 0)
        for (int q = 0; q < 3; ++q) tail.stats[q] = static_cast<float>(sum[q] / static_cast<double>(tail.pairs));
}

// ---- gradient from statistics -----------------------------------------------------------------------------------------------
constexpr int kGradThreads = 256, kGradVectors = 4;

// One block per segment of a row, rows from the last to the first: the statistics pass went the other way, so the rows it read
// last, which the L2 still holds, come first.  The logits are on their way before the factors are there.  Reads and writes two
// bytes an element (bf16): 2920 x 131072, a quarter of the rows without a
// weight and so only written, in 200 us (6.7 TB/s).
template <typename GT, bool ENTROPY>
__global__ void __launch_bounds__(kGradThreads, 6) row_grad_kernel(const __grid_constant__ RowsIn in, const RowStat *stat, const RowCoef *coef,
                                                                const float *entropy, unsigned char *out, long long out_stride, int segments, const __grid_constant__ PairTail tail)
{
    constexpr int T = kGradThreads, NV = kGradVectors, PV = per_vector<GT>();
    if (tail.stats && blockIdx.x == 0) {                   // a block of its own
        griddep_wait();
        if (threadIdx.x < 32) finish_pairs(tail);
        return;
    }
    const unsigned block = blockIdx.x - (tail.stats ? 1 : 0);
    const long long r = in.rows - 1 - block / static_cast<unsigned>(segments);
    const int segment = block % static_cast<unsigned>(segments), vocab = static_cast<int>(in.vocab);
    const unsigned char *row = in.data + r * in.stride * logit_bytes<GT>();
    unsigned char *dst = out + r * out_stride * logit_bytes<GT>();
    const RowVectors<GT> v(row, vocab);
    const bool masked = in.weights && in.weights[r] == 0.f;
    const int lo = segment * NV * T, q0 = lo + threadIdx.x;
    uint4 x[NV];
    if (!masked) load_vectors<GT, T, NV>(x, v, q0);
    griddep_wait();                                        // the factors
    const RowCoef k = coef[r];
    if (masked || (k.a == 0.f && k.b == 0.f)) {            // the gradient is zero, whatever the row holds
        zero_row<GT>(dst, vocab, segment * T + threadIdx.x, segments * T);
        return;
    }
    const RowStat st = stat[r];
    const long long tok = in.tokens[r];
    const RowGradient f(static_cast<const GT *>(nullptr), st.max, st.log2_sum, in.scale, k, ENTROPY ? entropy[r] : 0.f);
    if (((reinterpret_cast<uintptr_t>(row) ^ reinterpret_cast<uintptr_t>(dst)) & 15) == 0 && f.regular) {
        const int tok_q = tok >= 0 && tok < vocab ? (static_cast<int>(tok) + v.phase) / PV : -1, tok_j = (static_cast<int>(tok) + v.phase) % PV;
        unsigned char *p = dst - v.phase * logit_bytes<GT>() + static_cast<long long>(q0) * 16;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int q = q0 + i * T;
            if (q >= v.count) break;
            const uint4 g = f.template vector_of<GT, ENTROPY>(x[i]);
            if (v.whole(q)) __stcs(reinterpret_cast<uint4 *>(p + i * T * 16), g);
            else store_single<GT>(dst, v.first(q), vocab, g);
            if (q == tok_q) {                              // the token's entry once more, with its one
#pragma unroll
                for (int j = 0; j < PV; ++j) {
                    const float2 y = plain_pair<GT>(x[i], j / 2);
                    if (j == tok_j) store_logit<GT>(dst, tok, __fadd_rn(f.template single<GT, ENTROPY>(j & 1 ? y.y : y.x), f.one));
                }
            }
        }
    } else {                                               // single elements, one a thread
        const int end = min(v.first(lo + NV * T), vocab);
        for (int j = max(v.first(lo), 0) + threadIdx.x; j < end; j += T) {
            const float g = f.template single<GT, ENTROPY>(logit_at(static_cast<const GT *>(nullptr), row, j));
            store_logit<GT>(dst, j, j == tok ? __fadd_rn(g, f.one) : g);
        }
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

// Sum over the first `threads` threads of a block (all of them call it and meet at `sync`), the same bits in every thread.
template <typename Sync>
__device__ __forceinline__ double block_total(double x, double *scratch, int threads, Sync sync)
{
    for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    sync();
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = x;
    sync();
    double y = 0;
    for (int k = 0; k < threads / 32; ++k) y += scratch[k];
    return y;
}

struct PolicyState {
    double *inv_weight;                   // 1 / sum of the weights, 0 where that is 0
    unsigned *done;                       // parts whose sums are there: zero before and after a call
    double (*part_sum)[5];                // of the rows of each cluster (or block, policy_terms_kernel)
    float *stats;
    int *order, *live;                    // rows with a weight from the front, those without from the back; how many have one (may be null)
};

__device__ __forceinline__ double inverse_or_zero(double sum) { return sum != 0.0 ? 1.0 / sum : 0.0; }

// Sum of the weights, and (st.order) a list of the rows from `from` on that have one, so that they can be dealt out evenly: dealt out as
// they come, some clusters get a tenth to a third more live rows than the mean (4096 x 50257 fp32, a quarter without a weight: 269 us,
// from the list 251; 16384 x 152000 bf16, an eighth without: 1761, 1665; with a weight for every row the list costs 1 to 3 %).
static __global__ void __launch_bounds__(kTermThreads) policy_totals_kernel(const float *weights, long long rows, int from, const __grid_constant__ PolicyState st,
                                                                            float *logp, float *entropy)
{
    constexpr int T = kTermThreads, W = T / 32, N = 8;
    __shared__ double scratch[W];
    __shared__ int before[N * W];                          // live rows of each warp's N groups of 32, then of all groups before
    __shared__ int in_tile;
    griddep_launch_dependents();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    double sum = weights ? 0.0 : static_cast<double>(rows);
    int live = 0;
    for (long long base = 0; weights && base < rows; base += T * N) {
        unsigned alive[N];
        float w[N];
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const long long r = base + j * T + threadIdx.x;
            w[j] = r < rows ? weights[r] : 0.f;
        }
#pragma unroll
        for (int j = 0; j < N; ++j) {
            sum += w[j];
            alive[j] = __ballot_sync(0xffffffffu, w[j] != 0.f && base + j * T + threadIdx.x >= from);
        }
        if (!st.order) continue;
        if (lane == 0)
#pragma unroll
            for (int j = 0; j < N; ++j) before[j * W + warp] = __popc(alive[j]);
        __syncthreads();
        if (warp == 0) {
            int n[N], all = 0;
#pragma unroll
            for (int k = 0; k < N; ++k) { n[k] = all; all += before[lane * N + k]; }
            int upto = all;
            for (int o = 1; o < 32; o <<= 1) {
                const int y = __shfl_up_sync(0xffffffffu, upto, o);
                if (lane >= o) upto += y;
            }
#pragma unroll
            for (int k = 0; k < N; ++k) before[lane * N + k] = upto - all + n[k];
            if (lane == 31) in_tile = upto;
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int r = static_cast<int>(base) + j * T + threadIdx.x, at = live + before[j * W + warp] + __popc(alive[j] & ((1u << lane) - 1u));
            if (r >= rows) break;
            if (r < from) continue;
            if (w[j] != 0.f) st.order[at] = r;
            else {
                st.order[rows - from - 1 - (r - from - at)] = r;
                logp[r] = entropy[r] = 0.f;
            }
        }
        live += in_tile;
        __syncthreads();
    }
    if (weights) sum = block_total(sum, scratch, T, [] { __syncthreads(); });
    if (threadIdx.x == 0) {
        *st.inv_weight = inverse_or_zero(sum);
        if (st.live) *st.live = live;
    }
}

// Called by one warp of each of `parts` parts of the rows, with the part's sums: the one that comes last adds the parts up in their
// order, so the result does not depend on which one that is.
__device__ __forceinline__ void finish_sums(const PolicyState &st, int me, int parts, const double (&sum)[5])
{
    const int lane = threadIdx.x & 31;
    unsigned before = 0;
    if (lane == 0) {
#pragma unroll
        for (int q = 0; q < 5; ++q) __stcg(&st.part_sum[me][q], sum[q]);
        __threadfence();
        before = atomicInc(st.done, parts - 1);           // back to zero by the last one
    }
    if (__shfl_sync(0xffffffffu, before, 0) + 1 != static_cast<unsigned>(parts)) return;
    __threadfence();
#pragma unroll 1
    for (int q = 0; q < 5; ++q) {
        double all = 0;
        for (int k = lane; k < parts; k += 32) all += __ldcg(&st.part_sum[k][q]);
        for (int o = 16; o; o >>= 1) all += __shfl_xor_sync(0xffffffffu, all, o);
        if (lane == 0) st.stats[q] = static_cast<float>(all);
    }
}

// The terms alone, from statistics already there (rows too long to stay on chip): one warp for every gridDim-th row.
static __global__ void __launch_bounds__(32) policy_terms_kernel(const __grid_constant__ RowsIn rows, const __grid_constant__ PolicyIn in,
                                                                 const __grid_constant__ PolicyState st, const float *logp, const float *entropy, RowCoef *coef)
{
    const float inv_weight = static_cast<float>(*st.inv_weight);
    double sum[5] = {};
    for (long long r = blockIdx.x; r < rows.rows; r += gridDim.x) {
        const float w = rows.weights ? rows.weights[r] : 1.f;
        RowCoef k{0.f, 0.f};
        if (w != 0.f) {
            const PolicyTerms o = policy_terms(in, in.advantages[r], in.old_logp[r], in.ref_logp ? in.ref_logp[r] : 0.f, logp[r], entropy[r]);
            const float share = w * inv_weight;
            k.a = o.slope * share * rows.inv_temperature;
            k.b = in.entropy_coef * share * rows.inv_temperature;
            for (int q = 0; q < 5; ++q) sum[q] += static_cast<double>(share) * o.v[q];
        }
        if (coef && threadIdx.x == 0) coef[r] = k;
    }
    finish_sums(st, blockIdx.x, gridDim.x, sum);
}

// ---- the policy loss, rows kept on chip -------------------------------------------------------------------------------------
constexpr int kRingVectors = 4, kRingSlots = 7;
constexpr int kNarrow = 256, kWide = 512;           // threads that do the arithmetic
template <int T>
struct RingShape {
    static constexpr int chunk = T * kRingVectors;  // vectors: 16 or 32 KB
    static constexpr int row = kRingSlots * chunk;  // the most of a row that one block holds
    static constexpr int bytes = row * 16;          // 112 or 224 KB of shared memory
    static constexpr int block = T + 64;            // and two warps more
    static constexpr int per_sm = kWide / T;
};

struct RingPlan {
    int vectors, chunks;                  // of a row, in each block of its cluster
    int ahead;                            // chunks of the next row that fit the ring beside a whole row
    int wait_limit;
};

template <int T>
struct RingShared {
    float warp[3][T / 32];     // each warp's m, s, t
    float part[2][3][kMaxCluster];        // each block's m, s, t by the parity of the row, written by the blocks
    float row[6];                         // m, log2 s, entropy, a, b, token's logit
    int tok;                              // -1 where it is out of range
    float inv_weight;
    double sums[5];                       // of the cluster's rows, kept by its first block
    double scratch[T / 32];
    unsigned long long full[kRingSlots], empty[kRingSlots], exchange[2], ready, go;
};

__device__ __forceinline__ void mbar_arrive(unsigned bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" :: "r"(bar) : "memory"); }
__device__ __forceinline__ void mbar_arrive_remote(const void *mine, unsigned rank)
{
    unsigned addr;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(addr) : "r"(smem_addr(mine)), "r"(rank));
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" :: "r"(addr) : "memory");
}
__device__ __forceinline__ bool mbar_wait_cluster_bounded(unsigned bar, unsigned parity, int limit)
{
    for (int tries = 0; tries < limit; ++tries) {
        unsigned ok;
        asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2, %3;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                     : "=r"(ok) : "r"(bar), "r"(parity), "r"(1000u) : "memory");
        if (ok) return true;
    }
    return false;
}
template <int T>
__device__ __forceinline__ void ring_sync() { asm volatile("bar.sync 1, %0;" :: "n"(T) : "memory"); }

// Statistics, loss terms and gradient (out: null for none) of all rows from one read of the logits: a row is spread over the shared
// memory of a cluster of blocks and stays there between its statistics and its gradient.  Each block has a ring of slots that one thread
// of the copying warp keeps filling with bulk copies, chunk after chunk and row after row.  T threads take a row's statistics chunk by
// chunk as it arrives, and write its gradient, releasing each slot as they go.  In between the joining warp adds up what the
// warps and the cluster's other blocks found, computes the loss terms and the factors, while the T threads already take the statistics
// of the next row's first chunks, as many as the ring has room for beside the whole row.  The clusters are as many as fit the GPU, each
// takes every parts-th row.
//
// A vector at a row's ragged end comes with ordinary loads, through a register of the thread that handles it (the last thread the
// front's, the first thread the end's: never the same one).
//
// What bounds it: one read and one write of two bytes an element go at 5.1 to 5.6 TB/s of algorithmic bytes in bf16 (16384 x 32000: 400 us;
// 8192 x 131072: 770; 8192 x 152000: 929) and 6.0 in fp32 (4096 x 128000: 704), with 57 % of the issue slots, 58 % of the DRAM's
// cycles and two thirds of the exponential unit's busy at 152000: 16 warps an SM are too few to fill one of them, and the rows'
// bytes leave no room for more.  Of the forms tried (256 threads x 4 vectors x 7 slots x 2 blocks an SM, 128 x 8, 192 x 4 x 9, 384 x 2 x 9, 512 x
// 2; one block of 256, 384 and 512) these two were the fastest.
//
// Every wait is bounded.  One that runs out makes the block's later rows NaN; it waits for nothing after that, but the copying thread
// still sees, with a limit, its last copies arrive.
template <typename GT, bool ENTROPY_GRAD, int T>
__global__ void __launch_bounds__(RingShape<T>::block, RingShape<T>::per_sm) policy_ring_kernel(const __grid_constant__ RowsIn in, const __grid_constant__ PolicyIn pin,
                                                                    const __grid_constant__ PolicyState st, float *logp, float *entropy,
                                                                    unsigned char *out, long long out_stride, const __grid_constant__ RingPlan plan)
{
    constexpr int NV = kRingVectors, PV = per_vector<GT>(), kRingChunk = RingShape<T>::chunk;
    extern __shared__ __align__(128) unsigned char ring[];
    __shared__ RingShared<T> sh;
    const int blocks = cluster_size(), rank = cluster_rank(), tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int parts = gridDim.x / static_cast<unsigned>(blocks), vocab = static_cast<int>(in.vocab);
    const int r0 = static_cast<int>(blockIdx.x / static_cast<unsigned>(blocks)), lo = rank * plan.vectors;
    if (tid == 0) {
        for (int k = 0; k < kRingSlots; ++k) { mbar_init(smem_addr(&sh.full[k]), 1); mbar_init(smem_addr(&sh.empty[k]), T / 32); }
        for (int k = 0; k < 2; ++k) mbar_init(smem_addr(&sh.exchange[k]), blocks);
        mbar_init(smem_addr(&sh.ready), T / 32);
        mbar_init(smem_addr(&sh.go), 1);
        for (int k = 0; k < 5; ++k) sh.sums[k] = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    cluster_arrive();
    cluster_wait();                                        // every block's barriers are there
    const auto row_at = [&](long long r) { return in.data + r * in.stride * logit_bytes<GT>(); };
    // Each cluster begins with the row of its own number, if that has a weight, and goes on with every parts-th of the others: of a list of
    // those that have one, which the kernel before this one makes meanwhile, or, where nothing has weights, of all.
    const bool listed = st.order != nullptr;
    const int rows = static_cast<int>(in.rows);
    int live = 0;                                          // rows on the list
    const auto open_list = [&] { if (listed) { griddep_wait(); live = __ldcg(st.live); } };
    const auto row_of = [&](int i) { return listed ? (i - parts < live ? __ldcg(st.order + (i - parts)) : -1) : i < rows ? i : -1; };
    const float w_first = in.weights ? in.weights[r0] : 1.f;

    if (warp == T / 32) {                                  // the copying warp
        if (lane == 0) {
            unsigned g = 0;                                // chunks issued
            bool late = false;
            for (int i = r0, r = r0; r >= 0 && !late; i += parts) {
                int next = i > r0 ? row_of(i + parts) : -1;
                const bool dead = i == r0 && w_first == 0.f;
                const RowVectors<GT> v(row_at(r), vocab);
                const int hi = min(lo + plan.vectors, v.full);
                for (int c = 0; c < plan.chunks && !dead; ++c, ++g) {
                    const unsigned slot = g % kRingSlots, round = g / kRingSlots;
                    if (round && !mbar_wait_bounded(smem_addr(&sh.empty[slot]), (round - 1) & 1, plan.wait_limit)) { late = true; break; }
                    const int from = max(lo + c * kRingChunk, v.inner), to = min(lo + (c + 1) * kRingChunk, hi), n = max(to - from, 0);
                    mbar_expect_tx(smem_addr(&sh.full[slot]), n * 16);
                    if (n) bulk_load(smem_addr(ring + (static_cast<size_t>(slot) * kRingChunk + (from - lo - c * kRingChunk)) * 16), v.at(from), n * 16, smem_addr(&sh.full[slot]));
                }
                if (i == r0) {
                    open_list();
                    next = row_of(i + parts);
                }
                r = next;
            }
            for (unsigned k = g > kRingSlots ? g - kRingSlots : 0; k < g; ++k)      // nothing may arrive after the block has gone
                mbar_wait_bounded(smem_addr(&sh.full[k % kRingSlots]), (k / kRingSlots) & 1, plan.wait_limit);
        }
        __syncwarp();
    } else if (warp > T / 32) {                            // the joining warp
        int i = r0, r = r0;
        long long tok = 0;
        float w = w_first, x_tok = 0.f, adv = 0.f, old_logp = 0.f, ref_logp = 0.f;
        const auto fetch = [&] {                           // what belongs to the row beside its logits
            tok = in.tokens[r];
            adv = pin.advantages[r];
            old_logp = pin.old_logp[r];
            ref_logp = pin.ref_logp ? pin.ref_logp[r] : 0.f;
            x_tok = tok >= 0 && tok < in.vocab ? logit_at(static_cast<const GT *>(nullptr), row_at(r), tok) : CUDART_NAN_F;
        };
        const auto step = [&] {
            i += parts;
            r = row_of(i);
            if (r < 0) return;
            w = in.weights ? in.weights[r] : 1.f;
            fetch();
        };
        fetch();
        open_list();
        float inv_weight = listed ? static_cast<float>(__ldcg(st.inv_weight)) : 0.f;
        if (w == 0.f) {
            if (rank == 0 && lane == 0) { logp[r] = 0.f; entropy[r] = 0.f; }
            step();
        }
        bool late = false;
        for (unsigned turn = 0; r >= 0; ++turn) {
            late = late || !mbar_wait_bounded(smem_addr(&sh.ready), turn & 1, plan.wait_limit);
            if (!listed) inv_weight = sh.inv_weight;
            float m = lane < T / 32 ? sh.warp[0][lane] : kLowest, s = lane < T / 32 ? sh.warp[1][lane] : 0.f, t = lane < T / 32 ? sh.warp[2][lane] : 0.f;
            join_lanes(in.scale, m, s, t);
            if (blocks > 1) {
                const unsigned parity = turn & 1;
                if (lane < blocks) {
                    store_to_rank(&sh.part[parity][0][rank], lane, m);
                    store_to_rank(&sh.part[parity][1][rank], lane, s);
                    store_to_rank(&sh.part[parity][2][rank], lane, t);
                    mbar_arrive_remote(&sh.exchange[parity], lane);
                }
                late = late || !mbar_wait_cluster_bounded(smem_addr(&sh.exchange[parity]), (turn >> 1) & 1, plan.wait_limit);
                m = lane < blocks ? sh.part[parity][0][lane] : kLowest;
                s = lane < blocks ? sh.part[parity][1][lane] : 0.f;
                t = lane < blocks ? sh.part[parity][2][lane] : 0.f;
                join_lanes(in.scale, m, s, t);
            }
            if (late) s = CUDART_NAN_F;
            const float l2 = log2_or_nan(s, x_tok), h = kLn2 * (l2 - t / s);
            const float lp = (x_tok - m) * in.inv_temperature - kLn2 * l2;
            const PolicyTerms o = policy_terms(pin, adv, old_logp, ref_logp, lp, h);
            const float share = w * inv_weight;
            if (lane == 0) {
                sh.row[0] = m; sh.row[1] = l2; sh.row[2] = h; sh.row[5] = x_tok;
                sh.row[3] = o.slope * share * in.inv_temperature;
                sh.row[4] = pin.entropy_coef * share * in.inv_temperature;
                sh.tok = tok >= 0 && tok < in.vocab ? static_cast<int>(tok) : -1;
                mbar_arrive(smem_addr(&sh.go));
                if (rank == 0) {
                    logp[r] = lp;
                    entropy[r] = h;
#pragma unroll
                    for (int k = 0; k < 5; ++k) sh.sums[k] += static_cast<double>(share) * o.v[k];
                }
            }
            __syncwarp();
            step();
        }
        if (rank == 0) finish_sums(st, r0, parts, sh.sums);
    } else {
        if (!listed) {
            double sum = in.weights ? 0.0 : static_cast<double>(in.rows);
            if (in.weights) {
                for (int i = tid; i < rows; i += T) sum += in.weights[i];
                sum = block_total(sum, sh.scratch, T, ring_sync<T>);
            }
            if (tid == 0) sh.inv_weight = static_cast<float>(inverse_or_zero(sum));
        }
        const auto clear = [&](int r) { if (out) zero_row<GT>(out + r * out_stride * logit_bytes<GT>(), vocab, rank * T + tid, blocks * T); };
        int i = r0, r = r0, next = -1, dead = r0;          // dead: place among the listed rows without a weight
        const auto step = [&] {
            if (i == r0) {
                open_list();
                next = row_of(i + parts);
            }
            i += parts;
            r = next;
            next = row_of(i + parts);
        };
        const auto clear_listed = [&](int upto) {
            for (; listed && dead < rows - parts - live && dead < upto; dead += parts) clear(__ldcg(st.order + (rows - parts - 1 - dead)));
        };
        const auto advance = [](int &k) { if (++k == kRingSlots) { k = 0; return 1u; } return 0u; };
        if (w_first == 0.f) {
            clear(r);
            step();
        }
        int due = r;                                 // the row whose gradient comes next; r: it or the next, whose statistics are taken
        float m = kLowest, s = 0.f, t = 0.f;
        int c = 0, here = 0, slot = 0;                     // r's next chunk and its slot; the slot of the gradient's next chunk
        unsigned ph = 0, turn = 0;
        bool late = false;
        uint4 edge[1];
        int edge_q = -1;
        while (due >= 0) {
            {
                const RowVectors<GT> v(row_at(r), vocab);
                const int hi = min(lo + plan.vectors, v.full);          // vectors of the block that are in the ring: [max(lo, inner), hi)
                const bool clean = lo >= v.inner;          // no ragged front in the block's first chunk
                const int until = r == due ? plan.chunks : plan.ahead;
                for (int left = hi - lo - c * kRingChunk; c < until; ++c, left -= kRingChunk) {
                    late = late || !mbar_wait_bounded(smem_addr(&sh.full[here]), ph, plan.wait_limit);
                    const uint4 *mine = reinterpret_cast<const uint4 *>(ring) + here * kRingChunk + tid;
                    if (left > T * NV / 2) {
                        uint4 x[NV];
#pragma unroll
                        for (int k = 0; k < NV; ++k) x[k] = mine[k * T];
                        if (left < kRingChunk)
#pragma unroll
                            for (int k = 0; k < NV; ++k)
                                if (k * T + tid >= left) x[k] = no_vector<GT>();
                        if (c == 0 && !clean && tid == 0) x[0] = no_vector<GT>();
                        add_vectors<GT, NV, true>(x, in.scale, m, s, t);
                    } else {
                        for (int k = 0; k * T < left; ++k) {
                            uint4 x[1] = {no_vector<GT>()};
                            if (k * T + tid < left && (c > 0 || k * T + tid > 0 || clean)) x[0] = mine[k * T];
                            add_vectors<GT, 1, true>(x, in.scale, m, s, t);
                        }
                    }
                    ph ^= advance(here);
                }
                if (r == due) {
                    edge_q = -1;
                    if (v.ragged()) {
                        if (v.phase && v.full && lo == 0 && tid == T - 1) edge_q = 0;
                        if (v.count != v.full && v.full >= lo && v.full < lo + plan.vectors && tid == 0) edge_q = v.full;
                        edge[0] = edge_q >= 0 ? load_ragged_vector<GT>(v.row, v.first(edge_q), vocab) : no_vector<GT>();
                        if (__any_sync(0xffffffffu, edge_q >= 0)) add_vectors<GT, 1, true>(edge, in.scale, m, s, t);
                    }
                    if (late) s = CUDART_NAN_F;
                    s = warp_sum(s);
                    t = warp_sum(t);
                    if (lane == 0) {
                        sh.warp[0][warp] = m; sh.warp[1][warp] = s; sh.warp[2][warp] = t;
                        mbar_arrive(smem_addr(&sh.ready));
                    }
                    step();
                    clear_listed(dead + 1);                // one of the rows without a weight, while the row is joined
                    c = 0;
                    m = kLowest; s = 0.f; t = 0.f;
                    if (r >= 0 && plan.ahead > 0) continue;
                }
            }
            late = late || !mbar_wait_bounded(smem_addr(&sh.go), turn & 1, plan.wait_limit);
            ++turn;
            const RowGradient f(static_cast<const GT *>(nullptr), sh.row[0], late ? CUDART_NAN_F : sh.row[1], in.scale, RowCoef{sh.row[3], sh.row[4]}, sh.row[2]);
            const int tok = sh.tok;
            const RowVectors<GT> v(row_at(due), vocab);
            const int hi = min(lo + plan.vectors, v.full);
            const bool clean = lo >= v.inner;
            unsigned char *dst = out + static_cast<long long>(due) * out_stride * logit_bytes<GT>();
            const bool plain = ((reinterpret_cast<uintptr_t>(v.row) ^ reinterpret_cast<uintptr_t>(dst)) & 15) == 0 && f.regular;
            constexpr bool kShift = logit_bytes<GT>() == 2;
            const bool shifted = !kShift || f.shifted;     // a whole chunk of such a row saves the subtraction
            unsigned char *p = dst - v.phase * logit_bytes<GT>() + static_cast<long long>(lo + tid) * 16;
            for (int left = hi - lo, k = 0; k < plan.chunks; ++k, left -= kRingChunk) {
                const uint4 *mine = reinterpret_cast<const uint4 *>(ring) + slot * kRingChunk + tid;
                if (out && plain) {
                    if (shifted && left >= kRingChunk && (k > 0 || clean)) {
#pragma unroll
                        for (int q = 0; q < NV; ++q) __stcs(reinterpret_cast<uint4 *>(p + q * T * 16), f.template vector<GT, ENTROPY_GRAD, kShift>(mine[q * T]));
                    } else {
#pragma unroll
                        for (int q = 0; q < NV; ++q)
                            if (q * T + tid < left && (k > 0 || q * T + tid > 0 || clean))
                                __stcs(reinterpret_cast<uint4 *>(p + q * T * 16), f.template vector<GT, ENTROPY_GRAD, false>(mine[q * T]));
                    }
                    p += kRingChunk * 16;
                } else if (out) {
                    const unsigned char *bytes = ring + slot * kRingChunk * 16;
                    const int base = lo + k * kRingChunk, first = v.first(base), begin = v.first(max(base, v.inner)), end = v.first(min(base + kRingChunk, hi));
                    for (int j = begin + tid; j < end; j += T) {
                        const float x = f.template single<GT, ENTROPY_GRAD>(logit_at(static_cast<const GT *>(nullptr), bytes, j - first));
                        store_logit<GT>(dst, j, j == tok ? __fadd_rn(x, f.one) : x);
                    }
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_addr(&sh.empty[slot]));
                advance(slot);
            }
            if (out && plain && tok >= 0) {                // the token's entry once more, with its one, by the thread that has just written it
                const int q = (tok + v.phase) / PV;
                if (q >= max(lo, v.inner) && q < hi && (q - lo) % T == tid)
                    store_logit<GT>(dst, tok, __fadd_rn(f.template single<GT, ENTROPY_GRAD>(sh.row[5]), f.one));
            }
            if (out && edge_q >= 0) {                      // the row's own elements of a ragged vector
                const int j0 = v.first(edge_q);
                const unsigned char *bytes = reinterpret_cast<const unsigned char *>(&edge[0]);
#pragma unroll
                for (int k = 0; k < PV; ++k) {
                    const int j = j0 + k;
                    if (j < 0 || j >= vocab) continue;
                    const float y = logit_at(static_cast<const GT *>(nullptr), bytes, k);
                    const float x = f.template single<GT, ENTROPY_GRAD>(y);
                    store_logit<GT>(dst, j, j == tok ? __fadd_rn(x, f.one) : x);
                }
            }
            __syncwarp();                                  // the row's shared values are read: lane 0 may tell of the next row
            due = r;
        }
        clear_listed(rows);
    }
    cluster_arrive();
    cluster_wait();                                        // no block goes while another may write to it
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

constexpr int kPairThreads = 256, kSideThreads = kPairThreads / 2;

// One block per pair, half of it for each sequence.  The pairs' terms are added up in their order by the gradient's kernel, which runs
// next, or (stats not null) by the block that ends last here; `done` is zero before and after.  A few microseconds of latency between the two large passes, whatever the sizes.
static __global__ void __launch_bounds__(kPairThreads) preference_terms_kernel(const __grid_constant__ RowsIn rows, const __grid_constant__ PreferenceIn in,
                                                                               const float *logp, float *seq_logp, RowCoef *coef, double (*each)[3],
                                                                               unsigned *done, float *stats)
{
    __shared__ double scratch[kPairThreads / 32];
    __shared__ bool finish;
    griddep_launch_dependents();
    const long long i = blockIdx.x;
    const int side = threadIdx.x / kSideThreads, me = threadIdx.x % kSideThreads;
    long long lo, hi;
    sequence_rows(in, 2 * i + side, rows.rows, lo, hi);
    const double ref = static_cast<double>(in.ref_logp[2 * i]) - static_cast<double>(in.ref_logp[2 * i + 1]);
    // Weights come eight at a time, the first ones before the statistics are there (two pairs of
    // 1024 rows: 7.0 us, one at a time 14.3).
    constexpr int N = 8;
    float w[N];
    const auto weights = [&](long long r0) {
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const long long r = r0 + k * kSideThreads;
            w[k] = r >= hi ? 0.f : rows.weights ? rows.weights[r] : 1.f;
        }
    };
    weights(lo + me);
    griddep_wait();                                        // the statistics
    double s = 0;
    for (long long r0 = lo + me; r0 < hi; r0 += N * kSideThreads) {
        if (r0 != lo + me) weights(r0);
        float x[N];
#pragma unroll
        for (int k = 0; k < N; ++k) x[k] = r0 + k * kSideThreads < hi ? logp[r0 + k * kSideThreads] : 0.f;       // zero for a row without a weight
#pragma unroll
        for (int k = 0; k < N; ++k) s += static_cast<double>(w[k]) * x[k];
    }
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = s;
    __syncthreads();
    double pi[2] = {0, 0};
    for (int k = 0; k < kPairThreads / 32; ++k) pi[k / (kSideThreads / 32)] += scratch[k];
    if (me == 0) seq_logp[2 * i + side] = static_cast<float>(pi[side]);
    const float margin = static_cast<float>(static_cast<double>(in.beta) * ((pi[0] - pi[1]) - ref));
    if (threadIdx.x == 0) {
        const float up = log1pf(expf(-fabsf(margin)));                     // log(1 + e^-|x|)
        const float loss = (1.f - in.smoothing) * (up + fmaxf(-margin, 0.f)) + in.smoothing * (up + fmaxf(margin, 0.f));
        __stcg(&each[i][0], static_cast<double>(isnan(margin) ? margin : loss));
        __stcg(&each[i][1], margin > 0.f ? 1.0 : 0.0);
        __stcg(&each[i][2], static_cast<double>(margin));
        if (stats) {
            __threadfence();
            finish = atomicInc(done, gridDim.x - 1) == gridDim.x - 1;
        }
    }
    if (coef) {
        // sigmoid(margin) - (1 - s), written so that nothing cancels: the difference itself has no digits left at a margin of 17
        const float up_s = 1.f / (1.f + expf(-margin)), down_s = 1.f / (1.f + expf(margin));
        const float slope = (in.smoothing * up_s - (1.f - in.smoothing) * down_s) * in.beta / static_cast<float>(in.pairs);
        for (long long r0 = lo + me; r0 < hi; r0 += N * kSideThreads) {
            if (hi - lo > N * kSideThreads) weights(r0);
#pragma unroll
            for (int k = 0; k < N; ++k)
                if (r0 + k * kSideThreads < hi)
                    coef[r0 + k * kSideThreads] = RowCoef{w[k] != 0.f ? (side ? -slope : slope) * w[k] * rows.inv_temperature : 0.f, 0.f};
        }
    }
    if (!stats) return;
    __syncthreads();
    if (!finish || threadIdx.x >= 32) return;
    __threadfence();
    finish_pairs(PairTail{each, in.pairs, stats});
}

}  // namespace softsync
