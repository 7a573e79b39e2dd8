// Kernels over rows of logits: softmax statistics of a row, the per-token terms of the losses, gradients.
//
// A row's statistics are its maximum m (in the logits' own units), the sum of 2^((x - m) c) with c = log2(e) / T, and the sum of
// that times (x - m) c, from which log probability, log normaliser and entropy follow:
//     lse = m / T + ln 2 log2(s),    H = ln 2 (log2(s) - t / s),    p_j = 2^((x_j - m) c - log2(s)).
// Taking the difference to the maximum before scaling keeps rows whose every entry is the type's lowest value (a mask that
// leaves nothing) finite: their differences are zero, and the softmax is uniform.
#pragma once

#include "update_kernels.cuh"

#include <math_constants.h>

namespace softsync {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kLowest = -3.402823466e38f;

struct RowsIn {
    const unsigned char *data;
    long long rows, vocab, stride;        // stride in elements
    const long long *tokens;
    const float *weights;                 // nullptr: ones
    float scale;                          // log2(e) / T
    float inv_temperature;
};

// What a row leaves for the gradient pass.
struct RowStat { float max, log2_sum; };

__device__ __forceinline__ float max_nan(float a, float b)             // NaN if either is
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// Running statistics; `add` keeps the sums relative to the running maximum.  The floor on d turns exp2's argument of minus infinity
// (p = 0) into a finite one, so that 0 * d is 0; NaN passes through it.
struct Softmax {
    float m = kLowest, s = 0.f, t = 0.f;
    __device__ __forceinline__ void add(float x, float c)
    {
        if (x > m) {
            const float d = fmaxf((m - x) * c, -1000.f), f = exp2f(d);
            t = f * (t + s * d);
            s *= f;
            m = x;
        }
        const float d = max_nan((x - m) * c, -1000.f), e = exp2f(d);
        s += e;
        t = fmaf(e, d, t);
    }
    __device__ __forceinline__ void join(float m2, float s2, float t2, float c)
    {
        const float top = fmaxf(m, m2);
        const float d1 = fmaxf((m - top) * c, -1000.f), d2 = fmaxf((m2 - top) * c, -1000.f);
        const float f1 = exp2f(d1), f2 = exp2f(d2);
        t = f1 * (t + s * d1) + f2 * (t2 + s2 * d2);
        s = s * f1 + s2 * f2;
        m = top;
    }
};

__device__ __forceinline__ float load_logit(const GradFp32 *, const unsigned char *row, long long j) { return reinterpret_cast<const float *>(row)[j]; }
__device__ __forceinline__ float load_logit(const GradBf16 *, const unsigned char *row, long long j)
{ return __uint_as_float(static_cast<unsigned>(reinterpret_cast<const unsigned short *>(row)[j]) << 16); }
__device__ __forceinline__ void store_logit(const GradFp32 *, unsigned char *row, long long j, float x) { reinterpret_cast<float *>(row)[j] = x; }
__device__ __forceinline__ void store_logit(const GradBf16 *, unsigned char *row, long long j, float x)
{ reinterpret_cast<unsigned short *>(row)[j] = __bfloat16_as_ushort(__float2bfloat16_rn(x)); }
template <typename GT> __device__ __forceinline__ constexpr int logit_bytes() { return sizeof(Raw<GT, 1>); }

// One block per row.
template <typename GT>
__global__ void __launch_bounds__(512) row_stats_kernel(const __grid_constant__ RowsIn in, float *logp, float *lse, float *entropy, RowStat *stat)
{
    __shared__ float sm[16], ss[16], st[16];
    const long long r = blockIdx.x;
    const GT *tag = nullptr;
    if (in.weights && in.weights[r] == 0.f) {
        if (threadIdx.x == 0) {
            logp[r] = 0.f;
            if (lse) lse[r] = 0.f;
            if (entropy) entropy[r] = 0.f;
        }
        return;
    }
    const unsigned char *row = in.data + r * in.stride * logit_bytes<GT>();
    Softmax a;
    for (long long j = threadIdx.x; j < in.vocab; j += blockDim.x) a.add(load_logit(tag, row, j), in.scale);
    for (int o = 16; o; o >>= 1)
        a.join(__shfl_xor_sync(0xffffffffu, a.m, o), __shfl_xor_sync(0xffffffffu, a.s, o), __shfl_xor_sync(0xffffffffu, a.t, o), in.scale);
    if ((threadIdx.x & 31) == 0) { sm[threadIdx.x >> 5] = a.m; ss[threadIdx.x >> 5] = a.s; st[threadIdx.x >> 5] = a.t; }
    __syncthreads();
    if (threadIdx.x) return;
    for (int k = 1; k < static_cast<int>(blockDim.x >> 5); ++k) a.join(sm[k], ss[k], st[k], in.scale);
    const float l2 = log2f(a.s);
    const long long tok = in.tokens[r];
    const float x = tok >= 0 && tok < in.vocab ? load_logit(tag, row, tok) : CUDART_NAN_F;
    logp[r] = (x - a.m) * in.inv_temperature - kLn2 * l2;
    if (lse) lse[r] = a.m * in.inv_temperature + kLn2 * l2;
    if (entropy) entropy[r] = kLn2 * (l2 - a.t / a.s);
    if (stat) stat[r] = RowStat{a.m, l2};
}

// Per-row factors of the gradient: dz_j = a (1[j = token] - p_j) + b p_j (log p_j + H).
struct RowCoef { float a, b; };

template <typename GT>
__global__ void __launch_bounds__(512) row_grad_kernel(const __grid_constant__ RowsIn in, const RowStat *stat, const RowCoef *coef,
                                                       const float *entropy, unsigned char *out, long long out_stride)
{
    const long long r = blockIdx.x;
    const GT *tag = nullptr;
    const unsigned char *row = in.data + r * in.stride * logit_bytes<GT>();
    unsigned char *dst = out + r * out_stride * logit_bytes<GT>();
    const RowCoef k = coef[r];
    if ((in.weights && in.weights[r] == 0.f) || (k.a == 0.f && k.b == 0.f)) {        // nothing to read: the gradient is zero
        for (long long j = threadIdx.x; j < in.vocab; j += blockDim.x) store_logit(tag, dst, j, 0.f);
        return;
    }
    const RowStat s = stat[r];
    const float h = k.b != 0.f ? entropy[r] : 0.f;
    const long long tok = in.tokens[r];
    for (long long j = threadIdx.x; j < in.vocab; j += blockDim.x) {
        const float d = max_nan((load_logit(tag, row, j) - s.max) * in.scale, -1000.f) - s.log2_sum;
        const float p = exp2f(d);
        float g = -k.a * p;
        if (k.b != 0.f) g = fmaf(k.b * p, fmaf(kLn2, d, h), g);
        if (j == tok) g += k.a;
        store_logit(tag, dst, j, g);
    }
}

// ---- per-token terms ---------------------------------------------------------------------------------------------------
constexpr int kTermThreads = 1024;

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

struct PolicyIn {
    const float *old_logp, *advantages, *ref_logp;
    float low, high, kl_coef, entropy_coef;            // low = 1 - clip_low, high = 1 + clip_high
};

// One token's terms: {loss, clipped term, KL, entropy, clipped} and the slope dl / dlogp.
struct PolicyTerms { float v[5], slope; };
__device__ __forceinline__ PolicyTerms policy_terms(const PolicyIn &in, long long r, float logp, float entropy)
{
    const float adv = in.advantages[r];
    const float ratio = expf(logp - in.old_logp[r]);
    const float free_ = ratio * adv, held = fminf(max_nan(ratio, in.low), in.high) * adv;
    const bool clipped = free_ > held;
    PolicyTerms o;
    o.v[1] = clipped ? -held : -free_;
    o.slope = clipped ? 0.f : -free_;
    o.v[2] = 0.f;
    if (in.ref_logp) {
        const float d = in.ref_logp[r] - logp, e = expm1f(d);
        o.v[2] = e - d;
        o.slope -= in.kl_coef * e;
    }
    o.v[0] = o.v[1] + in.kl_coef * o.v[2] - in.entropy_coef * entropy;
    o.v[3] = entropy;
    o.v[4] = clipped ? 1.f : 0.f;
    return o;
}

static __global__ void __launch_bounds__(kTermThreads) policy_terms_kernel(const __grid_constant__ RowsIn rows, const __grid_constant__ PolicyIn in,
                                                                           const float *logp, const float *entropy, RowCoef *coef, float *stats)
{
    __shared__ double scratch[kTermThreads / 32];
    double total = 0;
    for (long long r = threadIdx.x; r < rows.rows; r += blockDim.x) total += rows.weights ? rows.weights[r] : 1.f;
    total = block_total(total, scratch);
    const double inv = total != 0.0 ? 1.0 / total : 0.0;
    double sum[5] = {};
    for (long long r = threadIdx.x; r < rows.rows; r += blockDim.x) {
        const float w = rows.weights ? rows.weights[r] : 1.f;
        RowCoef k{0.f, 0.f};
        if (w != 0.f) {
            const PolicyTerms o = policy_terms(in, r, logp[r], entropy[r]);
            const float share = static_cast<float>(w * inv);
            k.a = o.slope * share * rows.inv_temperature;
            k.b = in.entropy_coef * share * rows.inv_temperature;
            for (int q = 0; q < 5; ++q) sum[q] += static_cast<double>(share) * o.v[q];
        }
        if (coef) coef[r] = k;
    }
    for (int q = 0; q < 5; ++q) {
        const double s = block_total(sum[q], scratch);
        if (threadIdx.x == 0) stats[q] = static_cast<float>(s);
    }
}

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

static __global__ void __launch_bounds__(kTermThreads) preference_terms_kernel(const __grid_constant__ RowsIn rows, const __grid_constant__ PreferenceIn in,
                                                                               const float *logp, float *seq_logp, RowCoef *coef, float *stats)
{
    __shared__ double scratch[kTermThreads / 32];
    double sum[3] = {};
    for (long long i = 0; i < in.pairs; ++i) {
        double pi[2], total[2];
        for (int side = 0; side < 2; ++side) {
            long long lo, hi;
            sequence_rows(in, 2 * i + side, rows.rows, lo, hi);
            double s = 0;
            for (long long r = lo + threadIdx.x; r < hi; r += blockDim.x) {
                const float w = rows.weights ? rows.weights[r] : 1.f;
                if (w != 0.f) s += static_cast<double>(w) * logp[r];
            }
            total[side] = block_total(s, scratch);
            if (threadIdx.x == 0) seq_logp[2 * i + side] = static_cast<float>(total[side]);
            pi[side] = total[side] - in.ref_logp[2 * i + side];
        }
        const double margin = in.beta * (pi[0] - pi[1]);
        const double up = log1p(exp(-fabs(margin)));                       // log(1 + e^-|x|)
        const double loss = (1.0 - in.smoothing) * (up + fmax(-margin, 0.0)) + in.smoothing * (up + fmax(margin, 0.0));
        sum[0] += isnan(margin) ? margin : loss;
        sum[1] += margin > 0.0 ? 1.0 : 0.0;
        sum[2] += margin;
        const double slope = (1.0 / (1.0 + exp(-margin)) - (1.0 - in.smoothing)) * in.beta / static_cast<double>(in.pairs);
        for (int side = 0; side < 2; ++side) {
            long long lo, hi;
            sequence_rows(in, 2 * i + side, rows.rows, lo, hi);
            if (coef)
                for (long long r = lo + threadIdx.x; r < hi; r += blockDim.x) {
                    const float w = rows.weights ? rows.weights[r] : 1.f;
                    coef[r] = RowCoef{w != 0.f ? static_cast<float>((side ? -slope : slope) * w) * rows.inv_temperature : 0.f, 0.f};
                }
        }
    }
    if (threadIdx.x == 0)
        for (int q = 0; q < 3; ++q) stats[q] = in.pairs ? static_cast<float>(sum[q] / static_cast<double>(in.pairs)) : 0.f;
}

}  // namespace softsync
