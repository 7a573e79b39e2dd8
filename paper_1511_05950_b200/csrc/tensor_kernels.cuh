// Kernels over a list of tensors: global norm of a weighted sum of gradients, AdamW with moments in 32 or 8 bits.
//
// The list's elements are cut into chunks of kChunk elements, none of which spans two tensors; a table says which tensor a chunk
// belongs to.  AdamW takes a chunk with a block of two warps, each of which owns kStateBlock = 256 consecutive elements, eight a
// lane: exactly one block of 8-bit moments, so a block's largest value is one warp reduction and needs neither shared memory nor
// a second pass.  The norm takes runs of chunks.
//
// Every pass touches every byte once and is bound by HBM: AdamW reads and writes 28 bytes an element with one fp32 gradient and
// 32-bit moments, 16 with a bf16 gradient, 8-bit moments and a bf16 mirror.  The codes and their random rounding cost some 70
// instructions an element, which makes the instruction issue the second bound there (72 % of its slots used at 4.7e8 elements and 5.8 TB/s);
// the 32-bit step uses 27 %.
//
// Arithmetic contract, as in the momentum kernels: every product, sum, quotient and root is rounded to fp32 by itself, in the
// documented order, whatever the launch shape, so results can be compared bit by bit (one exception: quotients below 2^-126, at kMScale).
#pragma once

#include "packed.cuh"
#include "update_kernels.cuh"

#include <math_constants.h>

namespace softsync {

constexpr int kStateBlock = 256;
constexpr int kChunk = 512;               // elements of a chunk: one block of the AdamW kernel, two warps
constexpr int kListThreads = kChunk / 8;
constexpr int kNormThreads = 256, kNormStep = kNormThreads * 8;          // the norm takes so many elements at a time

struct __align__(16) TensorRec {          // three 16-byte loads
    float *w;
    unsigned short *mirror;
    long long n;                          // elements
    unsigned long long state_off;         // first element in the state arrays
    unsigned first_chunk;
    int on_grid;                          // w and mirror allow the vector form
    float lr_mult, decay_mult;
};

// Gradient pointers of the tensors [t0, t0 + ...) of one launch, tensor-major, in kernel-parameter space: they change with
// every call (a learner pushes another buffer each time), and passing them by value needs no copy to the device.
template <int MAXP>
struct GradTable {
    static constexpr int kPointers = MAXP, kMaxC = MAXP < 256 ? MAXP : 256;
    int t0, c;
    float s[kMaxC];
    const void *g[MAXP];
};
// With what a step multiplies each tensor's weights (x) and update (y) with.
template <int MAXP>
struct StepTable : GradTable<MAXP> {
    float2 coef[MAXP];
};

struct ListTables {
    const TensorRec *recs;
    const int *chunk_tensor;
    unsigned chunk0, nchunks;             // this launch's chunks
};

// Where a lane's element j (0..7) of a warp's 256 lies.  Vector form: two runs of four consecutive elements, so that
// every access of the warp is contiguous with 16 bytes (fp32), 8 (bf16) or 4 (codes) a lane.  Single form, for a tensor's ragged
// end and for pointers off the vector grid: element j * 32 + lane.
template <bool VECTOR>
__device__ __forceinline__ int lane_elem(int lane, int j) { return VECTOR ? (j >> 2) * 128 + lane * 4 + (j & 3) : j * 32 + lane; }

template <typename GT> struct GradBytes;
template <> struct GradBytes<GradFp32> { static constexpr int value = 4; };
template <> struct GradBytes<GradBf16> { static constexpr int value = 2; };

// g[j] of the lane's eight elements of one gradient; p points at the warp's first element.
template <typename GT, bool VECTOR>
__device__ __forceinline__ void load_grad8(float (&g)[8], const unsigned char *p, int lane, int count)
{
    if constexpr (VECTOR) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            Raw<GT, 4> r;
            load_raw(r, p, h * 32 + lane);
            float q[4];
            widen(r, q);
#pragma unroll
            for (int k = 0; k < 4; ++k) g[4 * h + k] = q[k];
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int e = j * 32 + lane;
            float q[1] = {0.f};
            if (e < count) {
                Raw<GT, 1> r;
                load_raw(r, p, e);
                widen(r, q);
            }
            g[j] = q[0];
        }
    }
}

// The weighted sum of the c gradients of tensor `t` for the warp's elements from `first` on.  ONE: c = 1.
template <typename GT, bool VECTOR, bool ONE, int MAXP>
__device__ __forceinline__ void weighted_gradient(float2 (&acc)[4], const GradTable<MAXP> &tab, int t, long long first, int lane, int count)
{
    const void *const *row = tab.g + (ONE ? t - tab.t0 : (t - tab.t0) * tab.c);
    for (int l = 0; l < (ONE ? 1 : tab.c); ++l) {
        float g[8];
        load_grad8<GT, VECTOR>(g, static_cast<const unsigned char *>(row[l]) + first * GradBytes<GT>::value, lane, count);
        const float2 s = make_float2(tab.s[l], tab.s[l]);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float2 x = mul2(s, make_float2(g[2 * k], g[2 * k + 1]));
            acc[k] = ONE || l == 0 ? x : make_float2(__fadd_rn(acc[k].x, x.x), __fadd_rn(acc[k].y, x.y));
        }
    }
}

// Whether every gradient of the tensor lies on the grid of the vector form.
template <typename GT, bool ONE, int MAXP>
__device__ __forceinline__ bool grads_on_grid(const GradTable<MAXP> &tab, int t)
{
    const void *const *row = tab.g + (ONE ? t - tab.t0 : (t - tab.t0) * tab.c);
    bool ok = true;
    for (int l = 0; l < (ONE ? 1 : tab.c); ++l) ok = ok && (reinterpret_cast<uintptr_t>(row[l]) & (4 * GradBytes<GT>::value - 1)) == 0;
    return ok;
}

// ---- global norm ---------------------------------------------------------------------------------------------------

struct NormTail {
    double *partial;                      // one per block of the grid (the same grid for every launch of a call)
    unsigned *done;                       // blocks that have finished; back at zero after the call's last launch
    float *out;
    float max_norm;
    int add;                              // not the call's first launch: add to the partial sums
    int last;                             // the call's last launch: its last block finishes the norm
};

__device__ __forceinline__ double block_sum(double x, double *scratch)
{
    for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = x;
    __syncthreads();
    double y = 0;
    for (int k = 0; k < static_cast<int>(blockDim.x >> 5); ++k) y += scratch[k];
    return y;
}

// Eight consecutive elements of a gradient.
template <typename GT> struct Raw8;
template <> struct Raw8<GradFp32> { float4 a, b; };
template <> struct Raw8<GradBf16> { float4 a; };
__device__ __forceinline__ void load8(Raw8<GradFp32> &r, const unsigned char *p) { r.a = ld_stream_f4(reinterpret_cast<const float4 *>(p)); r.b = ld_stream_f4(reinterpret_cast<const float4 *>(p) + 1); }
__device__ __forceinline__ void load8(Raw8<GradBf16> &r, const unsigned char *p) { r.a = ld_stream_f4(reinterpret_cast<const float4 *>(p)); }
__device__ __forceinline__ float2 pair_of(const Raw8<GradFp32> &r, int k)
{ return k == 0 ? make_float2(r.a.x, r.a.y) : k == 1 ? make_float2(r.a.z, r.a.w) : k == 2 ? make_float2(r.b.x, r.b.y) : make_float2(r.b.z, r.b.w); }
__device__ __forceinline__ float2 pair_of(const Raw8<GradBf16> &r, int k)
{
    const unsigned w = __float_as_uint(k == 0 ? r.a.x : k == 1 ? r.a.y : k == 2 ? r.a.z : r.a.w);
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}

// The sums of squares so far, moved to fp64.
__device__ __forceinline__ void fold_squares(double &total, float2 (&sq)[4])
{
    total += static_cast<double>(((sq[0].x + sq[0].y) + (sq[1].x + sq[1].y)) + ((sq[2].x + sq[2].y) + (sq[3].x + sq[3].y)));
#pragma unroll
    for (int k = 0; k < 4; ++k) sq[k] = make_float2(0.f, 0.f);
}

// Adds the squares of the weighted sum of the c gradients over elements [first, end) of tensor t to total.  Where the gradients lie on the
// 16-byte grid a thread has several loads of eight elements under way at a time, else (and at the end) single elements, those
// of four gradients together.  No more than eight squares are added to one another in fp32, whatever the length.  ONE: c = 1.
template <typename GT, bool ONE, int MAXP>
__device__ __forceinline__ void add_squares(double &total, const GradTable<MAXP> &tab, int t, long long first, long long end)
{
    constexpr int GB = GradBytes<GT>::value, U = ONE && GB == 2 ? 8 : 4;
    const int c = ONE ? 1 : tab.c;
    const void *const *row = tab.g + (t - tab.t0) * c;
    bool on_grid = true;
    for (int l = 0; l < c; ++l) on_grid = on_grid && (reinterpret_cast<uintptr_t>(row[l]) & 15) == 0;            // first is a multiple of kChunk
    long long at = first;
    float2 sq[4] = {};
    if (on_grid) {
        for (int trip = 1; at + U * kNormStep <= end; at += U * kNormStep, ++trip) {
            float2 acc[ONE ? 1 : U][4];
            for (int l = 0; l < c; ++l) {
                const unsigned char *p = static_cast<const unsigned char *>(row[l]) + (at + threadIdx.x * 8) * GB;
                const float2 s = make_float2(tab.s[l], tab.s[l]);
                Raw8<GT> r[U];
#pragma unroll
                for (int u = 0; u < U; ++u) load8(r[u], p + u * kNormStep * GB);
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const float2 x = mul2(s, pair_of(r[u], k));
                        if constexpr (ONE) sq[k] = fma2(x, x, sq[k]);
                        else acc[u][k] = l == 0 ? x : make_float2(__fadd_rn(acc[u][k].x, x.x), __fadd_rn(acc[u][k].y, x.y));
                    }
            }
            if constexpr (!ONE) {
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int k = 0; k < 4; ++k) sq[k] = fma2(acc[u][k], acc[u][k], sq[k]);
            }
            if (trip * U % 8 == 0) fold_squares(total, sq);          // every trip for 61M x 4 in fp32: 189 us, every other one 153
        }
    }
    constexpr int G = ONE ? 1 : 4;
#pragma unroll 1
    for (int trip = 1; at < end; at += kNormStep, ++trip) {
        float g[8] = {};
#pragma unroll 1
        for (int l0 = 0; l0 < c; l0 += G) {
            float x[G][8];
#pragma unroll
            for (int i = 0; i < G; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const long long e = at + j * kNormThreads + threadIdx.x;
                    float y[1] = {0.f};
                    if (l0 + i < c && e < end) {
                        Raw<GT, 1> r;
                        load_raw(r, row[l0 + i], e);
                        widen(r, y);
                    }
                    x[i][j] = y[0];
                }
#pragma unroll
            for (int i = 0; i < G; ++i) {
                if (l0 + i >= c) break;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float y = __fmul_rn(tab.s[l0 + i], x[i][j]);
                    g[j] = l0 + i == 0 ? y : __fadd_rn(g[j], y);
                }
            }
        }
#pragma unroll
        for (int j = 0; j < 8; j += 2) sq[j / 2] = fma2(make_float2(g[j], g[j + 1]), make_float2(g[j], g[j + 1]), sq[j / 2]);
        if (trip % 8 == 0) fold_squares(total, sq);
    }
    fold_squares(total, sq);
}

// Sum of squares of the weighted sum.  The chunks are dealt out in runs of equal length, one a block, so a block looks a tensor up
// once and then streams.  A block's sum goes to its own place, and the block that finishes last adds the places up in their order, so
// no result depends on which block came first.  One read of the gradients is all there is to it: 4.7e8 elements take 140 us in bf16
// (6.71 TB/s) and 268 us in fp32 (6.98), four bf16 gradients 568 us (6.60); a small network's four gradients 8 us, which are the launch, a
// trip to memory and the last block's turn.
template <typename GT, bool ONE, int MAXP>
__global__ void __launch_bounds__(kNormThreads, 3) grad_norm_kernel(const __grid_constant__ ListTables lt,
                                                                    const __grid_constant__ GradTable<MAXP> tab,
                                                                    const __grid_constant__ NormTail tail)
{
    __shared__ double scratch[kNormThreads / 32];
    __shared__ bool finish;
    const long long from = static_cast<long long>(lt.nchunks) * blockIdx.x / gridDim.x, to = static_cast<long long>(lt.nchunks) * (blockIdx.x + 1) / gridDim.x;
    double mine = 0;
    for (long long k = from; k < to;) {
        const int t = lt.chunk_tensor[lt.chunk0 + k];
        const TensorRec &rec = lt.recs[t];
        const long long n = rec.n, chunk = lt.chunk0 + k - rec.first_chunk, chunks = min((n + kChunk - 1) / kChunk - chunk, to - k);
        add_squares<GT, ONE>(mine, tab, t, chunk * kChunk, min(n, (chunk + chunks) * kChunk));
        k += chunks;
    }
    const double sum = block_sum(mine, scratch);
    if (threadIdx.x == 0) {
        tail.partial[blockIdx.x] = tail.add ? tail.partial[blockIdx.x] + sum : sum;
        if (tail.last) {
            __threadfence();
            finish = atomicInc(tail.done, gridDim.x - 1) == gridDim.x - 1;
        }
    }
    if (!tail.last) return;
    __syncthreads();
    if (!finish) return;
    __threadfence();
    double all = 0;
    for (int b = threadIdx.x; b < static_cast<int>(gridDim.x); b += blockDim.x) all += __ldcg(tail.partial + b);
    all = block_sum(all, scratch);
    if (threadIdx.x == 0) {
        const float norm = static_cast<float>(sqrt(all));
        tail.out[0] = norm;
        tail.out[1] = norm > tail.max_norm ? __fdiv_rn(tail.max_norm, norm) : (norm == norm ? 1.f : norm);
    }
}

// ---- 8-bit moments ---------------------------------------------------------------------------------------------------
// A code is the top of an fp32 number: its bits shifted to the place of the low exponent and the high fraction bits, times a
// power of two that moves the exponent back.  Codes without exponent bits become fp32 subnormals on the way, which the
// multiplication scales exactly, so the formats' own subnormals need no case of their own; the way back is the same
// multiplication, and what lies below the kept bits is where the random number is added.
constexpr int kDropBits = 19;                                            // 23 fraction bits of fp32 less the 4 kept
// The units: 2^120 for the first moment (exponent bias 7 = 127 - 120), 2^112 for the second (15 = 127 - 112).

// Code k (0..3) of four in a word, as the fp32 number whose top it is.
template <bool SIGNED>
__device__ __forceinline__ float code_top(unsigned four, int k)
{
    const unsigned top = __byte_perm(four, 0, k << 12 | 0x0444);          // the code in the highest byte
    return __uint_as_float(SIGNED ? static_cast<unsigned>(static_cast<int>(top) >> (24 - kDropBits)) & 0x83f80000u : top >> (24 - kDropBits));
}
template <bool SIGNED>
__device__ __forceinline__ float2 code_pair(unsigned four, int k) { return make_float2(code_top<SIGNED>(four, k), code_top<SIGNED>(four, k + 1)); }
// What a block's codes are multiplied with: unit and scale in one as far as that is a number, the rest in `more` (1 for all but blocks
// whose values pass 2^7 or 2^15; infinity for a marked one).
template <bool SIGNED>
struct BlockScale {
    float scale, more;
    __device__ __forceinline__ explicit BlockScale(unsigned e)
    {
        constexpr unsigned unit = SIGNED ? 120 : 112;
        scale = __uint_as_float(min(e + unit, 254u) << 23);
        more = e == 255u ? CUDART_INF_F : __uint_as_float(max(e + unit, 254u) - 127u << 23);
    }
    // four pairs of codes in two words
    __device__ __forceinline__ void decode(float2 (&x)[4], unsigned a, unsigned b) const
    {
        const float2 s = make_float2(scale, scale);
        x[0] = mul2(code_pair<SIGNED>(a, 0), s);
        x[1] = mul2(code_pair<SIGNED>(a, 2), s);
        x[2] = mul2(code_pair<SIGNED>(b, 0), s);
        x[3] = mul2(code_pair<SIGNED>(b, 2), s);
        if (more != 1.f)
#pragma unroll
            for (int k = 0; k < 4; ++k) x[k] = mul2(x[k], make_float2(more, more));
    }
};

// Exponent byte of a block whose largest magnitude has the bits `top`: the largest code is 31/16 of the power of two, so from
// there on the next one is taken (and no code ever exceeds the largest).  255 marks a block that met an infinity, a NaN or, like them
// beyond the format, 31/16 * 2^126.
__device__ __forceinline__ unsigned block_exponent(unsigned top)
{
    const unsigned e = (top + (1u << kDropBits)) >> 23;
    return e > 253u ? 255u : max(e, 27u);
}

// 32 random bits for the element whose place has the low word lo; hi_term: its high word times 0x9E3779B9.  An integer hash (two rounds
// of xor-shift and multiply) of the place and the step's key; multipliers and shifts are those that C. Wellons published in 2018 from a search for
// 32-bit hashes of low bias (0x7FEB352D, 0x846CA68B; 16, 15, 16).
__device__ __forceinline__ unsigned element_hash(unsigned lo, unsigned hi_term, unsigned key)
{
    unsigned x = (lo ^ key) + hi_term;
    x ^= x >> 16; x *= 0x7FEB352Du;
    x ^= x >> 15; x *= 0x846CA68Bu;
    return x ^ (x >> 16);
}

// Square root and quotient, correctly rounded as the contract wants them, without the branches of the compiler's: from the approximate reciprocal (root) by
// Newton steps in fused multiply-adds whose last correction uses the exact remainder (Markstein, IBM J. Res. Dev. 34, 1990).  Both
// pairs have to be ordinary numbers whose remainders do not underflow.
__device__ __forceinline__ float2 rounded_sqrt(float2 v)
{
    float2 y;
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y.x) : "f"(v.x));
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y.y) : "f"(v.y));
    const float2 half = make_float2(0.5f, 0.5f);
    float2 g = mul2(v, y), h = mul2(y, half);            // root, and half its reciprocal
    const float2 r = fma2(make_float2(-g.x, -g.y), h, half);
    g = fma2(g, r, g);
    h = fma2(h, r, h);
    return fma2(fma2(make_float2(-g.x, -g.y), g, v), h, g);
}
__device__ __forceinline__ float2 rounded_quotient(float2 a, float2 b)
{
    float2 y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y.x) : "f"(b.x));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y.y) : "f"(b.y));
    const float2 minus_b = make_float2(-b.x, -b.y);
    y = fma2(fma2(minus_b, y, make_float2(1.f, 1.f)), y, y);
    float2 q = mul2(a, y);
    q = fma2(fma2(minus_b, q, a), y, q);
    return fma2(fma2(minus_b, q, a), y, q);
}

// ---- AdamW -------------------------------------------------------------------------------------------------------------

struct AdamwParams {
    void *m, *v;                          // state arrays: fp32 or bytes
    unsigned char *m_scale, *v_scale;
    const float *clip;                    // nullptr: none
    float2 beta1, one_minus_beta1, beta2, one_minus_beta2;               // each twice: one 64-bit operand of a packed multiply
    float root_scale, eps;
    unsigned key;
    int short_forms;                      // eps allows the short root and quotient
};

__device__ __forceinline__ float max3_nan(float a, float b, float c)    // NaN if one of them is
{
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

// Scaling that keeps the short root and quotient away from underflow: powers of two that the roundings do not see, but for a quotient
// below 2^-126, which keeps all its bits here and is a subnormal in the other form (a step of the weight below 2^-126 times the step size, so
// only a weight of about zero shows it).  They serve while m < 2^20 and v < 2^30, with an eps of at least 2^-40 (so no quotient overflows, and
// a root of zero may be taken for 2^-78) and a step size of at least 2^-40.
constexpr float kMScale = 0x1p64f, kVScale = 0x1p96f, kVLeast = 0x1p-60f;
constexpr unsigned kMLimit = 0x49800000u, kVLimit = 0x4e800000u;         // bits of 2^20, 2^30

template <typename GT, int BITS, bool VECTOR, bool ONE, int MAXP>
__device__ __forceinline__ void adamw_block(const AdamwParams &p, const StepTable<MAXP> &tab, const TensorRec &rec, int t,
                                            long long first, int lane, int count, float clip)
{
    float2 w[4], m[4], v[4], g[4];
    const float decay = tab.coef[t - tab.t0].x, step = tab.coef[t - tab.t0].y;
    const unsigned long long at = rec.state_off + static_cast<unsigned long long>(first);    // a multiple of kStateBlock
    float *wp = rec.w + first;
    unsigned mcodes[2], vcodes[2];
    unsigned me = 0, ve = 0;
    if constexpr (VECTOR) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const float4 q = __ldcs(reinterpret_cast<const float4 *>(wp) + h * 32 + lane);
            w[2 * h] = make_float2(q.x, q.y); w[2 * h + 1] = make_float2(q.z, q.w);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; j += 2)
            w[j / 2] = make_float2(j * 32 + lane < count ? wp[j * 32 + lane] : 0.f, j * 32 + 32 + lane < count ? wp[j * 32 + 32 + lane] : 0.f);
    }
    if constexpr (BITS == 32) {
        const float *mp = static_cast<const float *>(p.m) + at, *vp = static_cast<const float *>(p.v) + at;
        if constexpr (VECTOR) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float4 a = __ldcs(reinterpret_cast<const float4 *>(mp) + h * 32 + lane);
                const float4 b = __ldcs(reinterpret_cast<const float4 *>(vp) + h * 32 + lane);
                m[2 * h] = make_float2(a.x, a.y); m[2 * h + 1] = make_float2(a.z, a.w);
                v[2 * h] = make_float2(b.x, b.y); v[2 * h + 1] = make_float2(b.z, b.w);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
                const int e = j * 32 + lane;
                m[j / 2] = make_float2(e < count ? mp[e] : 0.f, e + 32 < count ? mp[e + 32] : 0.f);
                v[j / 2] = make_float2(e < count ? vp[e] : 0.f, e + 32 < count ? vp[e + 32] : 0.f);
            }
        }
    } else {
        const unsigned char *mp = static_cast<const unsigned char *>(p.m) + at, *vp = static_cast<const unsigned char *>(p.v) + at;
        me = p.m_scale[at / kStateBlock];
        ve = p.v_scale[at / kStateBlock];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if constexpr (VECTOR) {
                mcodes[h] = __ldcs(reinterpret_cast<const unsigned *>(mp) + h * 32 + lane);
                vcodes[h] = __ldcs(reinterpret_cast<const unsigned *>(vp) + h * 32 + lane);
            } else {
                mcodes[h] = vcodes[h] = 0;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int e = (4 * h + k) * 32 + lane;
                    if (e < count) {
                        mcodes[h] |= static_cast<unsigned>(mp[e]) << (8 * k);
                        vcodes[h] |= static_cast<unsigned>(vp[e]) << (8 * k);
                    }
                }
            }
        }
    }
    weighted_gradient<GT, VECTOR, ONE>(g, tab, t, first, lane, count);
    if constexpr (BITS == 8) {
        BlockScale<true>(me).decode(m, mcodes[0], mcodes[1]);
        BlockScale<false>(ve).decode(v, vcodes[0], vcodes[1]);
        if (count < kStateBlock && (me == 255u || ve == 255u)) {       // a marked block: zero codes are NaN there, but not past the end
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (lane_elem<VECTOR>(lane, j) >= count) {
                    if (j & 1) m[j / 2].y = v[j / 2].y = 0.f;
                    else m[j / 2].x = v[j / 2].x = 0.f;
                }
        }
    }

    const auto two = [](float x) { return make_float2(x, x); };
    float m_top = 0.f, v_top = 0.f;                      // the largest magnitudes; NaN if there is one
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        float2 x = g[k];
        if (p.clip) x = mul2(x, two(clip));
        const float2 a = mul2(m[k], p.beta1), b = mul2(x, p.one_minus_beta1);
        const float2 c = mul2(v[k], p.beta2), d = mul2(mul2(x, x), p.one_minus_beta2);
        m[k] = make_float2(__fadd_rn(a.x, b.x), __fadd_rn(a.y, b.y));
        v[k] = make_float2(__fadd_rn(c.x, d.x), __fadd_rn(c.y, d.y));
        m_top = max3_nan(m_top, fabsf(m[k].x), fabsf(m[k].y));
        v_top = max3_nan(v_top, v[k].x, v[k].y);
    }
    unsigned mt = __float_as_uint(m_top), vt = __float_as_uint(v_top);
    if constexpr (BITS == 8) { mt = __reduce_max_sync(0xffffffffu, mt); vt = __reduce_max_sync(0xffffffffu, vt); }
    if (__all_sync(0xffffffffu, p.short_forms && fabsf(step) >= 0x1p-40f && mt < kMLimit && vt < kVLimit)) {
        const float2 rs = two(p.root_scale * 0x1p-48f), st = two(step * 0x1p-64f);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            float2 x = mul2(v[k], two(kVScale));
            x = make_float2(fmaxf(x.x, kVLeast), fmaxf(x.y, kVLeast));
            x = mul2(rounded_sqrt(x), rs);
            const float2 den = make_float2(__fadd_rn(x.x, p.eps), __fadd_rn(x.y, p.eps));
            const float2 u = mul2(rounded_quotient(mul2(m[k], two(kMScale)), den), st), y = mul2(w[k], two(decay));
            w[k] = make_float2(__fsub_rn(y.x, u.x), __fsub_rn(y.y, u.y));
        }
    } else {
        const auto one = [&](float wi, float mi, float vi) {
            const float den = __fadd_rn(__fmul_rn(__fsqrt_rn(vi), p.root_scale), p.eps);
            return __fsub_rn(__fmul_rn(wi, decay), __fmul_rn(__fdiv_rn(mi, den), step));
        };
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] = make_float2(one(w[k].x, m[k].x, v[k].x), one(w[k].y, m[k].y, v[k].y));
    }

    if constexpr (VECTOR) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
            __stcs(reinterpret_cast<float4 *>(wp) + h * 32 + lane, make_float4(w[2 * h].x, w[2 * h].y, w[2 * h + 1].x, w[2 * h + 1].y));
        if (rec.mirror) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
                __stcs(reinterpret_cast<uint2 *>(rec.mirror + first) + h * 32 + lane,
                       make_uint2(pack_bf16x2(w[2 * h].x, w[2 * h].y), pack_bf16x2(w[2 * h + 1].x, w[2 * h + 1].y)));
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j * 32 + lane < count) {
                const float x = j & 1 ? w[j / 2].y : w[j / 2].x;
                wp[j * 32 + lane] = x;
                if (rec.mirror) rec.mirror[first + j * 32 + lane] = __bfloat16_as_ushort(__float2bfloat16_rn(x));
            }
    }
    if constexpr (BITS == 32) {
        float *mp = static_cast<float *>(p.m) + at, *vp = static_cast<float *>(p.v) + at;
        if constexpr (VECTOR) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                __stcs(reinterpret_cast<float4 *>(mp) + h * 32 + lane, make_float4(m[2 * h].x, m[2 * h].y, m[2 * h + 1].x, m[2 * h + 1].y));
                __stcs(reinterpret_cast<float4 *>(vp) + h * 32 + lane, make_float4(v[2 * h].x, v[2 * h].y, v[2 * h + 1].x, v[2 * h + 1].y));
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (j * 32 + lane < count) {
                    mp[j * 32 + lane] = j & 1 ? m[j / 2].y : m[j / 2].x;
                    vp[j * 32 + lane] = j & 1 ? v[j / 2].y : v[j / 2].x;
                }
        }
    } else {
        // elements past the tensor's end hold zeros (their gradient and codes were never read) and leave the maxima alone
        me = block_exponent(mt);
        ve = block_exponent(vt);
        // to the codes' units: one factor unless the block's values pass 2^6 or 2^14 (the first product is then exact, or below every code)
        if (me > 133u)
#pragma unroll
            for (int k = 0; k < 4; ++k) m[k] = mul2(m[k], two(0x1p-120f));
        if (ve > 141u)
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = mul2(v[k], two(0x1p-112f));
        const float mi = __uint_as_float((me > 133u ? 254u - min(me, 253u) : 134u - me) << 23);
        const float vi = __uint_as_float((ve > 141u ? 254u - min(ve, 253u) : 142u - ve) << 23);
        const unsigned lo = static_cast<unsigned>(at), hi_term = static_cast<unsigned>(at >> 32) * 0x9E3779B9u;
        unsigned mc[2], vc[2];                           // four codes a word
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            unsigned mtop[4], vtop[4];                   // each code in its number's highest byte
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int j = 4 * h + i;
                const float mj = j & 1 ? m[j / 2].y : m[j / 2].x, vj = j & 1 ? v[j / 2].y : v[j / 2].x;
                const unsigned r = element_hash(lo + lane_elem<VECTOR>(lane, j), hi_term, p.key);
                // 16 random bits right below the kept ones, and 3 zeros: the sum's carry does the rounding
                const unsigned low = __byte_perm(r, 0, 0x4104), high = __byte_perm(r, 0, 0x4324);
                mtop[i] = (__float_as_uint(__fmul_rn(fabsf(mj), mi)) << (24 - kDropBits)) + low;
                mtop[i] |= __float_as_uint(mj) & 0x80000000u;
                vtop[i] = (__float_as_uint(__fmul_rn(vj, vi)) << (24 - kDropBits)) + high;
            }
            mc[h] = __byte_perm(__byte_perm(mtop[0], mtop[1], 0x0073), __byte_perm(mtop[2], mtop[3], 0x0073), 0x5410);
            vc[h] = __byte_perm(__byte_perm(vtop[0], vtop[1], 0x0073), __byte_perm(vtop[2], vtop[3], 0x0073), 0x5410);
            if ((vc[h] - 0x01010101u) & ~vc[h] & 0x80808080u) {          // a zero code among them: it stays one only for a v of zero
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int j = 4 * h + i;
                    if (!(vc[h] & 255u << (8 * i)) && (j & 1 ? v[j / 2].y : v[j / 2].x) > 0.f) vc[h] |= 1u << (8 * i);
                }
            }
        }
        unsigned char *mp = static_cast<unsigned char *>(p.m) + at, *vp = static_cast<unsigned char *>(p.v) + at;
        if constexpr (VECTOR) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                __stcs(reinterpret_cast<unsigned *>(mp) + h * 32 + lane, mc[h]);
                __stcs(reinterpret_cast<unsigned *>(vp) + h * 32 + lane, vc[h]);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (j * 32 + lane < count) {
                    mp[j * 32 + lane] = static_cast<unsigned char>(mc[j / 4] >> (8 * (j & 3)));
                    vp[j * 32 + lane] = static_cast<unsigned char>(vc[j / 4] >> (8 * (j & 3)));
                }
        }
        if (lane == 0) {
            p.m_scale[at / kStateBlock] = static_cast<unsigned char>(me);
            p.v_scale[at / kStateBlock] = static_cast<unsigned char>(ve);
        }
    }
}

// Blocks of two warps, so that an SM's registers are refilled in small pieces (61M elements, four fp32 gradients: 363 us, with
// eight warps 370).  For 8-bit moments, the form with the most instructions a byte, 18 of them an SM instead of 16 where the
// registers carry it, with one gradient (4.7e8 elements, fp32 gradient and a mirror: 1366 us, with 16 1402).
//
// A thread has only eight elements, so what it does once counts: with one gradient there is no loop over them, a tensor's two
// factors are computed on the host, in fp64, and a record comes in three loads (4.7e8 elements, bf16 gradient, 8-bit moments, mirror:
// 1295 us, 5.80 TB/s; with the loop, the factors in every thread and 64-bit chunk numbers 1451).  32-bit moments: bf16 gradient and
// mirror 1898 us (6.91 TB/s), fp32 gradient 1885 (6.95).
template <int BITS, bool ONE>
constexpr int adamw_blocks_per_sm() { return BITS == 8 && ONE ? 18 : 16; }

template <typename GT, int BITS, bool ONE, int MAXP>
__global__ void __launch_bounds__(kListThreads, adamw_blocks_per_sm<BITS, ONE>()) adamw_kernel(const __grid_constant__ ListTables lt,
                                                                                             const __grid_constant__ StepTable<MAXP> tab,
                                                                                             const __grid_constant__ AdamwParams p)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const unsigned chunk = lt.chunk0 + blockIdx.x;
    const int t = lt.chunk_tensor[chunk];
    const TensorRec rec = lt.recs[t];
    const long long first = static_cast<long long>(chunk - rec.first_chunk) * kChunk + warp * kStateBlock;
    const long long left = rec.n - first;
    if (left <= 0) return;
    float clip = 1.f;
    if (p.clip) {
        if (!(fabsf(p.clip[0]) <= 3.402823466e38f)) return;          // the norm is not finite: the step changes nothing
        clip = p.clip[1];
    }
    const int count = left < kStateBlock ? static_cast<int>(left) : kStateBlock;
    if (count == kStateBlock && rec.on_grid && grads_on_grid<GT, ONE>(tab, t)) adamw_block<GT, BITS, true, ONE>(p, tab, rec, t, first, lane, count, clip);
    else adamw_block<GT, BITS, false, ONE>(p, tab, rec, t, first, lane, count, clip);
}

// Codes to the values they stand for.  One thread per eight elements of the state arrays, the gaps between the tensors included
// (they hold zeros there, or what the caller put there: the output's gaps are the caller's too).  Two bytes in, four out:
// 4.7e8 elements take 425 us (6.62 TB/s).  The values are exact in bf16: a code has five significant bits.
static __global__ void moments_kernel(const uint2 *m, const uint2 *v, const unsigned char *m_scale, const unsigned char *v_scale,
                                      uint4 *m_out, uint4 *v_out, long long eights)
{
    const long long i = static_cast<long long>(blockIdx.x) * blockDim.x + threadIdx.x;
    if (i >= eights) return;
    const uint2 x = __ldcs(m + i), y = __ldcs(v + i);
    float2 a[4], b[4];
    BlockScale<true>(m_scale[i / (kStateBlock / 8)]).decode(a, x.x, x.y);
    BlockScale<false>(v_scale[i / (kStateBlock / 8)]).decode(b, y.x, y.y);
    const auto pack = [](const float2 &q) { return pack_bf16x2(q.x, q.y); };
    __stcs(m_out + i, make_uint4(pack(a[0]), pack(a[1]), pack(a[2]), pack(a[3])));
    __stcs(v_out + i, make_uint4(pack(b[0]), pack(b[1]), pack(b[2]), pack(b[3])));
}

}  // namespace softsync
