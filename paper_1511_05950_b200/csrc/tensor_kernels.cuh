// Kernels over a list of tensors: global norm of a weighted sum of gradients, AdamW with moments in 32 or 8 bits.
//
// The list's elements are cut into chunks of kChunk elements, none of which spans two tensors; a table says which tensor a chunk
// belongs to.  Within a chunk every warp owns kStateBlock = 256 consecutive elements, eight a lane: exactly one block of
// 8-bit moments, so a block's largest value is one warp reduction and needs neither shared memory nor a second pass.
//
// Both passes touch every byte once and are bound by HBM: AdamW reads and writes 28 bytes an element with one fp32 gradient and
// 32-bit moments, 14 with a bf16 gradient and 8-bit moments, for about 20 (60 with the codes) arithmetic instructions.
//
// Arithmetic contract, as in the momentum kernels: every product, sum, quotient and root is rounded to fp32 by itself, in the
// documented order, whatever the launch shape, so results can be compared bit by bit.
#pragma once

#include "update_kernels.cuh"

namespace softsync {

constexpr int kStateBlock = 256;
constexpr int kChunk = 2048;              // elements of a chunk: one block of 8 warps
constexpr int kListThreads = kChunk / 8;

struct TensorRec {
    float *w;
    unsigned short *mirror;
    long long n;                          // elements
    long long state_off;                  // first element in the state arrays
    long long first_chunk;
    float lr_mult, decay_mult;
};

// Gradient pointers of the tensors [t0, t0 + ...) of one launch, tensor-major, in kernel-parameter space: they change with
// every call (a learner pushes another buffer each time), and passing them by value needs no copy to the device.
template <int MAXP>
struct GradTable {
    static constexpr int kMaxC = MAXP < 256 ? MAXP : 256;
    int t0, c;
    float s[kMaxC];
    const void *g[MAXP];
};

struct ListTables {
    const TensorRec *recs;
    const int *chunk_tensor;
    long long chunk0, nchunks;            // this launch's chunks
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

// The weighted sum of the c gradients of tensor `t` for the warp's elements from `first` on.
template <typename GT, bool VECTOR, int MAXP>
__device__ __forceinline__ void weighted_gradient(float (&acc)[8], const GradTable<MAXP> &tab, int t, long long first, int lane, int count)
{
    const void *const *row = tab.g + (t - tab.t0) * tab.c;
    for (int l = 0; l < tab.c; ++l) {
        float g[8];
        load_grad8<GT, VECTOR>(g, static_cast<const unsigned char *>(row[l]) + first * GradBytes<GT>::value, lane, count);
        const float s = tab.s[l];
        if (l == 0) {
#pragma unroll
            for (int j = 0; j < 8; ++j) acc[j] = __fmul_rn(s, g[j]);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) acc[j] = __fadd_rn(acc[j], __fmul_rn(s, g[j]));
        }
    }
}

// Whether every gradient of the tensor lies on the grid of the vector form.
template <typename GT, int MAXP>
__device__ __forceinline__ bool grads_on_grid(const GradTable<MAXP> &tab, int t)
{
    const void *const *row = tab.g + (t - tab.t0) * tab.c;
    bool ok = true;
    for (int l = 0; l < tab.c; ++l) ok = ok && (reinterpret_cast<uintptr_t>(row[l]) & (4 * GradBytes<GT>::value - 1)) == 0;
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

// Sum of squares of the weighted sum.  Each block walks every gridDim.x-th chunk; a block's sum goes to its own place, and the
// block that finishes last adds the places up in their order, so no result depends on which block came first.
template <typename GT, int MAXP>
__global__ void __launch_bounds__(kListThreads) grad_norm_kernel(const __grid_constant__ ListTables lt,
                                                                 const __grid_constant__ GradTable<MAXP> tab,
                                                                 const __grid_constant__ NormTail tail)
{
    __shared__ double scratch[kListThreads / 32];
    __shared__ bool finish;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    float sq[8] = {};
    for (long long k = blockIdx.x; k < lt.nchunks; k += gridDim.x) {
        const int t = lt.chunk_tensor[lt.chunk0 + k];
        const TensorRec &rec = lt.recs[t];
        const long long first = (lt.chunk0 + k - rec.first_chunk) * kChunk + warp * kStateBlock;
        const long long left = rec.n - first;
        if (left <= 0) continue;
        const int count = left < kStateBlock ? static_cast<int>(left) : kStateBlock;
        float g[8];
        if (count == kStateBlock && grads_on_grid<GT>(tab, t)) weighted_gradient<GT, true>(g, tab, t, first, lane, count);
        else weighted_gradient<GT, false>(g, tab, t, first, lane, count);
#pragma unroll
        for (int j = 0; j < 8; ++j) sq[j] = fmaf(g[j], g[j], sq[j]);
    }
    double mine = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) mine += sq[j];
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
constexpr unsigned kMaxCodeM = 127, kMaxCodeV = 255;
#define SOFTSYNC_M_UNIT 0x1p120f                                         // first moment: exponent bias 7 = 127 - 120
#define SOFTSYNC_V_UNIT 0x1p112f                                         // second moment: bias 15 = 127 - 112

__device__ __forceinline__ float decode_m(unsigned code, float scale)
{
    const float x = __fmul_rn(__fmul_rn(__uint_as_float((code & 127u) << kDropBits), SOFTSYNC_M_UNIT), scale);
    return code & 128u ? -x : x;
}
__device__ __forceinline__ float decode_v(unsigned code, float scale)
{
    return __fmul_rn(__fmul_rn(__uint_as_float(code << kDropBits), SOFTSYNC_V_UNIT), scale);
}
__device__ __forceinline__ float block_scale(unsigned e) { return __uint_as_float(e << 23); }

// Exponent byte of a block whose largest magnitude has the bits `top`: the largest code is 31/16 of the power of two, so from
// there on the next one is taken; 255 marks a block that met an infinity or a NaN.
__device__ __forceinline__ unsigned block_exponent(unsigned top)
{
    if (top >= 0x7f800000u) return 255u;
    return min(max((top + (1u << kDropBits)) >> 23, 27u), 253u);
}
__device__ __forceinline__ unsigned encode(float mag, float inv_scale, float unit, unsigned rnd, unsigned top)
{
    const unsigned bits = __float_as_uint(__fmul_rn(__fmul_rn(mag, inv_scale), unit));
    return min((bits + rnd) >> kDropBits, top);
}

// 32 random bits for element i: an integer hash (two rounds of xor-shift and multiply) of its place and the step's key.
__device__ __forceinline__ unsigned element_hash(unsigned long long i, unsigned key)
{
    unsigned x = (static_cast<unsigned>(i) ^ key) + static_cast<unsigned>(i >> 32) * 0x9E3779B9u;
    x ^= x >> 16; x *= 0x7FEB352Du;
    x ^= x >> 15; x *= 0x846CA68Bu;
    return x ^ (x >> 16);
}

// ---- AdamW -------------------------------------------------------------------------------------------------------------

struct AdamwParams {
    void *m, *v;                          // state arrays: fp32 or bytes
    unsigned char *m_scale, *v_scale;
    const float *clip;                    // nullptr: none
    double lr_decay, step_size;           // lr * weight_decay; lr / (1 - beta1^t)
    float beta1, one_minus_beta1, beta2, one_minus_beta2, root_scale, eps;
    unsigned key;
};

template <typename GT, int BITS, bool VECTOR, int MAXP>
__device__ __forceinline__ void adamw_block(const AdamwParams &p, const GradTable<MAXP> &tab, const TensorRec &rec, int t,
                                            long long first, int lane, int count, float clip)
{
    float g[8], w[8], m[8], v[8];
    const long long at = rec.state_off + first;          // a multiple of kStateBlock
    float *wp = rec.w + first;
    if constexpr (VECTOR) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const float4 q = __ldcs(reinterpret_cast<const float4 *>(wp) + h * 32 + lane);
            w[4 * h] = q.x; w[4 * h + 1] = q.y; w[4 * h + 2] = q.z; w[4 * h + 3] = q.w;
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = j * 32 + lane < count ? wp[j * 32 + lane] : 0.f;
    }
    if constexpr (BITS == 32) {
        const float *mp = static_cast<const float *>(p.m) + at, *vp = static_cast<const float *>(p.v) + at;
        if constexpr (VECTOR) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float4 a = __ldcs(reinterpret_cast<const float4 *>(mp) + h * 32 + lane);
                const float4 b = __ldcs(reinterpret_cast<const float4 *>(vp) + h * 32 + lane);
                m[4 * h] = a.x; m[4 * h + 1] = a.y; m[4 * h + 2] = a.z; m[4 * h + 3] = a.w;
                v[4 * h] = b.x; v[4 * h + 1] = b.y; v[4 * h + 2] = b.z; v[4 * h + 3] = b.w;
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                m[j] = j * 32 + lane < count ? mp[j * 32 + lane] : 0.f;
                v[j] = j * 32 + lane < count ? vp[j * 32 + lane] : 0.f;
            }
        }
    } else {
        const unsigned char *mp = static_cast<const unsigned char *>(p.m) + at, *vp = static_cast<const unsigned char *>(p.v) + at;
        const float ms = block_scale(p.m_scale[at / kStateBlock]), vs = block_scale(p.v_scale[at / kStateBlock]);
        if constexpr (VECTOR) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const unsigned a = __ldcs(reinterpret_cast<const unsigned *>(mp) + h * 32 + lane);
                const unsigned b = __ldcs(reinterpret_cast<const unsigned *>(vp) + h * 32 + lane);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    m[4 * h + k] = decode_m((a >> (8 * k)) & 255u, ms);
                    v[4 * h + k] = decode_v((b >> (8 * k)) & 255u, vs);
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const bool in = j * 32 + lane < count;
                m[j] = in ? decode_m(mp[j * 32 + lane], ms) : 0.f;
                v[j] = in ? decode_v(vp[j * 32 + lane], vs) : 0.f;
            }
        }
    }
    weighted_gradient<GT, VECTOR>(g, tab, t, first, lane, count);

    const float decay = static_cast<float>(1.0 - p.lr_decay * (static_cast<double>(rec.lr_mult) * rec.decay_mult));
    const float step = static_cast<float>(p.step_size * rec.lr_mult);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float x = p.clip ? __fmul_rn(g[j], clip) : g[j];
        m[j] = __fadd_rn(__fmul_rn(m[j], p.beta1), __fmul_rn(x, p.one_minus_beta1));
        v[j] = __fadd_rn(__fmul_rn(v[j], p.beta2), __fmul_rn(__fmul_rn(x, x), p.one_minus_beta2));
        const float den = __fadd_rn(__fmul_rn(__fsqrt_rn(v[j]), p.root_scale), p.eps);
        w[j] = __fsub_rn(__fmul_rn(w[j], decay), __fmul_rn(__fdiv_rn(m[j], den), step));
    }

    if constexpr (VECTOR) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
            __stcs(reinterpret_cast<float4 *>(wp) + h * 32 + lane, make_float4(w[4 * h], w[4 * h + 1], w[4 * h + 2], w[4 * h + 3]));
        if (rec.mirror) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
                __stcs(reinterpret_cast<uint2 *>(rec.mirror + first) + h * 32 + lane,
                       make_uint2(pack_bf16x2(w[4 * h], w[4 * h + 1]), pack_bf16x2(w[4 * h + 2], w[4 * h + 3])));
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j * 32 + lane < count) {
                wp[j * 32 + lane] = w[j];
                if (rec.mirror) rec.mirror[first + j * 32 + lane] = __bfloat16_as_ushort(__float2bfloat16_rn(w[j]));
            }
    }
    if constexpr (BITS == 32) {
        float *mp = static_cast<float *>(p.m) + at, *vp = static_cast<float *>(p.v) + at;
        if constexpr (VECTOR) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                __stcs(reinterpret_cast<float4 *>(mp) + h * 32 + lane, make_float4(m[4 * h], m[4 * h + 1], m[4 * h + 2], m[4 * h + 3]));
                __stcs(reinterpret_cast<float4 *>(vp) + h * 32 + lane, make_float4(v[4 * h], v[4 * h + 1], v[4 * h + 2], v[4 * h + 3]));
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (j * 32 + lane < count) { mp[j * 32 + lane] = m[j]; vp[j * 32 + lane] = v[j]; }
        }
    } else {
        // elements past the tensor's end hold zeros (their gradient and moments were never read) and leave the maxima alone
        unsigned mt = 0, vt = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            mt = max(mt, __float_as_uint(m[j]) & 0x7fffffffu);
            vt = max(vt, __float_as_uint(v[j]) & 0x7fffffffu);
        }
        const unsigned me = block_exponent(__reduce_max_sync(0xffffffffu, mt));
        const unsigned ve = block_exponent(__reduce_max_sync(0xffffffffu, vt));
        const float mi = __uint_as_float((254u - min(me, 253u)) << 23), vi = __uint_as_float((254u - min(ve, 253u)) << 23);
        unsigned mc[8], vc[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const unsigned r = element_hash(static_cast<unsigned long long>(at) + lane_elem<VECTOR>(lane, j), p.key);
            mc[j] = encode(fabsf(m[j]), mi, 1.f / SOFTSYNC_M_UNIT, (r & 0xffffu) << 3, kMaxCodeM) | (m[j] < 0.f ? 128u : 0u);
            vc[j] = encode(v[j], vi, 1.f / SOFTSYNC_V_UNIT, (r >> 16) << 3, kMaxCodeV);
            if (v[j] > 0.f) vc[j] = max(vc[j], 1u);
        }
        unsigned char *mp = static_cast<unsigned char *>(p.m) + at, *vp = static_cast<unsigned char *>(p.v) + at;
        if constexpr (VECTOR) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                __stcs(reinterpret_cast<unsigned *>(mp) + h * 32 + lane, mc[4 * h] | mc[4 * h + 1] << 8 | mc[4 * h + 2] << 16 | mc[4 * h + 3] << 24);
                __stcs(reinterpret_cast<unsigned *>(vp) + h * 32 + lane, vc[4 * h] | vc[4 * h + 1] << 8 | vc[4 * h + 2] << 16 | vc[4 * h + 3] << 24);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (j * 32 + lane < count) {
                    mp[j * 32 + lane] = static_cast<unsigned char>(mc[j]);
                    vp[j * 32 + lane] = static_cast<unsigned char>(vc[j]);
                }
        }
        if (lane == 0) {
            p.m_scale[at / kStateBlock] = static_cast<unsigned char>(me);
            p.v_scale[at / kStateBlock] = static_cast<unsigned char>(ve);
        }
    }
}

template <typename GT, int BITS, int MAXP>
__global__ void __launch_bounds__(kListThreads) adamw_kernel(const __grid_constant__ ListTables lt,
                                                             const __grid_constant__ GradTable<MAXP> tab,
                                                             const __grid_constant__ AdamwParams p)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const long long chunk = lt.chunk0 + blockIdx.x;
    const int t = lt.chunk_tensor[chunk];
    const TensorRec rec = lt.recs[t];
    const long long first = (chunk - rec.first_chunk) * kChunk + warp * kStateBlock;
    const long long left = rec.n - first;
    if (left <= 0) return;
    float clip = 1.f;
    if (p.clip) {
        if (!(fabsf(p.clip[0]) <= 3.402823466e38f)) return;          // the norm is not finite: the step changes nothing
        clip = p.clip[1];
    }
    const int count = left < kStateBlock ? static_cast<int>(left) : kStateBlock;
    const bool grid = (reinterpret_cast<uintptr_t>(rec.w) & 15) == 0 && (reinterpret_cast<uintptr_t>(rec.mirror) & 7) == 0;
    if (count == kStateBlock && grid && grads_on_grid<GT>(tab, t)) adamw_block<GT, BITS, true>(p, tab, rec, t, first, lane, count, clip);
    else adamw_block<GT, BITS, false>(p, tab, rec, t, first, lane, count, clip);
}

// Codes to the values they stand for.  One thread per four elements of the state arrays, the gaps between the tensors included
// (they hold zeros there, or what the caller put there: the output's gaps are the caller's too).
static __global__ void moments_kernel(const unsigned *m, const unsigned *v, const unsigned char *ms, const unsigned char *vs,
                               uint2 *m_out, uint2 *v_out, long long quads)
{
    const long long i = static_cast<long long>(blockIdx.x) * blockDim.x + threadIdx.x;
    if (i >= quads) return;
    const float a = block_scale(ms[i / (kStateBlock / 4)]), b = block_scale(vs[i / (kStateBlock / 4)]);
    const unsigned x = m[i], y = v[i];
    float p[4], q[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) { p[k] = decode_m((x >> (8 * k)) & 255u, a); q[k] = decode_v((y >> (8 * k)) & 255u, b); }
    __stcs(m_out + i, make_uint2(pack_bf16x2(p[0], p[1]), pack_bf16x2(p[2], p[3])));
    __stcs(v_out + i, make_uint2(pack_bf16x2(q[0], q[1]), pack_bf16x2(q[2], q[3])));
}

}  // namespace softsync
