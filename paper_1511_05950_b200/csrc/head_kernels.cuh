// Losses without logits: what runs around the products of mma_kernels.cuh.
#pragma once

#include "mma_kernels.cuh"

namespace softsync {

// Rows with a factor (weight or gradient) other than zero, in order: order[j] is the j-th of them, place[row] its number or -1, *live how many; and
// their sum.  Rows without get zeros in up to two outputs.  One block; each thread takes a run of neighbouring rows a turn.
constexpr int kOrderThreads = 1024, kOrderRun = 8;
struct OrderOut {
    int *order, *place, *live;
    float *inverse, *sum;                  // 1 / sum of the factors (0 for 0), the sum; may be null
    float *zero_a, *zero_b;                // may be null
};
__global__ void __launch_bounds__(kOrderThreads) order_kernel(const float *factors, int rows, const __grid_constant__ OrderOut out)
{
    __shared__ int counts[32];
    __shared__ double sums[32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int base = 0;
    double sum = 0;
    for (long long first = 0; first < rows; first += kOrderThreads * kOrderRun) {
        const long long at = first + threadIdx.x * kOrderRun;
        float f[kOrderRun];
        int mine = 0;
#pragma unroll
        for (int k = 0; k < kOrderRun; ++k) {
            f[k] = at + k < rows ? factors[at + k] : 0.f;
            mine += f[k] != 0.f;                           // NaN takes part
            sum += f[k];
        }
        int before = mine;
        for (int o = 1; o < 32; o <<= 1) {
            const int other = __shfl_up_sync(kAllLanes, before, o);
            if (lane >= o) before += other;
        }
        if (lane == 31) counts[warp] = before;
        __syncthreads();
        int offset = base, all = 0;
        for (int w = 0; w < 32; ++w) {
            if (w < warp) offset += counts[w];
            all += counts[w];
        }
        offset += before - mine;
#pragma unroll
        for (int k = 0; k < kOrderRun; ++k) {
            if (at + k >= rows) break;
            if (f[k] != 0.f) {
                out.order[offset] = static_cast<int>(at + k);
                out.place[at + k] = offset++;
            } else {
                out.place[at + k] = -1;
                if (out.zero_a) out.zero_a[at + k] = 0.f;
                if (out.zero_b) out.zero_b[at + k] = 0.f;
            }
        }
        base += all;
        __syncthreads();                                   // counts are written again
    }
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(kAllLanes, sum, o);
    if (lane == 0) sums[warp] = sum;
    __syncthreads();
    if (threadIdx.x) return;
    *out.live = base;
    for (int w = 1; w < 32; ++w) sum += sums[w];
    if (out.sum) *out.sum = static_cast<float>(sum);
    if (out.inverse) *out.inverse = sum == 0 ? 0.f : static_cast<float>(1.0 / sum);
}

// Rows of a matrix one behind the other in 16-byte vectors, padded with zeros: all of them, or the listed ones, and zero rows up to a whole stage of
// a product's contraction.  A block a row.
__global__ void __launch_bounds__(128) gather_kernel(const __nv_bfloat16 *x, int rows, int width, long long stride, const int *order, const int *live, int aligned,
                                                     __nv_bfloat16 *out, int out_stride)
{
    const int row = blockIdx.x, count = live ? *live : rows;
    if (row >= (count + kStep - 1) / kStep * kStep) return;
    const __nv_bfloat16 *from = x + (row < count ? (order ? order[row] : row) * stride : 0);
    for (int col = threadIdx.x * kUnit; col < out_stride; col += 128 * kUnit) {
        const int left = row < count ? width - col : 0;
        RawUnit<__nv_bfloat16> raw;
        load_unit(raw, from + (left > 0 ? col : 0), left, aligned && left >= kUnit);
        *reinterpret_cast<uint4 *>(out + static_cast<long long>(row) * out_stride + col) = raw.a;
    }
}

// A row's parts joined: lse and log probability; and the block's share of sum w logp.  32 rows a block, the warps share the parts.
constexpr int kJoinWarps = 16;
struct JoinIn {
    const float2 *parts;
    long long part_stride;
    int count;                             // parts of a row
    const float *picked;
    const long long *tokens;
    const int *order, *live;               // may be null
    const float *weights;                  // may be null
    int rows, vocab;
    float scale, inv_temperature;          // log2(e) / T, 1 / T
    float *logp, *lse;
    double *sums;                          // one for each block, or null
};
__global__ void __launch_bounds__(32 * kJoinWarps) join_kernel(const __grid_constant__ JoinIn in)
{
    __shared__ float2 found[kJoinWarps][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int row = static_cast<int>(blockIdx.x) * 32 + lane, count = in.live ? *in.live : in.rows;
    const auto join = [&](float2 a, float2 b) {
        const float m = fmaxf(a.x, b.x);
        if (m == -CUDART_INF_F) return make_float2(m, a.y + b.y);           // both empty, or NaN
        return make_float2(m, a.y * mma_ex2((a.x - m) * in.scale) + b.y * mma_ex2((b.x - m) * in.scale));
    };
    float2 s = make_float2(-CUDART_INF_F, 0.f);
    if (row < count)
#pragma unroll 4
        for (int k = warp; k < in.count; k += kJoinWarps) s = join(s, in.parts[k * in.part_stride + row]);
    found[warp][lane] = s;
    __syncthreads();
    if (warp) return;
    double share = 0;
    if (row < count) {
        for (int w = 1; w < kJoinWarps; ++w) s = join(s, found[w][lane]);
        const int at = in.order ? in.order[row] : row;
        const long long t = in.tokens[at];
        const bool known = t >= 0 && t < in.vocab;
        // products' difference first: the rounding is that of a small number where the token is likely
        const float rest = s.y == 0.f ? CUDART_NAN_F : logf(s.y), lse = known ? fmaf(s.x, in.inv_temperature, rest) : CUDART_NAN_F;
        const float logp = known ? fmaf(in.picked[row] - s.x, in.inv_temperature, -rest) : CUDART_NAN_F;
        in.lse[at] = lse;
        in.logp[at] = logp;
        share = in.weights ? static_cast<double>(in.weights[at]) * logp : logp;
    }
    if (!in.sums) return;
    for (int o = 16; o; o >>= 1) share += __shfl_xor_sync(kAllLanes, share, o);
    if (lane == 0) in.sums[blockIdx.x] = share;
}

// loss and sum of the weights.
__global__ void __launch_bounds__(256) loss_kernel(const double *sums, int blocks, const float *total, int rows, float *stats)
{
    __shared__ double part[8];
    double s = 0;
    for (int k = threadIdx.x; k < blocks; k += 256) s += sums[k];
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(kAllLanes, s, o);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = s;
    __syncthreads();
    if (threadIdx.x) return;
    for (int w = 1; w < 8; ++w) s += part[w];
    const float all = total ? *total : static_cast<float>(rows);
    stats[0] = all == 0.f ? 0.f : static_cast<float>(-s / all);
    stats[1] = all;
}

// Sums of a product's splits added up, in order, times alpha (and a gain for each column); rows by their place, zeros where they have none.
struct SplitSum {
    const float *part;
    long long part_stride, part_rows;
    int splits;
    const int *place;                      // may be null: row r at r
    int rows, cols;
    float alpha;
    const float *alpha_dev;
    const void *gain;
    int gain_bf16;
    void *out;
    int out_bf16, vectors;
    long long stride;
};
__global__ void __launch_bounds__(128) split_sum_kernel(const __grid_constant__ SplitSum in)
{
    const int row = blockIdx.x;
    const int from = in.place ? in.place[row] : row;
    const float factor = in.alpha_dev ? in.alpha * *in.alpha_dev : in.alpha;
    for (int col = threadIdx.x * kUnit; col < in.cols; col += 128 * kUnit) {
        Unit u{};
        const int left = in.cols - col;
        const bool whole = in.vectors && left >= kUnit;
        if (from >= 0) {
            const float *p = in.part + from * in.part_stride + col;
            for (int s = 0; s < in.splits; ++s, p += in.part_rows) {
                const float4 a = __ldcs(reinterpret_cast<const float4 *>(p)), b = __ldcs(reinterpret_cast<const float4 *>(p) + 1);
                const float v[kUnit] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
                for (int k = 0; k < kUnit; ++k) u.v[k] += v[k];
            }
#pragma unroll
            for (int k = 0; k < kUnit; ++k) u.v[k] *= factor;
            if (in.gain) {
                const Unit w = load_gain(in.gain, in.gain_bf16, col, left, whole);
#pragma unroll
                for (int k = 0; k < kUnit; ++k) u.v[k] *= w.v[k];
            }
        }
        if (in.out_bf16) store_unit(static_cast<__nv_bfloat16 *>(in.out) + row * in.stride + col, u, left, whole);
        else store_unit(static_cast<float *>(in.out) + row * in.stride + col, u, left, whole);
    }
}

}  // namespace softsync
