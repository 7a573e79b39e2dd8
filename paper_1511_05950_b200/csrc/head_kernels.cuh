// Losses without logits: what runs around the products of mma_kernels.cuh.
#pragma once

#include "mma_kernels.cuh"

namespace softsync {

// Rows with a factor (weight or gradient) other than zero, in order: order[j] is the j-th of them, place[row] its number or -1, *live how many; their
// sum (fp64: beyond fp32's range too), and the power of two that they are taken relative to, that of the largest finite one (2^-126 to 2^100: its product with 1 / T stays finite for T of 2^-28 and more), so that entries of G are rounded
// alike whatever all factors are multiplied by.  Rows without get zeros in up to two outputs.  One block; each thread takes a run of neighbouring rows a turn.
constexpr int kOrderThreads = 1024, kOrderRun = 8;
struct OrderOut {
    int *order, *place, *live;
    double *sum;
    float *scales;                         // 1 / the power, the power, the power / the sum (0 for a sum of 0)
    float *zero_a, *zero_b;                // may be null
};
__global__ void __launch_bounds__(kOrderThreads) order_kernel(const float *factors, int rows, const __grid_constant__ OrderOut out)
{
    __shared__ int counts[32];
    __shared__ double sums[32];
    __shared__ unsigned tops[32];
    let_next_start();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int base = 0;
    double sum = 0;
    unsigned top = 0;                                      // bits of the largest finite magnitude
    for (long long first = 0; first < rows; first += kOrderThreads * kOrderRun) {
        const long long at = first + threadIdx.x * kOrderRun;
        float f[kOrderRun];
        int mine = 0;
#pragma unroll
        for (int k = 0; k < kOrderRun; ++k) {
            f[k] = at + k < rows ? factors[at + k] : 0.f;
            mine += f[k] != 0.f;                           // NaN takes part
            sum += f[k];
            const unsigned bits = __float_as_uint(f[k]) & 0x7fffffffu;
            if (bits < 0x7f800000u) top = max(top, bits);
        }
        int before = mine;
        for (int o = 1; o < 32; o <<= 1) {
            const int other = __shfl_up_sync(kAllLanes, before, o);
            if (lane >= o) before += other;
        }
        if (lane == 31) counts[warp] = before;
        __syncthreads();
        int upto = counts[lane];                           // every warp adds up the warps' counts for itself
        for (int o = 1; o < 32; o <<= 1) {
            const int other = __shfl_up_sync(kAllLanes, upto, o);
            if (lane >= o) upto += other;
        }
        const int all = __shfl_sync(kAllLanes, upto, 31);
        int offset = base + before - mine + (warp ? __shfl_sync(kAllLanes, upto, warp - 1) : 0);
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
    top = __reduce_max_sync(kAllLanes, top);
    if (lane == 0) { sums[warp] = sum; tops[warp] = top; }
    __syncthreads();
    if (warp) return;
    sum = sums[lane];
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(kAllLanes, sum, o);
    top = __reduce_max_sync(kAllLanes, tops[lane]);
    if (lane) return;
    *out.live = base;
    *out.sum = sum;
    const unsigned exponent = min(max(top >> 23, 1u), 227u);
    const float power = __uint_as_float(exponent << 23);
    out.scales[0] = __uint_as_float((254u - exponent) << 23);
    out.scales[1] = power;
    out.scales[2] = sum == 0 ? 0.f : static_cast<float>(power / sum);
}

// Rows of a matrix one behind the other in 16-byte vectors, padded with zeros: all of them, or the listed ones, and zero rows up to a whole stage of
// a product's contraction.  `zeros`: where a row without a place is set to zero.  A warp takes 256 columns of a row; where rows allow no vectors, its lanes
// read neighbouring values.
constexpr int kGatherThreads = 256, kGatherColumns = 32 * kUnit;
struct GatherIn {
    const __nv_bfloat16 *x;
    int rows, width;
    long long stride;
    const int *order, *place, *live;       // may be null
    int aligned;
    __nv_bfloat16 *out;
    int out_stride;
    __nv_bfloat16 *zeros;                  // may be null; dense rows
};
__global__ void __launch_bounds__(kGatherThreads) gather_kernel(const __grid_constant__ GatherIn in)
{
    __shared__ WarpDesk<__nv_bfloat16> desks[kGatherThreads / 32];
    wait_for_earlier();
    let_next_start();
    const int chunks = (in.out_stride + kGatherColumns - 1) / kGatherColumns, lane = threadIdx.x & 31;
    const long long item = static_cast<long long>(blockIdx.x) * (kGatherThreads / 32) + (threadIdx.x >> 5);
    const int row = static_cast<int>(item / chunks), first = static_cast<int>(item - static_cast<long long>(row) * chunks) * kGatherColumns, col = first + lane * kUnit;
    const int count = in.live ? *in.live : in.rows;
    if (in.zeros && row < in.rows && in.place[row] < 0 && col < in.width)
        store_unit(in.zeros + static_cast<long long>(row) * in.width + col, Unit{}, in.width - col, in.width % kUnit == 0);
    if (row >= (count + kStep - 1) / kStep * kStep) return;          // a whole warp
    const int width = row < count ? in.width : 0;
    const __nv_bfloat16 *from = in.x + (row < count ? (in.order ? in.order[row] : row) * in.stride : 0);
    RawUnit<__nv_bfloat16> raw;
    if (in.aligned) {
        load_unit(raw, from + (col < width ? col : 0), width - col, width - col >= kUnit);
    } else {
        __nv_bfloat16 *v = desks[threadIdx.x >> 5].v;
#pragma unroll
        for (int k = 0; k < kUnit; ++k) v[k * 32 + lane] = first + k * 32 + lane < width ? from[first + k * 32 + lane] : __nv_bfloat16(0.f);
        __syncwarp();
        raw.a = *reinterpret_cast<const uint4 *>(v + lane * kUnit);
    }
    if (col < in.out_stride) *reinterpret_cast<uint4 *>(in.out + static_cast<long long>(row) * in.out_stride + col) = raw.a;
}

// Rows of whole vectors to dense rows of any width, seen as one run of values: a warp takes 256 of them, reads neighbouring values and writes aligned vectors.  (Written
// by the product itself, two bytes a lane, 70723 x 3711 took 0.9 ms, and 0.25 by way of aligned rows.)  magic: 2^64 / cols, rounded up, as in PackShape; 0 for one column.
constexpr int kDenseThreads = 256;
template <typename T>
__global__ void __launch_bounds__(kDenseThreads) dense_rows_kernel(const T *from, long long stride, unsigned count, int cols, unsigned long long magic, T *to)
{
    __shared__ WarpDesk<T> desks[kDenseThreads / 32];
    wait_for_earlier();
    let_next_start();
    const int lane = threadIdx.x & 31;
    const unsigned first = (blockIdx.x * (kDenseThreads / 32) + (threadIdx.x >> 5)) * (32u * kUnit);
    if (first >= count) return;                            // a whole warp
    T *v = desks[threadIdx.x >> 5].v;
    const unsigned width = static_cast<unsigned>(cols), row0 = magic ? static_cast<unsigned>(__umul64hi(first, magic)) : first, col0 = first - row0 * width;
    T got[kUnit];                                          // all eight under way at once
#pragma unroll
    for (int k = 0; k < kUnit; ++k) {
        const unsigned at = first + k * 32 + lane;
        unsigned row = row0, col = col0 + k * 32 + lane;
        if (cols >= 32 * kUnit) {                          // at most one row ends among them
            if (col >= width) { col -= width; ++row; }
        } else {
            row = magic ? static_cast<unsigned>(__umul64hi(at, magic)) : at;
            col = at - row * width;
        }
        got[k] = at < count ? from[row * stride + col] : T(0.f);
    }
#pragma unroll
    for (int k = 0; k < kUnit; ++k) v[k * 32 + lane] = got[k];
    __syncwarp();
    const unsigned mine = first + lane * kUnit;
    if (mine + kUnit <= count) {
#pragma unroll
        for (int k = 0; k < static_cast<int>(sizeof(T)) / 2; ++k) reinterpret_cast<uint4 *>(to + mine)[k] = reinterpret_cast<const uint4 *>(v + lane * kUnit)[k];
    } else {
        for (unsigned k = mine; k < count; ++k) to[k] = v[k - first];
    }
}

// A row's parts joined: normaliser, lse, log probability; and, by the last block, the loss.  Eight rows a block, 64 threads share a row's parts (152000
// entries: 1188 parts).  Bound by latency: two loads' worth of waiting and a short tree (512 rows of 1188 parts: 11.6 us; with 32 rows a block it took 25.8).
constexpr int kJoinRows = 8, kJoinThreads = 512;
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
    float2 *norms;
    double *sums;                          // sum w logp of each block
    unsigned *done;
    const double *total;                   // sum of the weights, or null: rows
    float *stats;                          // loss and sum of the weights, or null
};
__device__ __forceinline__ float2 join_parts(float2 a, float2 b, float scale)
{
    const float m = fmaxf(a.x, b.x);
    if (m == -CUDART_INF_F) return make_float2(m, a.y + b.y);               // both empty, or NaN
    return make_float2(m, a.y * mma_ex2((a.x - m) * scale) + b.y * mma_ex2((b.x - m) * scale));
}
__global__ void __launch_bounds__(kJoinThreads) join_kernel(const __grid_constant__ JoinIn in)
{
    __shared__ float2 found[kJoinThreads / 32][kJoinRows];
    __shared__ bool last;
    wait_for_earlier();
    let_next_start();
    const int tid = threadIdx.x, of = tid % kJoinRows, slice = tid / kJoinRows;
    const int row = static_cast<int>(blockIdx.x) * kJoinRows + of, count = in.live ? *in.live : in.rows;
    float2 s = make_float2(-CUDART_INF_F, 0.f);
    if (row < count)
#pragma unroll 4
        for (int k = slice; k < in.count; k += kJoinThreads / kJoinRows) s = join_parts(s, __ldcg(in.parts + k * in.part_stride + row), in.scale);
#pragma unroll
    for (int o = 16; o >= kJoinRows; o >>= 1) {
        float2 b;
        b.x = __shfl_xor_sync(kAllLanes, s.x, o);
        b.y = __shfl_xor_sync(kAllLanes, s.y, o);
        s = (tid & 31) & o ? join_parts(b, s, in.scale) : join_parts(s, b, in.scale);
    }
    if ((tid & 31) < kJoinRows) found[tid >> 5][of] = s;
    __syncthreads();
    if (tid >= 32) {
        if (!in.stats) return;
    } else {
        double share = 0;
        s = found[tid / kJoinRows][of];
#pragma unroll
        for (int w = 32 / kJoinRows; w < kJoinThreads / 32; w += 32 / kJoinRows) s = join_parts(s, found[w + tid / kJoinRows][of], in.scale);
#pragma unroll
        for (int o = 16; o >= kJoinRows; o >>= 1) {
            const float2 b = make_float2(__shfl_xor_sync(kAllLanes, s.x, o), __shfl_xor_sync(kAllLanes, s.y, o));
            s = tid & o ? join_parts(b, s, in.scale) : join_parts(s, b, in.scale);
        }
        if (tid < kJoinRows && row < count) {
            const int at = in.order ? in.order[row] : row;
            const long long t = in.tokens[at];
            const bool known = t >= 0 && t < in.vocab;
            if (!known || s.y == 0.f) s.y = CUDART_NAN_F;
            // products' difference first: the rounding is that of a small number where the token is likely
            const float rest = logf(s.y), logp = known ? fmaf(in.picked[row] - s.x, in.inv_temperature, -rest) : CUDART_NAN_F;
            in.norms[row] = make_float2(s.x, log2f(s.y));
            in.lse[at] = fmaf(s.x, in.inv_temperature, rest);
            in.logp[at] = logp;
            share = in.weights ? static_cast<double>(in.weights[at]) * logp : logp;
        }
        if (!in.stats) return;
        for (int o = kJoinRows / 2; o; o >>= 1) share += __shfl_xor_sync(kAllLanes, share, o);
        if (tid == 0) {
            in.sums[blockIdx.x] = share;
            __threadfence();
            last = atomicAdd(in.done, 1u) == gridDim.x - 1;
        }
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    __shared__ double part[kJoinThreads / 32];
    double sum = 0;
    for (int k = tid; k < static_cast<int>(gridDim.x); k += kJoinThreads) sum += __ldcg(in.sums + k);
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(kAllLanes, sum, o);
    if ((tid & 31) == 0) part[tid >> 5] = sum;
    __syncthreads();
    if (tid) return;
    for (int w = 1; w < kJoinThreads / 32; ++w) sum += part[w];
    const double all = in.total ? *in.total : static_cast<double>(in.rows);
    in.stats[0] = all == 0 ? 0.f : static_cast<float>(-sum / all);
    in.stats[1] = static_cast<float>(all);
}

// G of the kept piece, from its exponentials and in their place: p = e 2^(scale (part's maximum - row's) - log2 sum).  A token that is its part's
// maximum has e = 1 exactly, any other has p <= 1/2: so p - 1 does not suffer from e's rounding.  Bound by HBM: one read, one write, 6.4 TB/s (7168 x 65536: 292 us).
constexpr int kKeptThreads = 256, kKeptTurns = 4, kKeptColumns = kKeptThreads * kKeptTurns * kUnit;
struct KeptIn {
    uint4 *g;                              // eight values each
    long long stride;                      // vectors of a row
    int first, width, segments;            // blocks a row
    const float2 *parts, *norms;
    long long part_stride;
    const long long *tokens;
    const int *order, *live;
    const float *coef, *coef_scale;        // factors of all rows, and what they are multiplied by; null: 1
    float sign, scale;
    int rows;
};
__global__ void __launch_bounds__(kKeptThreads) kept_grad_kernel(const __grid_constant__ KeptIn in)
{
    wait_for_earlier();
    let_next_start();
    const int row = static_cast<int>(blockIdx.x / static_cast<unsigned>(in.segments)), segment = static_cast<int>(blockIdx.x % static_cast<unsigned>(in.segments));
    const int count = in.live ? *in.live : in.rows;
    if (row >= (count + kStep - 1) / kStep * kStep) return;
    uint4 *g = in.g + row * in.stride;
    const int col0 = segment * kKeptColumns + static_cast<int>(threadIdx.x) * kUnit;
    uint4 e[kKeptTurns];
    float top[kKeptTurns];
    if (row < count) {
#pragma unroll
        for (int j = 0; j < kKeptTurns; ++j) {
            const int col = col0 + j * kKeptThreads * kUnit;
            if (col < in.width) {
                e[j] = g[col / kUnit];
                top[j] = __ldcg(&in.parts[static_cast<long long>((in.first + col) / kHalf) * in.part_stride + row].x);
            }
        }
    }
    const int at = row < count ? in.order ? in.order[row] : row : 0;
    const long long token = row < count ? in.tokens[at] - in.first : -1;
    const float a = row < count ? in.coef ? in.sign * in.coef[at] * *in.coef_scale : 1.f : 0.f;
    const float2 norm = row < count ? in.norms[row] : make_float2(0.f, 0.f);
#pragma unroll
    for (int j = 0; j < kKeptTurns; ++j) {
        const int col = col0 + j * kKeptThreads * kUnit;
        if (col >= in.width) break;
        uint4 out = make_uint4(0, 0, 0, 0);
        if (row < count) {
            const float f = a * (mma_ex2(fmaf(top[j] - norm.x, in.scale, -norm.y)) * 18446744073709551616.f);
            const unsigned w[4] = {e[j].x, e[j].y, e[j].z, e[j].w};
            Unit u;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float2 v = shares_below(w[k]);
                u.v[2 * k] = v.x * f;
                u.v[2 * k + 1] = v.y * f;
            }
            if (token >= col && token < col + kUnit) {
                const int own = static_cast<int>(token) - col;
#pragma unroll
                for (int k = 0; k < kUnit; ++k) if (k == own) u.v[k] -= a;
            }
            out = make_uint4(bf16_pair(u.v[0], u.v[1]), bf16_pair(u.v[2], u.v[3]), bf16_pair(u.v[4], u.v[5]), bf16_pair(u.v[6], u.v[7]));
        }
        g[col / kUnit] = out;
    }
}

}  // namespace softsync
