// Root-mean-square norm with the residual's addition, its backward pass, and activations in 8 bits.
#pragma once

#include "units.cuh"

namespace softsync {

__device__ __forceinline__ float norm_warp_sum(float x)
{
    for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(kAllLanes, x, o);
    return x;
}

// Sum over the threads of a row: a warp, or the WARPS warps of the block.  slot: one of two places that successive calls take in turn, so
// that one barrier a call is enough.
template <int WARPS>
__device__ __forceinline__ float row_sum(float x, float (*part)[32], int slot)
{
    x = norm_warp_sum(x);
    if constexpr (WARPS > 1) {
        if ((threadIdx.x & 31) == 0) part[slot][threadIdx.x >> 5] = x;
        __syncthreads();
        x = (threadIdx.x & 31) < WARPS ? part[slot][threadIdx.x & 31] : 0.f;
        x = norm_warp_sum(x);
    }
    return x;
}

// ---- forward -----------------------------------------------------------------------------------------------------------
struct NormIn {
    const void *x, *residual, *gain;      // residual, gain: may be null
    int gain_bf16;
    long long rows, x_stride, residual_stride, total_stride;
    int cols;
    float eps;
    void *total, *out;                    // may be null
    uint2 *codes;                         // may be null; rows of round_up(cols, 32) codes
    uint8_t *scales;
    float *rstd;
    int aligned;                          // every row and the gain allow vectors
};

// What is left of a row's unit once its normalised values n are known.
template <typename T>
__device__ __forceinline__ void norm_outputs(const NormIn &in, long long row, int unit, const Unit &n, const Unit &gain, bool live)
{
    const int col = unit * kUnit, left = in.cols - col, units = (in.cols + kPackBlock - 1) / kPackBlock * (kPackBlock / kUnit);
    if (in.codes) {                                       // the whole warp: lanes of a block work together
        unsigned scale;
        const uint2 codes = pack_unit(n, scale);
        if (unit < units) {
            in.codes[row * units + unit] = codes;
            if ((unit & 3) == 0) in.scales[row * (units / 4) + unit / 4] = static_cast<uint8_t>(scale);
        }
    }
    if (in.out && live) {
        Unit y;
#pragma unroll
        for (int k = 0; k < kUnit; ++k) y.v[k] = n.v[k] * gain.v[k];
        store_unit(static_cast<T *>(in.out) + row * in.cols + col, y, left, in.aligned && left >= kUnit);
    }
}

// total = round(x + residual), r = 1 / sqrt(mean(total^2) + eps), n = total r; out = round(n gain), codes of n.
// WARPS warps a row (one warp: a block has kNormRows rows), UNITS units a thread: the row stays in registers between its sum and its outputs, so
// each byte crosses HBM once.
constexpr int kNormRows = 4;
template <typename T, int WARPS, int UNITS>
__global__ void __launch_bounds__(WARPS == 1 ? 32 * kNormRows : 32 * WARPS) rms_norm_kernel(const __grid_constant__ NormIn in)
{
    __shared__ float part[2][32];
    constexpr int T_ROW = 32 * WARPS;
    const int tid = WARPS == 1 ? threadIdx.x & 31 : threadIdx.x;
    const long long row = WARPS == 1 ? static_cast<long long>(blockIdx.x) * kNormRows + (threadIdx.x >> 5) : blockIdx.x;
    if (row >= in.rows) return;                            // a whole warp, and no barrier in that form
    const T *x = static_cast<const T *>(in.x) + row * in.x_stride, *res = static_cast<const T *>(in.residual) + (in.residual ? row * in.residual_stride : 0);
    RawUnit<T> a[UNITS], b[UNITS];
#pragma unroll
    for (int j = 0; j < UNITS; ++j) {
        const int col = (j * T_ROW + tid) * kUnit, left = in.cols - col;
        if (left > 0) {
            load_unit(a[j], x + col, left, in.aligned && left >= kUnit);
            if (in.residual) load_unit(b[j], res + col, left, in.aligned && left >= kUnit);
        }
    }
    Unit u[UNITS];
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < UNITS; ++j) {
        const int col = (j * T_ROW + tid) * kUnit, left = in.cols - col;
        if (left > 0) {
            u[j] = a[j].values();
            if (in.residual) {
                const Unit r = b[j].values();
#pragma unroll
                for (int k = 0; k < kUnit; ++k) u[j].v[k] = rounded<T>(u[j].v[k] + r.v[k]);
            }
            if (in.total) store_unit(static_cast<T *>(in.total) + row * in.total_stride + col, u[j], left, in.aligned && left >= kUnit);
        } else {
#pragma unroll
            for (int k = 0; k < kUnit; ++k) u[j].v[k] = 0.f;
        }
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < kUnit; ++k) s = fmaf(u[j].v[k], u[j].v[k], s);
        sum += s;
    }
    sum = row_sum<WARPS>(sum, part, 0);
    const float r = __frsqrt_rn(sum / static_cast<float>(in.cols) + in.eps);
    if (tid == 0) in.rstd[row] = r;
#pragma unroll
    for (int j = 0; j < UNITS; ++j) {
        const int unit = j * T_ROW + tid, left = in.cols - unit * kUnit;
        if (j * T_ROW * kUnit >= in.cols) break;           // the same for the whole row
#pragma unroll
        for (int k = 0; k < kUnit; ++k) u[j].v[k] *= r;
        Unit gain{};
        if (in.out && left > 0) gain = load_gain(in.gain, in.gain_bf16, unit * kUnit, left, in.aligned && left >= kUnit);
        norm_outputs<T>(in, row, unit, u[j], gain, left > 0);
    }
}

// Rows longer than the registers of a block: read twice (the second time mostly from the L2), squares added up in fp64 across a thread's units.
constexpr int kLongThreads = 512;
template <typename T>
__global__ void __launch_bounds__(kLongThreads) rms_norm_long_kernel(const __grid_constant__ NormIn in)
{
    __shared__ double part[kLongThreads / 32];
    const long long row = blockIdx.x;
    const T *x = static_cast<const T *>(in.x) + row * in.x_stride, *res = static_cast<const T *>(in.residual) + (in.residual ? row * in.residual_stride : 0);
    T *total = static_cast<T *>(in.total) + (in.total ? row * in.total_stride : 0);
    const auto values = [&](int col, int left) {
        const bool whole = in.aligned && left >= kUnit;
        RawUnit<T> a, b;
        load_unit(a, x + col, left, whole);
        Unit u = a.values();
        if (in.residual) {
            load_unit(b, res + col, left, whole);
            const Unit r = b.values();
#pragma unroll
            for (int k = 0; k < kUnit; ++k) u.v[k] = rounded<T>(u.v[k] + r.v[k]);
        }
        return u;
    };
    double sum = 0;
    for (int col = threadIdx.x * kUnit; col < in.cols; col += kLongThreads * kUnit) {
        const Unit u = values(col, in.cols - col);
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < kUnit; ++k) s = fmaf(u.v[k], u.v[k], s);
        sum += s;
    }
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(kAllLanes, sum, o);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = sum;
    __syncthreads();
    sum = 0;
    for (int k = 0; k < kLongThreads / 32; ++k) sum += part[k];
    const float r = __frsqrt_rn(static_cast<float>(sum / in.cols) + in.eps);
    if (threadIdx.x == 0) in.rstd[row] = r;
    const int units = (in.cols + kPackBlock - 1) / kPackBlock * (kPackBlock / kUnit);
    for (int first = 0; first < units; first += kLongThreads) {           // a unit is read and, where total replaces its source, written by one thread
        const int unit = first + static_cast<int>(threadIdx.x), col = unit * kUnit, left = in.cols - col;
        Unit u{}, gain{};
        if (left > 0) {
            u = values(col, left);
            if (in.total) store_unit(total + col, u, left, in.aligned && left >= kUnit);
            if (in.out) gain = load_gain(in.gain, in.gain_bf16, col, left, in.aligned && left >= kUnit);
        }
#pragma unroll
        for (int k = 0; k < kUnit; ++k) u.v[k] *= r;
        norm_outputs<T>(in, row, unit, u, gain, left > 0);
    }
}

// ---- backward ----------------------------------------------------------------------------------------------------------
struct NormGradIn {
    const void *dout, *gain, *dtotal, *total;      // gain, dtotal: may be null; total: null where the codes are given
    const uint2 *codes;
    const uint8_t *scales;
    const float *rstd;
    void *dx;
    float *parts;                                  // one row of `cols` for each block, or null: no gradient of the gain
    int gain_bf16;
    long long rows, dout_stride, dtotal_stride, total_stride;
    int cols;
    int aligned;
};

// n of one unit, from the codes or from the total.
template <typename T>
struct KeptUnit {
    RawUnit<T> raw;
    uint2 codes;
    unsigned scale;
    __device__ __forceinline__ void load(const NormGradIn &in, long long row, int unit, int left)
    {
        if (in.codes) {
            const int units = (in.cols + kPackBlock - 1) / kPackBlock * (kPackBlock / kUnit);
            codes = __ldcs(in.codes + row * units + unit);
            scale = __ldcs(in.scales + row * (units / 4) + unit / 4);
        } else {
            load_unit(raw, static_cast<const T *>(in.total) + row * in.total_stride + unit * kUnit, left, in.aligned && left >= kUnit);
        }
    }
    __device__ __forceinline__ Unit values(const NormGradIn &in, float rstd) const
    {
        if (in.codes) return unpack_unit(codes, scale);
        Unit u = raw.values();
#pragma unroll
        for (int k = 0; k < kUnit; ++k) u.v[k] *= rstd;
        return u;
    }
};

// g = dout gain, dx = dtotal + r (g - n mean(g n)), and each block's part of dgain = sum of dout n over its rows: rows are dealt out in turn, so
// the parts, and their sum in the next kernel, have a fixed order.
template <typename T, int WARPS, int UNITS>
__global__ void __launch_bounds__(WARPS == 1 ? 32 * kNormRows : 32 * WARPS) rms_norm_grad_kernel(const __grid_constant__ NormGradIn in)
{
    __shared__ float part[2][32];
    constexpr int T_ROW = 32 * WARPS, GROUPS = WARPS == 1 ? kNormRows : 1;
    const int tid = WARPS == 1 ? threadIdx.x & 31 : threadIdx.x, group = WARPS == 1 ? threadIdx.x >> 5 : 0;
    Unit acc[UNITS];
#pragma unroll
    for (int j = 0; j < UNITS; ++j)
#pragma unroll
        for (int k = 0; k < kUnit; ++k) acc[j].v[k] = 0.f;
    int slot = 0;
    for (long long row = static_cast<long long>(blockIdx.x) * GROUPS + group; row < in.rows; row += static_cast<long long>(gridDim.x) * GROUPS, slot ^= 1) {
        const T *dout = static_cast<const T *>(in.dout) + row * in.dout_stride;
        const T *dtotal = static_cast<const T *>(in.dtotal) + (in.dtotal ? row * in.dtotal_stride : 0);
        RawUnit<T> d[UNITS], t[UNITS];
        KeptUnit<T> kept[UNITS];
        const float r = in.rstd[row];
#pragma unroll
        for (int j = 0; j < UNITS; ++j) {
            const int unit = j * T_ROW + tid, left = in.cols - unit * kUnit;
            if (left > 0) {
                load_unit(d[j], dout + unit * kUnit, left, in.aligned && left >= kUnit);
                kept[j].load(in, row, unit, left);
                if (in.dtotal) load_unit(t[j], dtotal + unit * kUnit, left, in.aligned && left >= kUnit);
            }
        }
        Unit g[UNITS], n[UNITS];
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < UNITS; ++j) {
            const int unit = j * T_ROW + tid, left = in.cols - unit * kUnit;
            if (left <= 0) continue;
            g[j] = d[j].values();
            n[j] = kept[j].values(in, r);
            const Unit gain = load_gain(in.gain, in.gain_bf16, unit * kUnit, left, in.aligned && left >= kUnit);
            float s = 0.f;
#pragma unroll
            for (int k = 0; k < kUnit; ++k) {
                acc[j].v[k] = fmaf(g[j].v[k], n[j].v[k], acc[j].v[k]);
                g[j].v[k] *= gain.v[k];
                s = fmaf(g[j].v[k], n[j].v[k], s);
            }
            sum += s;
        }
        const float mean = row_sum<WARPS>(sum, part, slot) / static_cast<float>(in.cols);
#pragma unroll
        for (int j = 0; j < UNITS; ++j) {
            const int col = (j * T_ROW + tid) * kUnit, left = in.cols - col;
            if (left <= 0) continue;
            Unit dx;
#pragma unroll
            for (int k = 0; k < kUnit; ++k) dx.v[k] = r * fmaf(-n[j].v[k], mean, g[j].v[k]);
            if (in.dtotal) {
                const Unit more = t[j].values();
#pragma unroll
                for (int k = 0; k < kUnit; ++k) dx.v[k] += more.v[k];
            }
            store_unit(static_cast<T *>(in.dx) + row * in.cols + col, dx, left, in.aligned && left >= kUnit);
        }
    }
    if (!in.parts) return;
#pragma unroll
    for (int j = 0; j < UNITS; ++j) {
        const int col = (j * T_ROW + tid) * kUnit;
        float *to = in.parts + (static_cast<long long>(blockIdx.x) * GROUPS + group) * in.cols + col;
#pragma unroll
        for (int k = 0; k < kUnit; ++k) if (col + k < in.cols) to[k] = acc[j].v[k];
    }
}

// Longer rows: dout and the kept values are read twice (the second time mostly from the L2); the gain's gradient is a kernel of its own.
template <typename T>
__global__ void __launch_bounds__(kLongThreads) rms_norm_grad_long_kernel(const __grid_constant__ NormGradIn in)
{
    __shared__ double part[kLongThreads / 32];
    const long long row = blockIdx.x;
    const float r = in.rstd[row];
    const auto values = [&](int unit, int left, Unit &g, Unit &n) {
        RawUnit<T> d;
        KeptUnit<T> kept;
        load_unit(d, static_cast<const T *>(in.dout) + row * in.dout_stride + unit * kUnit, left, in.aligned && left >= kUnit);
        kept.load(in, row, unit, left);
        g = d.values();
        n = kept.values(in, r);
        const Unit gain = load_gain(in.gain, in.gain_bf16, unit * kUnit, left, in.aligned && left >= kUnit);
#pragma unroll
        for (int k = 0; k < kUnit; ++k) g.v[k] *= gain.v[k];
    };
    double sum = 0;
    for (int unit = threadIdx.x; unit * kUnit < in.cols; unit += kLongThreads) {
        Unit g, n;
        values(unit, in.cols - unit * kUnit, g, n);
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < kUnit; ++k) s = fmaf(g.v[k], n.v[k], s);
        sum += s;
    }
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(kAllLanes, sum, o);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = sum;
    __syncthreads();
    sum = 0;
    for (int k = 0; k < kLongThreads / 32; ++k) sum += part[k];
    const float mean = static_cast<float>(sum / in.cols);
    for (int unit = threadIdx.x; unit * kUnit < in.cols; unit += kLongThreads) {
        const int col = unit * kUnit, left = in.cols - col;
        Unit g, n, dx;
        values(unit, left, g, n);
#pragma unroll
        for (int k = 0; k < kUnit; ++k) dx.v[k] = r * fmaf(-n.v[k], mean, g.v[k]);
        if (in.dtotal) {
            RawUnit<T> t;
            load_unit(t, static_cast<const T *>(in.dtotal) + row * in.dtotal_stride + col, left, in.aligned && left >= kUnit);
            const Unit more = t.values();
#pragma unroll
            for (int k = 0; k < kUnit; ++k) dx.v[k] += more.v[k];
        }
        store_unit(static_cast<T *>(in.dx) + row * in.cols + col, dx, left, in.aligned && left >= kUnit);
    }
}
template <typename T>
__global__ void __launch_bounds__(128) gain_grad_long_kernel(const __grid_constant__ NormGradIn in)
{
    const int unit = static_cast<int>(blockIdx.x) * 128 + static_cast<int>(threadIdx.x), left = in.cols - unit * kUnit;
    if (left <= 0) return;
    Unit acc{};
    for (long long row = blockIdx.y; row < in.rows; row += gridDim.y) {
        RawUnit<T> d;
        KeptUnit<T> kept;
        load_unit(d, static_cast<const T *>(in.dout) + row * in.dout_stride + unit * kUnit, left, in.aligned && left >= kUnit);
        kept.load(in, row, unit, left);
        const Unit g = d.values(), n = kept.values(in, in.rstd[row]);
#pragma unroll
        for (int k = 0; k < kUnit; ++k) acc.v[k] = fmaf(g.v[k], n.v[k], acc.v[k]);
    }
    float *to = in.parts + static_cast<long long>(blockIdx.y) * in.cols + unit * kUnit;
#pragma unroll
    for (int k = 0; k < kUnit; ++k) if (k < left) to[k] = acc.v[k];
}

// dgain: the parts added up, 32 columns a block, every warp a share of the parts.
constexpr int kGainWarps = 16;
__global__ void __launch_bounds__(32 * kGainWarps) gain_grad_kernel(const float *parts, int count, int cols, void *dgain, int is_bf16)
{
    __shared__ float sums[kGainWarps][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, col = static_cast<int>(blockIdx.x) * 32 + lane;
    float s = 0.f;
    if (col < cols)
        for (int k = warp; k < count; k += kGainWarps) s += parts[static_cast<long long>(k) * cols + col];
    sums[warp][lane] = s;
    __syncthreads();
    if (warp || col >= cols) return;
    for (int k = 1; k < kGainWarps; ++k) s += sums[k][lane];
    if (is_bf16) static_cast<__nv_bfloat16 *>(dgain)[col] = __float2bfloat16_rn(s);
    else static_cast<float *>(dgain)[col] = s;
}

// ---- packing and unpacking ---------------------------------------------------------------------------------------------
// One unit a thread and turn, kPackTurns of them under way; a row's units are padded to whole blocks.  Bound by HBM.
constexpr int kPackThreads = 256, kPackTurns = 4;
template <typename T>
__global__ void __launch_bounds__(kPackThreads) pack_kernel(const T *x, long long rows, int cols, long long stride, uint2 *codes, uint8_t *scales, int aligned)
{
    const int units = (cols + kPackBlock - 1) / kPackBlock * (kPackBlock / kUnit);
    const long long count = rows * units, base = static_cast<long long>(blockIdx.x) * (kPackThreads * kPackTurns) + threadIdx.x;
    RawUnit<T> raw[kPackTurns];
#pragma unroll
    for (int j = 0; j < kPackTurns; ++j) {
        const long long at = base + j * kPackThreads;
        const long long row = at / units;
        const int col = static_cast<int>(at - row * units) * kUnit, left = at < count ? cols - col : 0;
        load_unit(raw[j], x + (left > 0 ? row * stride + col : 0), left, aligned && left >= kUnit);
    }
#pragma unroll
    for (int j = 0; j < kPackTurns; ++j) {
        const long long at = base + j * kPackThreads;
        unsigned scale;
        const uint2 c = pack_unit(raw[j].values(), scale);
        if (at < count) {
            codes[at] = c;
            if ((at & 3) == 0) scales[at >> 2] = static_cast<uint8_t>(scale);
        }
    }
}
template <typename T>
__global__ void __launch_bounds__(kPackThreads) unpack_kernel(const uint2 *codes, const uint8_t *scales, long long rows, int cols, T *out, long long stride, int aligned)
{
    const int units = (cols + kPackBlock - 1) / kPackBlock * (kPackBlock / kUnit);
    const long long count = rows * units, base = static_cast<long long>(blockIdx.x) * (kPackThreads * kPackTurns) + threadIdx.x;
    uint2 c[kPackTurns];
    unsigned s[kPackTurns];
#pragma unroll
    for (int j = 0; j < kPackTurns; ++j) {
        const long long at = base + j * kPackThreads;
        if (at < count) { c[j] = __ldcs(codes + at); s[j] = __ldcs(scales + (at >> 2)); }
    }
#pragma unroll
    for (int j = 0; j < kPackTurns; ++j) {
        const long long at = base + j * kPackThreads;
        if (at >= count) break;
        const long long row = at / units;
        const int col = static_cast<int>(at - row * units) * kUnit, left = cols - col;
        if (left > 0) store_unit(out + row * stride + col, unpack_unit(c[j], s[j]), left, aligned && left >= kUnit);
    }
}

}  // namespace softsync
