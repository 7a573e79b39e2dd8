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
        if constexpr (WARPS <= 8) {                        // a few broadcast loads, instead of another tree
            const float4 *p = reinterpret_cast<const float4 *>(part[slot]);
            float4 s = p[0];
#pragma unroll
            for (int k = 1; k < WARPS / 4; ++k) { const float4 t = p[k]; s.x += t.x; s.y += t.y; s.z += t.z; s.w += t.w; }
            x = (s.x + s.y) + (s.z + s.w);
        } else {
            x = (threadIdx.x & 31) < WARPS ? part[slot][threadIdx.x & 31] : 0.f;
            x = norm_warp_sum(x);
        }
    }
    return x;
}

// Whether a row's mean square plus eps, made in fp32, is what it should be: no square or sum overflowed, and what vanished below 2^-126 (at most 2^-150 of the mean) does not matter beside it.
// Otherwise the squares are those of the values times a power of two: of large rows 2^-80 (of values up to 2^128, up to 2^28 of them; what vanishes is nothing beside one of 2^49 and more),
// of small ones 2^100 (values below 2^-46, since their mean square is below 2^-120; the least subnormal's square is a normal number).
__device__ __forceinline__ bool mean_square_fits(float m) { return m >= 7.52316385e-37f && m <= 3.40282347e38f; }              // 2^-120, the largest

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
};

// What is left of a row's unit once its normalised values n are known; by whole warps.
template <typename T, bool ALIGNED>
__device__ __forceinline__ void norm_outputs(const NormIn &in, long long row, int unit, const Unit &n, const Unit &gain, WarpDesk<T> *desk)
{
    const int units = (in.cols + kPackBlock - 1) / kPackBlock * (kPackBlock / kUnit);
    if (in.codes) {                                       // the whole warp: lanes of a block work together
        unsigned scale;
        const uint2 codes = pack_unit(n, scale);
        if (unit < units) {
            in.codes[row * units + unit] = codes;
            if ((unit & 3) == 0) in.scales[row * (units / 4) + unit / 4] = static_cast<uint8_t>(scale);
        }
    }
    if (in.out) {
        Unit y;
#pragma unroll
        for (int k = 0; k < kUnitPairs; ++k) y.set(k, mul2(n.pair(k), gain.pair(k)));
        store_row<ALIGNED>(static_cast<T *>(in.out) + row * in.cols, unit, in.cols, y, desk);
    }
}

// total = round(x + residual), r = 1 / sqrt(mean(total^2) + eps), n = total r; out = round(n gain), codes of n.  Rows whose squares overflow fp32 (values around 1e18 and more), or vanish in it beside an
// eps that does too, are added up again times a power of two: the row is there, and the test for it costs nothing (one comparison a row).
// WARPS warps a row (one warp: a block has kNormRows rows), UNITS units a thread: the row stays in registers between its sum and its outputs, so
// each byte crosses HBM once.  Bound by HBM: 16384 x 4096 bf16 with residual and both outputs moves 606 MB in 93 us (6.5 TB/s).
constexpr int kNormRows = 4;
// Blocks that an SM has registers for, where the compiler would take a few too many for them (bf16, 64 M elements: 16384 wide 130 us with one block and 96 with two, 512 wide 98 with eight and 95 with
// nine); 0: as it likes.
template <typename T, int WARPS, int UNITS> constexpr int kNormBlocks = sizeof(T) == 4 ? 0 : WARPS == 16 && UNITS == 4 ? 2 : WARPS == 1 && UNITS == 2 ? 9 : 0;
template <typename T, int WARPS, int UNITS, bool ALIGNED>
__global__ void __launch_bounds__(WARPS == 1 ? 32 * kNormRows : 32 * WARPS, kNormBlocks<T, WARPS, UNITS>) rms_norm_kernel(const __grid_constant__ NormIn in)
{
    __shared__ __align__(16) float part[2][32];
    __shared__ WarpDesk<T> desk[ALIGNED ? 1 : WARPS == 1 ? kNormRows : WARPS];
    constexpr int T_ROW = 32 * WARPS;
    wait_for_earlier();
    let_next_start();
    const int tid = WARPS == 1 ? threadIdx.x & 31 : threadIdx.x;
    const long long row = WARPS == 1 ? static_cast<long long>(blockIdx.x) * kNormRows + (threadIdx.x >> 5) : blockIdx.x;
    if (row >= in.rows) return;                            // a whole warp, and no barrier in that form
    const T *x = static_cast<const T *>(in.x) + row * in.x_stride, *res = static_cast<const T *>(in.residual) + (in.residual ? row * in.residual_stride : 0);
    RawUnit<T> a[UNITS], b[UNITS];
#pragma unroll
    for (int j = 0; j < UNITS; ++j) {
        const int col = (j * T_ROW + tid) * kUnit, left = in.cols - col;
        if (left > 0) {
            load_unit(a[j], x + col, left, ALIGNED && left >= kUnit);
            if (in.residual) load_unit(b[j], res + col, left, ALIGNED && left >= kUnit);
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
                for (int k = 0; k < kUnitPairs; ++k) u[j].set(k, rounded<T>(add2(u[j].pair(k), r.pair(k))));
            }
        } else {
#pragma unroll
            for (int k = 0; k < kUnit; ++k) u[j].v[k] = 0.f;
        }
        if (in.total) store_row<ALIGNED>(static_cast<T *>(in.total) + row * in.total_stride, j * T_ROW + tid, in.cols, u[j], desk);
        float2 s = make_float2(0.f, 0.f);
#pragma unroll
        for (int k = 0; k < kUnitPairs; ++k) s = fma2(u[j].pair(k), u[j].pair(k), s);
        sum += s.x + s.y;
    }
    sum = row_sum<WARPS>(sum, part, 0);
    const float m = sum / static_cast<float>(in.cols) + in.eps;
    float r = __frsqrt_rn(m);
    if (!mean_square_fits(m)) {                            // the same for the whole row
        const float scale = m < 1.f ? 1.26765060e30f : 8.27180613e-25f;               // 2^100, 2^-80
        sum = 0.f;
#pragma unroll
        for (int j = 0; j < UNITS; ++j)
#pragma unroll
            for (int k = 0; k < kUnit; ++k) {
                const float v = u[j].v[k] * scale;
                sum = fmaf(v, v, sum);
            }
        r = __frsqrt_rn(row_sum<WARPS>(sum, part, 1) / static_cast<float>(in.cols) + in.eps * scale * scale) * scale;
    }
    if (tid == 0) in.rstd[row] = r;
#pragma unroll
    for (int j = 0; j < UNITS; ++j) {
        const int unit = j * T_ROW + tid, left = in.cols - unit * kUnit;
        if (j * T_ROW * kUnit >= in.cols) break;           // the same for the whole row
#pragma unroll
        for (int k = 0; k < kUnitPairs; ++k) u[j].set(k, mul2(u[j].pair(k), make_float2(r, r)));
        Unit gain{};
        if (in.out && left > 0) gain = load_gain(in.gain, in.gain_bf16, unit * kUnit, left, ALIGNED && left >= kUnit);
        norm_outputs<T, ALIGNED>(in, row, unit, u[j], gain, desk);
    }
}

// Rows longer than the registers of a block: read twice (the second time mostly from the L2), squares added up in fp64 across a thread's units.
constexpr int kLongThreads = 512;
template <typename T, bool ALIGNED>
__global__ void __launch_bounds__(kLongThreads) rms_norm_long_kernel(const __grid_constant__ NormIn in)
{
    __shared__ double part[kLongThreads / 32];
    __shared__ WarpDesk<T> desk[ALIGNED ? 1 : kLongThreads / 32];
    wait_for_earlier();
    let_next_start();
    const long long row = blockIdx.x;
    const T *x = static_cast<const T *>(in.x) + row * in.x_stride, *res = static_cast<const T *>(in.residual) + (in.residual ? row * in.residual_stride : 0);
    T *total = static_cast<T *>(in.total) + (in.total ? row * in.total_stride : 0);
    const auto values = [&](int col, int left) {
        const bool whole = ALIGNED && left >= kUnit;
        RawUnit<T> a, b;
        load_unit(a, x + col, left, whole);
        Unit u = a.values();
        if (in.residual) {
            load_unit(b, res + col, left, whole);
            const Unit r = b.values();
#pragma unroll
            for (int k = 0; k < kUnitPairs; ++k) u.set(k, rounded<T>(add2(u.pair(k), r.pair(k))));
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
    float r = __frsqrt_rn(static_cast<float>(sum / in.cols) + in.eps);
    if (!mean_square_fits(static_cast<float>(sum / in.cols) + in.eps)) {
        sum = 0;
        for (int col = threadIdx.x * kUnit; col < in.cols; col += kLongThreads * kUnit) {
            const Unit u = values(col, in.cols - col);
            for (int k = 0; k < kUnit; ++k) sum = fma(static_cast<double>(u.v[k]), static_cast<double>(u.v[k]), sum);
        }
        for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(kAllLanes, sum, o);
        __syncthreads();                                   // the first sums have been read
        if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = sum;
        __syncthreads();
        sum = 0;
        for (int k = 0; k < kLongThreads / 32; ++k) sum += part[k];
        r = static_cast<float>(1.0 / sqrt(sum / in.cols + in.eps));
    }
    if (threadIdx.x == 0) in.rstd[row] = r;
    const int units = (in.cols + kPackBlock - 1) / kPackBlock * (kPackBlock / kUnit);
    for (int first = 0; first < units; first += kLongThreads) {           // a unit is read and, where total replaces its source, written by one thread
        const int unit = first + static_cast<int>(threadIdx.x), col = unit * kUnit, left = in.cols - col;
        Unit u{}, gain{};
        if (left > 0) {
            u = values(col, left);
            if (in.out) gain = load_gain(in.gain, in.gain_bf16, col, left, ALIGNED && left >= kUnit);
        }
        if (in.total) {
            __syncwarp();                                  // total may be the residual: no lane writes before all have read
            store_row<ALIGNED>(total, unit, in.cols, u, desk);
        }
#pragma unroll
        for (int k = 0; k < kUnit; ++k) u.v[k] *= r;
        norm_outputs<T, ALIGNED>(in, row, unit, u, gain, desk);
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
};

// n of one unit, from the codes or from the total.
template <typename T, bool CODES, bool ALIGNED> struct KeptUnit;
template <typename T, bool ALIGNED> struct KeptUnit<T, true, ALIGNED> {
    uint2 codes;
    unsigned scale;
    __device__ __forceinline__ void load(const NormGradIn &in, long long row, int unit, int)
    {
        const int units = (in.cols + kPackBlock - 1) / kPackBlock * (kPackBlock / kUnit);
        codes = __ldcs(in.codes + row * units + unit);
        scale = __ldcs(in.scales + row * (units / 4) + unit / 4);
    }
    __device__ __forceinline__ Unit values(float) const { return unpack_unit(codes, scale); }
};
template <typename T, bool ALIGNED> struct KeptUnit<T, false, ALIGNED> {
    RawUnit<T> raw;
    __device__ __forceinline__ void load(const NormGradIn &in, long long row, int unit, int left)
    {
        load_unit(raw, static_cast<const T *>(in.total) + row * in.total_stride + unit * kUnit, left, ALIGNED && left >= kUnit);
    }
    __device__ __forceinline__ Unit values(float rstd) const
    {
        Unit u = raw.values();
#pragma unroll
        for (int k = 0; k < kUnit; ++k) u.v[k] *= rstd;
        return u;
    }
};

// Warps of an SM: as many as have registers for what a thread holds of two rows.
template <typename T, int UNITS> constexpr int kGradWarps = UNITS == 1 && sizeof(T) == 2 ? 32 : 16;

// What a thread loads of one row.
template <typename T, int WARPS, int UNITS, bool CODES, bool ALIGNED>
struct GradRow {
    RawUnit<T> dout[UNITS], dtotal[UNITS];
    KeptUnit<T, CODES, ALIGNED> kept[UNITS];
    float rstd;
    __device__ __forceinline__ void load(const NormGradIn &in, long long row, int tid)
    {
        const T *d = static_cast<const T *>(in.dout) + row * in.dout_stride, *t = static_cast<const T *>(in.dtotal) + (in.dtotal ? row * in.dtotal_stride : 0);
        rstd = in.rstd[row];
#pragma unroll
        for (int j = 0; j < UNITS; ++j) {
            const int unit = j * 32 * WARPS + tid, left = in.cols - unit * kUnit;
            if (left <= 0) continue;
            load_unit(dout[j], d + unit * kUnit, left, ALIGNED && left >= kUnit);
            kept[j].load(in, row, unit, left);
            if (in.dtotal) load_unit(dtotal[j], t + unit * kUnit, left, ALIGNED && left >= kUnit);
        }
    }
};

// g = dout gain, dx = dtotal + r (g - n mean(g n)), and each block's part of dgain = sum of dout n over its rows: rows are dealt out in turn, so
// the parts, and their sum in the next kernel, have a fixed order.  The next row's loads are under way while a row waits for its sum.
template <typename T, int WARPS, int UNITS, bool CODES, bool ALIGNED>
__global__ void __launch_bounds__(WARPS == 1 ? 32 * kNormRows : 32 * WARPS, kGradWarps<T, UNITS> / (WARPS == 1 ? kNormRows : WARPS)) rms_norm_grad_kernel(const __grid_constant__ NormGradIn in)
{
    __shared__ __align__(16) float part[2][32];
    __shared__ WarpDesk<T> desk[ALIGNED ? 1 : WARPS == 1 ? kNormRows : WARPS];
    constexpr int T_ROW = 32 * WARPS, GROUPS = WARPS == 1 ? kNormRows : 1;
    wait_for_earlier();
    let_next_start();
    const int tid = WARPS == 1 ? threadIdx.x & 31 : threadIdx.x, group = WARPS == 1 ? threadIdx.x >> 5 : 0;
    Unit acc[UNITS];
#pragma unroll
    for (int j = 0; j < UNITS; ++j)
#pragma unroll
        for (int k = 0; k < kUnit; ++k) acc[j].v[k] = 0.f;
    int slot = 0;
    const long long step = static_cast<long long>(gridDim.x) * GROUPS;
    long long row = static_cast<long long>(blockIdx.x) * GROUPS + group;
    GradRow<T, WARPS, UNITS, CODES, ALIGNED> next;
    if (row < in.rows) next.load(in, row, tid);
    for (; row < in.rows; row += step, slot ^= 1) {
        const float r = next.rstd;
        Unit g[UNITS], n[UNITS];
        RawUnit<T> more[UNITS];
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < UNITS; ++j) {
            const int unit = j * T_ROW + tid, left = in.cols - unit * kUnit;
            if (left <= 0) continue;
            g[j] = next.dout[j].values();
            n[j] = next.kept[j].values(r);
            more[j] = next.dtotal[j];
            const Unit gain = load_gain(in.gain, in.gain_bf16, unit * kUnit, left, ALIGNED && left >= kUnit);
            float s = 0.f;
#pragma unroll
            for (int k = 0; k < kUnit; ++k) {
                acc[j].v[k] = fmaf(g[j].v[k], n[j].v[k], acc[j].v[k]);
                g[j].v[k] *= gain.v[k];
                s = fmaf(g[j].v[k], n[j].v[k], s);
            }
            sum += s;
        }
        if (row + step < in.rows) next.load(in, row + step, tid);
        const float mean = row_sum<WARPS>(sum, part, slot) / static_cast<float>(in.cols);
#pragma unroll
        for (int j = 0; j < UNITS; ++j) {
            const int unit = j * T_ROW + tid;
            if (ALIGNED && unit * kUnit >= in.cols) continue;
            Unit dx{};
            if (ALIGNED || unit * kUnit < in.cols) {
#pragma unroll
                for (int k = 0; k < kUnit; ++k) dx.v[k] = r * fmaf(-n[j].v[k], mean, g[j].v[k]);
                if (in.dtotal) {
                    const Unit m = more[j].values();
#pragma unroll
                    for (int k = 0; k < kUnit; ++k) dx.v[k] += m.v[k];
                }
            }
            store_row<ALIGNED>(static_cast<T *>(in.dx) + row * in.cols, unit, in.cols, dx, desk);
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

// The same for rows whose bytes are whole vectors, from the codes: rows come by bulk copies into a ring of shared memory, several ahead, and a thread's registers hold one row. (With the next row's
// loads in registers instead the same arithmetic takes 96 us where this takes 77, 4096 wide, 64 M elements of bf16.)  Bound by HBM: 472 MB in 72 us, then 7 for the gain's.
//
// A slot is free once every thread has taken its part, which the barrier of the row's sum shows.  Waits are bounded: one that runs out makes the rest of the block's rows
// NaN, and its thread's columns of the block's part; it waits for nothing after that but the copies under way, with the same limit.
constexpr int kNormWaitLimit = 1 << 20, kMostSlots = 8;
__device__ __forceinline__ unsigned norm_smem(const void *p) { return static_cast<unsigned>(__cvta_generic_to_shared(p)); }
__device__ __forceinline__ bool norm_wait(unsigned bar, unsigned parity)
{
    for (int tries = 0; tries < kNormWaitLimit; ++tries) {
        unsigned ok;
        asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(ok) : "r"(bar), "r"(parity), "r"(1000u) : "memory");
        if (ok) return true;
    }
    return false;
}
__device__ __forceinline__ void norm_copy(unsigned to, const void *from, unsigned bytes, unsigned bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" :: "r"(to), "l"(from), "r"(bytes), "r"(bar) : "memory");
}

struct GradRing { int slots, row_bytes, code_bytes, slot_bytes; };          // of a row of activations, of codes, of all that a slot holds
template <typename T, int WARPS, int UNITS>
__global__ void __launch_bounds__(32 * WARPS, kGradWarps<T, UNITS> / WARPS) rms_norm_grad_ring_kernel(const __grid_constant__ NormGradIn in, const __grid_constant__ GradRing ring)
{
    extern __shared__ __align__(128) unsigned char slots[];
    __shared__ __align__(16) float part[2][32];
    __shared__ __align__(8) unsigned long long full[kMostSlots];
    constexpr int T_ROW = 32 * WARPS;
    const int tid = threadIdx.x, units = in.cols / kUnit, blocks = (in.cols + kPackBlock - 1) / kPackBlock;
    if (tid == 0) {
        for (int k = 0; k < ring.slots; ++k) asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" :: "r"(norm_smem(&full[k])) : "memory");
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    wait_for_earlier();
    let_next_start();
    const long long step = gridDim.x;
    const auto fetch = [&](long long row, int slot) {
        const unsigned bar = norm_smem(&full[slot]), to = norm_smem(slots + slot * ring.slot_bytes);
        asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" :: "r"(bar), "r"(ring.row_bytes * (in.dtotal ? 2 : 1) + ring.code_bytes) : "memory");
        norm_copy(to, static_cast<const T *>(in.dout) + row * in.dout_stride, ring.row_bytes, bar);
        norm_copy(to + ring.row_bytes, reinterpret_cast<const unsigned char *>(in.codes) + row * ring.code_bytes, ring.code_bytes, bar);
        if (in.dtotal) norm_copy(to + ring.row_bytes + ring.code_bytes, static_cast<const T *>(in.dtotal) + row * in.dtotal_stride, ring.row_bytes, bar);
    };
    long long row = blockIdx.x;
    if (tid == 0)
        for (int k = 0; k < ring.slots; ++k) if (row + k * step < in.rows) fetch(row + k * step, k);
    Unit acc[UNITS];
    unsigned scale[UNITS], next_scale[UNITS];
    float r = 0.f, next_r = 0.f;
    const float *rstd = in.rstd + row;
    const uint8_t *scales = in.scales + row * blocks + tid / 4;
    const auto ahead = [&](long long at) {                 // what is too small to copy in bulk, a row ahead
        if (at >= in.rows) return;
        next_r = *rstd;
#pragma unroll
        for (int j = 0; j < UNITS; ++j) if (j * T_ROW + tid < units) next_scale[j] = scales[j * (T_ROW / 4)];
        rstd += step;
        scales += step * blocks;
    };
    T *dx_row = static_cast<T *>(in.dx) + row * in.cols + tid * kUnit;
    const float share = 1.f / static_cast<float>(in.cols);
#pragma unroll
    for (int j = 0; j < UNITS; ++j) {
        next_scale[j] = 0;
#pragma unroll
        for (int k = 0; k < kUnit; ++k) acc[j].v[k] = 0.f;
    }
    ahead(row);
    Unit gains[UNITS];                                     // of this thread's columns, for all its rows
#pragma unroll
    for (int j = 0; j < UNITS; ++j) if (j * T_ROW + tid < units) gains[j] = load_gain(in.gain, in.gain_bf16, (j * T_ROW + tid) * kUnit, kUnit, true);
    bool late = false;
    int slot = 0, side = 0;
    unsigned parity = 0;
    for (; row < in.rows; row += step, side ^= 1) {
        r = next_r;
#pragma unroll
        for (int j = 0; j < UNITS; ++j) scale[j] = next_scale[j];
        ahead(row + step);
        late = late || !norm_wait(norm_smem(&full[slot]), parity);
        const unsigned char *here = slots + slot * ring.slot_bytes;
        Unit g[UNITS], n[UNITS];
        RawUnit<T> more[UNITS];
        float sum = late ? __int_as_float(0x7fc00000) : 0.f;          // one late thread is enough: the row's mean, and with it the whole row
#pragma unroll
        for (int j = 0; j < UNITS; ++j) {
            const int unit = j * T_ROW + tid;
            if (unit >= units) continue;
            RawUnit<T> d;
            d.take(here + unit * (kUnit * sizeof(T)));
            const uint2 codes = *reinterpret_cast<const uint2 *>(here + ring.row_bytes + unit * kUnit);
            if (in.dtotal) more[j].take(here + ring.row_bytes + ring.code_bytes + unit * (kUnit * sizeof(T)));
            g[j] = d.values();
            n[j] = unpack_unit(codes, scale[j]);
            float2 s = make_float2(0.f, 0.f);
#pragma unroll
            for (int k = 0; k < kUnitPairs; ++k) {
                acc[j].set(k, fma2(g[j].pair(k), n[j].pair(k), acc[j].pair(k)));
                g[j].set(k, mul2(g[j].pair(k), gains[j].pair(k)));
                s = fma2(g[j].pair(k), n[j].pair(k), s);
            }
            sum += s.x + s.y;
        }
        const float mean = row_sum<WARPS>(sum, part, side) * share;
        if (tid == 0 && !late && row + ring.slots * step < in.rows) fetch(row + ring.slots * step, slot);
        if (++slot == ring.slots) { slot = 0; parity ^= 1; }
#pragma unroll
        for (int j = 0; j < UNITS; ++j) {
            const int unit = j * T_ROW + tid;
            if (unit >= units) continue;
            Unit dx;
            if (in.dtotal) {
                const Unit m = more[j].values();
#pragma unroll
                for (int k = 0; k < kUnitPairs; ++k)
                    dx.set(k, fma2(fma2(n[j].pair(k), make_float2(-mean, -mean), g[j].pair(k)), make_float2(r, r), m.pair(k)));
            } else {
#pragma unroll
                for (int k = 0; k < kUnitPairs; ++k) dx.set(k, mul2(fma2(n[j].pair(k), make_float2(-mean, -mean), g[j].pair(k)), make_float2(r, r)));
            }
            store_unit(dx_row + j * (T_ROW * kUnit), dx, kUnit, true);
        }
        dx_row += step * in.cols;
    }
    if (late && tid == 0)                                  // copies may still be under way
        for (int k = 0; k < ring.slots; ++k) { norm_wait(norm_smem(&full[k]), 0); norm_wait(norm_smem(&full[k]), 1); }
    if (!in.parts) return;
#pragma unroll
    for (int j = 0; j < UNITS; ++j) {
        const int unit = j * T_ROW + tid;
        if (unit >= units) continue;
        if (late) {
#pragma unroll
            for (int k = 0; k < kUnit; ++k) acc[j].v[k] = __int_as_float(0x7fc00000);
        }
        float4 *to = reinterpret_cast<float4 *>(in.parts + static_cast<long long>(blockIdx.x) * in.cols + unit * kUnit);
        to[0] = make_float4(acc[j].v[0], acc[j].v[1], acc[j].v[2], acc[j].v[3]);
        to[1] = make_float4(acc[j].v[4], acc[j].v[5], acc[j].v[6], acc[j].v[7]);
    }
}

// Longer rows: dout and the kept values are read twice (the second time mostly from the L2); the gain's gradient is a kernel of its own.
template <typename T, bool CODES, bool ALIGNED>
__global__ void __launch_bounds__(kLongThreads) rms_norm_grad_long_kernel(const __grid_constant__ NormGradIn in)
{
    __shared__ double part[kLongThreads / 32];
    wait_for_earlier();
    let_next_start();
    const long long row = blockIdx.x;
    const float r = in.rstd[row];
    const auto values = [&](int unit, int left, Unit &g, Unit &n) {
        RawUnit<T> d;
        KeptUnit<T, CODES, ALIGNED> kept;
        load_unit(d, static_cast<const T *>(in.dout) + row * in.dout_stride + unit * kUnit, left, ALIGNED && left >= kUnit);
        kept.load(in, row, unit, left);
        g = d.values();
        n = kept.values(r);
        const Unit gain = load_gain(in.gain, in.gain_bf16, unit * kUnit, left, ALIGNED && left >= kUnit);
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
            load_unit(t, static_cast<const T *>(in.dtotal) + row * in.dtotal_stride + col, left, ALIGNED && left >= kUnit);
            const Unit more = t.values();
#pragma unroll
            for (int k = 0; k < kUnit; ++k) dx.v[k] += more.v[k];
        }
        store_unit(static_cast<T *>(in.dx) + row * in.cols + col, dx, left, ALIGNED && left >= kUnit);
    }
}
template <typename T, bool CODES, bool ALIGNED>
__global__ void __launch_bounds__(128) gain_grad_long_kernel(const __grid_constant__ NormGradIn in)
{
    wait_for_earlier();
    let_next_start();
    const int unit = static_cast<int>(blockIdx.x) * 128 + static_cast<int>(threadIdx.x), left = in.cols - unit * kUnit;
    if (left <= 0) return;
    Unit acc{};
    for (long long row = blockIdx.y; row < in.rows; row += gridDim.y) {
        RawUnit<T> d;
        KeptUnit<T, CODES, ALIGNED> kept;
        load_unit(d, static_cast<const T *>(in.dout) + row * in.dout_stride + unit * kUnit, left, ALIGNED && left >= kUnit);
        kept.load(in, row, unit, left);
        const Unit g = d.values(), n = kept.values(in.rstd[row]);
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
    wait_for_earlier();
    let_next_start();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, col = static_cast<int>(blockIdx.x) * 32 + lane;
    float s = 0.f;
    if (col < cols)
#pragma unroll 8
        for (int k = warp; k < count; k += kGainWarps) s += parts[static_cast<long long>(k) * cols + col];
    sums[warp][lane] = s;
    __syncthreads();
    if (warp || col >= cols) return;
    for (int k = 1; k < kGainWarps; ++k) s += sums[k][lane];
    if (is_bf16) static_cast<__nv_bfloat16 *>(dgain)[col] = __float2bfloat16_rn(s);
    else static_cast<float *>(dgain)[col] = s;
}

}  // namespace softsync
