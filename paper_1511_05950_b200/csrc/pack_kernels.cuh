// Activations into 8 bits and back.  One unit a thread and turn, kPackTurns of them under way.  Bound by HBM: 8192 x 8192 bf16, 203 MB each way, 32 and 31 us (6.4 TB/s).
#pragma once

#include "units.cuh"

namespace softsync {

constexpr int kPackThreads = 256, kPackTurns = 4;

// Rows of `units` units (whole blocks of 32 columns), numbered through: fewer than 2^32.  magic: 2^64 / units, rounded up, so that the upper half of the product is the row
// exactly (a division would be a third of the instructions).
struct PackShape {
    unsigned count;
    int units, cols;
    unsigned long long magic;
    long long stride;                      // of the activations
    int aligned;                           // every row allows vectors
    __device__ __forceinline__ void find(unsigned at, unsigned &row, int &col) const
    {
        row = static_cast<unsigned>(__umul64hi(at, magic));
        col = static_cast<int>(at - row * static_cast<unsigned>(units)) * kUnit;
    }
};

template <typename T>
__global__ void __launch_bounds__(kPackThreads) pack_kernel(const T *x, const __grid_constant__ PackShape shape, uint2 *codes, uint8_t *scales)
{
    wait_for_earlier();
    let_next_start();
    const unsigned base = blockIdx.x * (kPackThreads * kPackTurns) + threadIdx.x;
    RawUnit<T> raw[kPackTurns];
#pragma unroll
    for (int j = 0; j < kPackTurns; ++j) {
        const unsigned at = base + j * kPackThreads;
        unsigned row;
        int col;
        shape.find(at, row, col);
        const int left = at < shape.count ? shape.cols - col : 0;
        load_unit(raw[j], x + (left > 0 ? row * shape.stride + col : 0), left, shape.aligned && left >= kUnit);
    }
#pragma unroll
    for (int j = 0; j < kPackTurns; ++j) {
        const unsigned at = base + j * kPackThreads;
        unsigned scale;
        const uint2 c = pack_unit(raw[j].values(), scale);
        if (at < shape.count) {
            codes[at] = c;
            if ((at & 3) == 0) scales[at >> 2] = static_cast<uint8_t>(scale);
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(kPackThreads) unpack_kernel(const uint2 *codes, const uint8_t *scales, const __grid_constant__ PackShape shape, T *out)
{
    wait_for_earlier();
    let_next_start();
    const unsigned base = blockIdx.x * (kPackThreads * kPackTurns) + threadIdx.x;
    uint2 c[kPackTurns];
    unsigned s[kPackTurns];
#pragma unroll
    for (int j = 0; j < kPackTurns; ++j) {
        const unsigned at = base + j * kPackThreads;
        if (at < shape.count) { c[j] = __ldcs(codes + at); s[j] = __ldcs(scales + (at >> 2)); }
    }
#pragma unroll
    for (int j = 0; j < kPackTurns; ++j) {
        const unsigned at = base + j * kPackThreads;
        if (at >= shape.count) break;
        unsigned row;
        int col;
        shape.find(at, row, col);
        const int left = shape.cols - col;
        if (left > 0) store_unit(out + row * shape.stride + col, unpack_unit(c[j], s[j]), left, left >= kUnit);
    }
}

// The same for rows that allow no vectors: a warp takes 32 units of one row.
template <typename T>
__global__ void __launch_bounds__(kPackThreads) unpack_rows_kernel(const uint2 *codes, const uint8_t *scales, const __grid_constant__ PackShape shape, T *out)
{
    __shared__ WarpDesk<T> desk[kPackThreads / 32];
    wait_for_earlier();
    let_next_start();
    const unsigned warps = static_cast<unsigned>(shape.units + 31) / 32, item = blockIdx.x * (kPackThreads / 32) + (threadIdx.x >> 5), row = item / warps;
    if (row >= shape.count / static_cast<unsigned>(shape.units)) return;            // a whole warp
    const int unit = static_cast<int>(item - row * warps) * 32 + static_cast<int>(threadIdx.x & 31);
    Unit u{};
    if (unit < shape.units) {
        const unsigned at = row * static_cast<unsigned>(shape.units) + unit;
        u = unpack_unit(__ldcs(codes + at), __ldcs(scales + (at >> 2)));
    }
    store_row<false>(out + row * shape.stride, unit, shape.cols, u, desk);
}

}  // namespace softsync
