// Entry points of softsync_learn.h that work on rows of activations: the norm with its backward pass, packing and unpacking.
#include "../../include/softsync_learn.h"
#include "host_util.h"
#include "norm_kernels.cuh"
#include "pack_kernels.cuh"

#include <algorithm>
#include <atomic>
#include <cmath>
#include <type_traits>

using softsync::aligned_to;
using softsync::NormGradIn;
using softsync::NormIn;
using softsync::PackShape;
using bf16 = __nv_bfloat16;

namespace {

constexpr int64_t kMaxRows = 0x7fffffff, kMaxCols = int64_t{1} << 28;

int64_t div_up(int64_t x, int64_t by) { return (x + by - 1) / by; }
bool is_dtype(int t) { return t == PS_GRAD_FP32 || t == PS_GRAD_BF16; }
int64_t size_of(int dtype) { return dtype == PS_GRAD_BF16 ? 2 : 4; }

// Rows `stride` elements apart, at a place that the type allows.
bool rows_ok(const void *p, int dtype, int64_t rows, int64_t cols, int64_t stride)
{
    return p && aligned_to(p, size_of(dtype)) && (rows <= 1 || (stride >= cols && stride <= (int64_t{1} << 60) / rows));
}
bool vectors_ok(const void *p, int dtype, int64_t rows, int64_t stride) { return aligned_to(p, 16) && (rows <= 1 || stride * size_of(dtype) % 16 == 0); }
bool shape_ok(int64_t rows, int64_t cols) { return rows >= 0 && rows <= kMaxRows && cols >= 1 && cols <= kMaxCols; }
bool packed_ok(const int8_t *codes, const uint8_t *scales) { return codes && scales && aligned_to(codes, 16); }

// A launch for every so many rows as have fewer than 2^32 units (nearly always one).
template <typename F>
int over_rows(int64_t rows, int64_t cols, int64_t stride, bool aligned, F launch)
{
    PackShape shape;
    shape.units = static_cast<int>(div_up(cols, PS_PACK_BLOCK) * (PS_PACK_BLOCK / softsync::kUnit));
    shape.cols = static_cast<int>(cols);
    shape.magic = ~uint64_t{0} / static_cast<uint64_t>(shape.units) + 1;
    shape.stride = stride;
    shape.aligned = aligned;
    const int64_t block = softsync::kPackThreads * softsync::kPackTurns, most = ((int64_t{1} << 32) - block) / shape.units;
    for (int64_t first = 0; first < rows; first += most) {
        const int64_t count = std::min(most, rows - first) * shape.units;
        shape.count = static_cast<unsigned>(count);
        if (!launch(first, first * shape.units, shape, div_up(count, block))) return PS_ERR_CUDA;
    }
    return PS_OK;
}

// Warps of a row and units (of eight elements) a thread.  As many units as a thread can hold where rows are many: a row costs each of its warps some hundred instructions.  More warps where
// rows are few and the row's latency counts.  us, bf16, residual, both outputs; 32 rows in the L2 (in a graph; from HBM 0.2 to 0.4 more, in the same order) | 64 M elements:
//     width 1024: 1 x 4 3.7 | 95.3, 4 x 1 2.0 | 101.7 (2368 rows: 5.5, 4.7)       2048: 4 x 2 2.5 | 92.4, 8 x 1 2.1 | 106.2 (296 rows: 2.8, 2.4; 592: 3.2, 3.4)
//     width 4096: 4 x 4 3.8 | 93.3, 8 x 2 2.7 | 94.3, 16 x 1 2.4 | 114.3 (148 rows: 3.9, 2.8, 2.5; 296: 4.1, 3.2, 3.5; 592: 4.8, 4.6, 5.4; 1184: 6.5, 7.0, 8.2)
//     width 8192: 8 x 4 4.0 | 93.9, 16 x 2 3.2 | 108.2 (148 rows: 4.2, 3.4; 296: 4.9, 4.2; 592: 6.4, 7.4)
// fp32 at 8192: 16 x 2 at every number of rows (296: 6.8 against 10.5; 592: 12.9, 18.2; 8192, twice the bytes: 172, 173).  Rows of more than 16384 are read twice (32768: 197 us; 16384: 96).
constexpr int64_t kSms = 148;
template <typename T, bool ALIGNED>
int launch_norm(const NormIn &in, cudaStream_t st)
{
    const int64_t units = div_up(in.cols, softsync::kUnit);
    const auto go = [&](auto kernel, int warps) {
        const int64_t blocks = warps == 1 ? div_up(in.rows, softsync::kNormRows) : in.rows;
        return softsync::launch(kernel, blocks, warps == 1 ? 32 * softsync::kNormRows : 32 * warps, 0, true, st, in) ? PS_OK : PS_ERR_CUDA;
    };
    if (units <= 32) return go(softsync::rms_norm_kernel<T, 1, 1, ALIGNED>, 1);
    if (units <= 64) return go(softsync::rms_norm_kernel<T, 1, 2, ALIGNED>, 1);
    if (units <= 128) return in.rows <= 16 * kSms ? go(softsync::rms_norm_kernel<T, 4, 1, ALIGNED>, 4) : go(softsync::rms_norm_kernel<T, 1, 4, ALIGNED>, 1);
    if (units <= 256) return in.rows <= 2 * kSms ? go(softsync::rms_norm_kernel<T, 8, 1, ALIGNED>, 8) : go(softsync::rms_norm_kernel<T, 4, 2, ALIGNED>, 4);
    if (units <= 512) {
        if (in.rows <= kSms) return go(softsync::rms_norm_kernel<T, 16, 1, ALIGNED>, 16);
        return in.rows <= 4 * kSms ? go(softsync::rms_norm_kernel<T, 8, 2, ALIGNED>, 8) : go(softsync::rms_norm_kernel<T, 4, 4, ALIGNED>, 4);
    }
    if (units <= 1024) return in.rows <= kSms || sizeof(T) == 4 ? go(softsync::rms_norm_kernel<T, 16, 2, ALIGNED>, 16) : go(softsync::rms_norm_kernel<T, 8, 4, ALIGNED>, 8);
    if (units <= 2048) return go(softsync::rms_norm_kernel<T, 16, 4, ALIGNED>, 16);
    return softsync::launch(softsync::rms_norm_long_kernel<T, ALIGNED>, in.rows, softsync::kLongThreads, 0, true, st, in) ? PS_OK : PS_ERR_CUDA;
}

// Blocks of the backward pass, as many as are resident at once, and with them the parts that the gain's gradient is summed in.  Two units a thread where a row has enough, with
// its bytes through the ring where they are whole vectors (us, 64 M elements bf16, ring / loads to registers): width 1024 4 x 1 79.0 / 95.2, 4 x 2 91.6 / 121.0; 2048 4 x 2 77.3 /
// 95.1, 8 x 1 78.5 / 93.4; 4096 8 x 2 77.2 / 96.3, 16 x 1 79.5 / 94.9; 8192 16 x 2 77.8 / 97.2, long 207.  Narrow rows have a warp each: 512 1 x 2 99.0, 4 x 1 113.7 / 124.7.
constexpr int64_t kLongParts = 64;
struct GradShape { int warps, units; int64_t blocks, parts; };
template <typename T>
GradShape grad_shape(int64_t rows, int64_t cols)
{
    const int64_t units = div_up(cols, softsync::kUnit);
    const auto of = [&](int warps, auto per) {
        const int64_t groups = warps == 1 ? softsync::kNormRows : 1, resident = softsync::kGradWarps<T, per> / (warps == 1 ? softsync::kNormRows : warps);
        const int64_t blocks = std::min(div_up(rows, groups), kSms * resident);
        return GradShape{warps, per, blocks, blocks * groups};
    };
    const std::integral_constant<int, 1> one;
    const std::integral_constant<int, 2> two;
    if (units <= 32) return of(1, one);
    if (units <= 64) return of(1, two);
    if (units <= 128) return of(4, one);
    if (units <= 256) return of(4, two);
    if (units <= 512) return of(8, two);
    if (units <= 1024) return of(16, two);
    return GradShape{0, 0, rows, std::min(rows, kLongParts)};
}
GradShape grad_shape(int dtype, int64_t rows, int64_t cols) { return dtype == PS_GRAD_BF16 ? grad_shape<bf16>(rows, cols) : grad_shape<float>(rows, cols); }

constexpr int kNoRoom = 1;
// The kernel with a ring, where the blocks of an SM have room for at least three rows each; else kNoRoom.
template <typename T, int WARPS, int UNITS>
int launch_ring(const NormGradIn &in, const GradShape &shape, cudaStream_t st)
{
    const auto kernel = softsync::rms_norm_grad_ring_kernel<T, WARPS, UNITS>;
    constexpr int resident = softsync::kGradWarps<T, UNITS> / WARPS, room = (224 * 1024) / resident - 1536;          // an SM's shared memory, less what a block takes beside its ring
    softsync::GradRing ring;
    ring.row_bytes = in.cols * static_cast<int>(sizeof(T));
    ring.code_bytes = static_cast<int>(div_up(in.cols, PS_PACK_BLOCK) * PS_PACK_BLOCK);
    ring.slot_bytes = ring.row_bytes * (in.dtotal ? 2 : 1) + ring.code_bytes;
    ring.slots = std::min(room / ring.slot_bytes, softsync::kMostSlots);
    if (ring.slots < 3) return kNoRoom;
    static std::atomic<bool> ready[64] = {};
    int device = 0;
    if (cudaGetDevice(&device) != cudaSuccess || device < 0 || device >= 64) return PS_ERR_CUDA;
    if (!ready[device].load(std::memory_order_relaxed)) {
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, room) != cudaSuccess) return PS_ERR_CUDA;
        ready[device].store(true, std::memory_order_relaxed);
    }
    return softsync::launch(kernel, shape.blocks, 32 * WARPS, ring.slots * ring.slot_bytes, true, st, in, ring) ? PS_OK : PS_ERR_CUDA;
}

template <typename T, bool CODES, bool ALIGNED>
int launch_norm_grad(const NormGradIn &in, const GradShape &shape, cudaStream_t st)
{
    if (CODES && ALIGNED && in.cols % softsync::kUnit == 0) {
        int status = kNoRoom;
        switch (shape.warps * 8 + shape.units) {
        case 4 * 8 + 1: status = launch_ring<T, 4, 1>(in, shape, st); break;
        case 4 * 8 + 2: status = launch_ring<T, 4, 2>(in, shape, st); break;
        case 8 * 8 + 2: status = launch_ring<T, 8, 2>(in, shape, st); break;
        case 16 * 8 + 2: status = launch_ring<T, 16, 2>(in, shape, st); break;
        }
        if (status != kNoRoom) return status;
    }
    const auto go = [&](auto kernel) {
        return softsync::launch(kernel, shape.blocks, shape.warps == 1 ? 32 * softsync::kNormRows : 32 * shape.warps, 0, true, st, in) ? PS_OK : PS_ERR_CUDA;
    };
    switch (shape.warps * 8 + shape.units) {
    case 1 * 8 + 1: return go(softsync::rms_norm_grad_kernel<T, 1, 1, CODES, ALIGNED>);
    case 1 * 8 + 2: return go(softsync::rms_norm_grad_kernel<T, 1, 2, CODES, ALIGNED>);
    case 4 * 8 + 1: return go(softsync::rms_norm_grad_kernel<T, 4, 1, CODES, ALIGNED>);
    case 4 * 8 + 2: return go(softsync::rms_norm_grad_kernel<T, 4, 2, CODES, ALIGNED>);
    case 8 * 8 + 2: return go(softsync::rms_norm_grad_kernel<T, 8, 2, CODES, ALIGNED>);
    case 16 * 8 + 2: return go(softsync::rms_norm_grad_kernel<T, 16, 2, CODES, ALIGNED>);
    }
    if (!softsync::launch(softsync::rms_norm_grad_long_kernel<T, CODES, ALIGNED>, in.rows, softsync::kLongThreads, 0, true, st, in)) return PS_ERR_CUDA;
    if (!in.parts) return PS_OK;
    const dim3 grid(static_cast<unsigned>(div_up(div_up(in.cols, softsync::kUnit), 128)), static_cast<unsigned>(shape.parts));
    softsync::gain_grad_long_kernel<T, CODES, ALIGNED><<<grid, 128, 0, st>>>(in);
    return cudaGetLastError() == cudaSuccess ? PS_OK : PS_ERR_CUDA;
}

}  // namespace

extern "C" {

int ps_pack8(const void *x_dev, int dtype, int64_t rows, int64_t cols, int64_t row_stride, int8_t *codes_dev, uint8_t *scales_dev, void *stream)
{
    if (!is_dtype(dtype) || !shape_ok(rows, cols)) return PS_ERR_INVALID_ARG;
    if (rows == 0) return PS_OK;
    if (!rows_ok(x_dev, dtype, rows, cols, row_stride) || !packed_ok(codes_dev, scales_dev)) return PS_ERR_INVALID_ARG;
    const auto go = [&](auto *x) {
        return over_rows(rows, cols, row_stride, vectors_ok(x_dev, dtype, rows, row_stride), [&](int64_t first, int64_t unit, const PackShape &shape, int64_t blocks) {
            return softsync::launch(softsync::pack_kernel<std::remove_cv_t<std::remove_pointer_t<decltype(x)>>>, blocks, softsync::kPackThreads, 0, true, static_cast<cudaStream_t>(stream),
                                    x + first * row_stride, shape, reinterpret_cast<uint2 *>(codes_dev) + unit, scales_dev + unit / 4);
        });
    };
    return dtype == PS_GRAD_BF16 ? go(static_cast<const bf16 *>(x_dev)) : go(static_cast<const float *>(x_dev));
}

int ps_unpack8(const int8_t *codes_dev, const uint8_t *scales_dev, int64_t rows, int64_t cols, void *out_dev, int dtype, int64_t row_stride, void *stream)
{
    if (!is_dtype(dtype) || !shape_ok(rows, cols)) return PS_ERR_INVALID_ARG;
    if (rows == 0) return PS_OK;
    if (!rows_ok(out_dev, dtype, rows, cols, row_stride) || !packed_ok(codes_dev, scales_dev)) return PS_ERR_INVALID_ARG;
    const auto go = [&](auto *out) {
        return over_rows(rows, cols, row_stride, vectors_ok(out_dev, dtype, rows, row_stride), [&](int64_t first, int64_t unit, const PackShape &shape, int64_t blocks) {
            using T = std::remove_pointer_t<decltype(out)>;
            const int64_t warps = shape.count / static_cast<unsigned>(shape.units) * div_up(shape.units, 32);
            return softsync::launch(shape.aligned ? softsync::unpack_kernel<T> : softsync::unpack_rows_kernel<T>, shape.aligned ? blocks : div_up(warps, softsync::kPackThreads / 32), softsync::kPackThreads, 0, true, static_cast<cudaStream_t>(stream),
                                    reinterpret_cast<const uint2 *>(codes_dev) + unit, scales_dev + unit / 4, shape, out + first * row_stride);
        });
    };
    return dtype == PS_GRAD_BF16 ? go(static_cast<bf16 *>(out_dev)) : go(static_cast<float *>(out_dev));
}

int ps_rms_norm(const ps_norm *a, void *stream)
{
    if (!a || !is_dtype(a->dtype) || !shape_ok(a->rows, a->cols) || !(a->eps >= 0.f) || !std::isfinite(a->eps)) return PS_ERR_INVALID_ARG;
    if (a->gain_dev && (!is_dtype(a->gain_dtype) || !aligned_to(a->gain_dev, size_of(a->gain_dtype)))) return PS_ERR_INVALID_ARG;
    if (a->rows == 0) return PS_OK;
    if (!rows_ok(a->x_dev, a->dtype, a->rows, a->cols, a->x_stride) || !a->rstd_dev || !aligned_to(a->rstd_dev, 4)) return PS_ERR_INVALID_ARG;
    if (a->residual_dev && !rows_ok(a->residual_dev, a->dtype, a->rows, a->cols, a->residual_stride)) return PS_ERR_INVALID_ARG;
    if (a->total_dev && !rows_ok(a->total_dev, a->dtype, a->rows, a->cols, a->total_stride)) return PS_ERR_INVALID_ARG;
    if (a->total_dev && a->rows > 1 && ((a->total_dev == a->x_dev && a->total_stride != a->x_stride) ||
                                        (a->total_dev == a->residual_dev && a->total_stride != a->residual_stride)))
        return PS_ERR_INVALID_ARG;
    if (a->out_dev && (!rows_ok(a->out_dev, a->dtype, a->rows, a->cols, a->cols) || a->out_dev == a->total_dev || a->out_dev == a->residual_dev ||
                       (a->out_dev == a->x_dev && a->rows > 1 && a->x_stride != a->cols)))
        return PS_ERR_INVALID_ARG;
    if ((a->codes_dev || a->scales_dev) && !packed_ok(a->codes_dev, a->scales_dev)) return PS_ERR_INVALID_ARG;
    NormIn in;
    in.x = a->x_dev; in.residual = a->residual_dev; in.gain = a->gain_dev;
    in.gain_bf16 = a->gain_dtype == PS_GRAD_BF16;
    in.rows = a->rows; in.x_stride = a->x_stride; in.residual_stride = a->residual_stride; in.total_stride = a->total_stride;
    in.cols = static_cast<int>(a->cols);
    in.eps = a->eps;
    in.total = a->total_dev; in.out = a->out_dev;
    in.codes = reinterpret_cast<uint2 *>(a->codes_dev);
    in.scales = a->scales_dev;
    in.rstd = a->rstd_dev;
    const bool aligned = vectors_ok(a->x_dev, a->dtype, a->rows, a->x_stride) && vectors_ok(a->residual_dev, a->dtype, a->rows, a->residual_dev ? a->residual_stride : 0) &&
                 vectors_ok(a->total_dev, a->dtype, a->rows, a->total_dev ? a->total_stride : 0) && vectors_ok(a->out_dev, a->dtype, a->rows, a->out_dev ? a->cols : 0) &&
                 aligned_to(a->gain_dev, 16);
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    const auto go = [&](auto vectors) { return a->dtype == PS_GRAD_BF16 ? launch_norm<bf16, vectors>(in, st) : launch_norm<float, vectors>(in, st); };
    return aligned ? go(std::true_type{}) : go(std::false_type{});
}

int ps_norm_grad_workspace(int64_t rows, int64_t cols, int64_t *bytes)
{
    if (!bytes || !shape_ok(rows, cols)) return PS_ERR_INVALID_ARG;
    *bytes = std::max(grad_shape<bf16>(rows, cols).parts, grad_shape<float>(rows, cols).parts) * cols * 4;
    return PS_OK;
}

int ps_rms_norm_grad(const ps_norm_grad *a, void *workspace_dev, int64_t workspace_bytes, void *stream)
{
    if (!a || !is_dtype(a->dtype) || !shape_ok(a->rows, a->cols)) return PS_ERR_INVALID_ARG;
    if ((a->gain_dev || a->dgain_dev) && (!is_dtype(a->gain_dtype) || !aligned_to(a->gain_dev, size_of(a->gain_dtype)) || !aligned_to(a->dgain_dev, size_of(a->gain_dtype))))
        return PS_ERR_INVALID_ARG;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (a->rows == 0)
        return a->dgain_dev && cudaMemsetAsync(a->dgain_dev, 0, static_cast<size_t>(a->cols * size_of(a->gain_dtype)), st) != cudaSuccess ? PS_ERR_CUDA : PS_OK;
    if (!rows_ok(a->dout_dev, a->dtype, a->rows, a->cols, a->dout_stride) || !rows_ok(a->dx_dev, a->dtype, a->rows, a->cols, a->cols)) return PS_ERR_INVALID_ARG;
    if (!a->rstd_dev || !aligned_to(a->rstd_dev, 4)) return PS_ERR_INVALID_ARG;
    if (a->dtotal_dev && !rows_ok(a->dtotal_dev, a->dtype, a->rows, a->cols, a->dtotal_stride)) return PS_ERR_INVALID_ARG;
    if (a->codes_dev || a->scales_dev ? !packed_ok(a->codes_dev, a->scales_dev) || a->total_dev : !rows_ok(a->total_dev, a->dtype, a->rows, a->cols, a->total_stride))
        return PS_ERR_INVALID_ARG;
    if (a->rows > 1 && ((a->dx_dev == a->dout_dev && a->dout_stride != a->cols) || (a->dx_dev == a->dtotal_dev && a->dtotal_stride != a->cols))) return PS_ERR_INVALID_ARG;
    const GradShape shape = grad_shape(a->dtype, a->rows, a->cols);
    // rows beyond a block's registers: the gain's gradient reads dout again after dx is there
    if (a->dx_dev == a->total_dev || (!shape.warps && a->dgain_dev && a->dx_dev == a->dout_dev)) return PS_ERR_INVALID_ARG;
    if (a->dgain_dev && (!workspace_dev || !aligned_to(workspace_dev, 16) || workspace_bytes < shape.parts * a->cols * 4)) return PS_ERR_INVALID_ARG;
    NormGradIn in;
    in.dout = a->dout_dev; in.gain = a->gain_dev; in.dtotal = a->dtotal_dev; in.total = a->total_dev;
    in.codes = reinterpret_cast<const uint2 *>(a->codes_dev);
    in.scales = a->scales_dev;
    in.rstd = a->rstd_dev;
    in.dx = a->dx_dev;
    in.parts = a->dgain_dev ? static_cast<float *>(workspace_dev) : nullptr;
    in.gain_bf16 = a->gain_dtype == PS_GRAD_BF16;
    in.rows = a->rows; in.dout_stride = a->dout_stride; in.dtotal_stride = a->dtotal_stride; in.total_stride = a->total_stride;
    in.cols = static_cast<int>(a->cols);
    const bool aligned = vectors_ok(a->dout_dev, a->dtype, a->rows, a->dout_stride) && vectors_ok(a->dx_dev, a->dtype, a->rows, a->cols) &&
                 vectors_ok(a->dtotal_dev, a->dtype, a->rows, a->dtotal_dev ? a->dtotal_stride : 0) && vectors_ok(a->total_dev, a->dtype, a->rows, a->total_dev ? a->total_stride : 0) &&
                 aligned_to(a->gain_dev, 16);
    const auto go = [&](auto codes, auto vectors) {
        return a->dtype == PS_GRAD_BF16 ? launch_norm_grad<bf16, codes, vectors>(in, shape, st) : launch_norm_grad<float, codes, vectors>(in, shape, st);
    };
    const std::true_type yes;
    const std::false_type no;
    const int status = in.codes ? aligned ? go(yes, yes) : go(yes, no) : aligned ? go(no, yes) : go(no, no);
    if (status != PS_OK || !a->dgain_dev) return status;
    return softsync::launch(softsync::gain_grad_kernel, div_up(a->cols, 32), 32 * softsync::kGainWarps, 0, true, st, in.parts, static_cast<int>(shape.parts), in.cols, a->dgain_dev,
                            in.gain_bf16) ? PS_OK : PS_ERR_CUDA;
}

}  // extern "C"
