// Entry points of softsync_learn.h that are matrix products: losses without logits, and the weight gradient from 8-bit activations.
#include "../../include/softsync_learn.h"
#include "head_kernels.cuh"
#include "host_util.h"

#include <algorithm>
#include <atomic>
#include <cmath>

using softsync::aligned_to;
using softsync::kHalf;
using softsync::kStep;
using softsync::kTile;
using softsync::MmaPlan;
using bf16 = __nv_bfloat16;

namespace {

int64_t round_up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }
int64_t div_up(int64_t x, int64_t by) { return (x + by - 1) / by; }
int launched() { return cudaGetLastError() == cudaSuccess ? PS_OK : PS_ERR_CUDA; }

constexpr int64_t kMaxRows = int64_t{1} << 26, kMaxWidth = int64_t{1} << 20, kMaxVocab = int64_t{1} << 28;
constexpr int kPairs = 74;                                 // CTA pairs that the GPU holds: sizes of workspaces go by it, launches by the device
constexpr int64_t kPieceBytes = int64_t{256} << 20;        // of G, or the hidden states' own size where that is more

// ---- a matrix for the loads ---------------------------------------------------------------------------------------------
struct Matrix {
    const bf16 *data;
    int64_t rows, cols, stride;
};

using EncodeTiled = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                                 const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiled encoder()
{
    static std::atomic<EncodeTiled> known{nullptr};
    EncodeTiled f = known.load(std::memory_order_relaxed);
    if (f) return f;
    void *p = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) return nullptr;
    f = reinterpret_cast<EncodeTiled>(p);
    known.store(f, std::memory_order_relaxed);
    return f;
}

// Blocks of 64 columns (128 bytes, swizzled) by box_rows rows; zeros outside the matrix.
bool encode(CUtensorMap &map, const Matrix &m, int box_rows)
{
    const EncodeTiled f = encoder();
    if (!f) return false;
    const cuuint64_t dims[2] = {static_cast<cuuint64_t>(m.cols), static_cast<cuuint64_t>(m.rows)};
    const cuuint64_t strides[1] = {static_cast<cuuint64_t>(m.stride * 2)};
    const cuuint32_t box[2] = {static_cast<cuuint32_t>(kStep), static_cast<cuuint32_t>(box_rows)}, ones[2] = {1, 1};
    return f(&map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<bf16 *>(m.data), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
             CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

int pairs_on_device()
{
    static std::atomic<int> cached[64] = {};
    int device = 0;
    if (cudaGetDevice(&device) != cudaSuccess || device < 0 || device >= 64) return 0;
    int n = cached[device].load(std::memory_order_relaxed);
    if (!n && cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, device) == cudaSuccess) {
        n /= 2;
        cached[device].store(n, std::memory_order_relaxed);
    }
    return n;
}

// D = A B^T.  MN_A: A is given as k x m (else m x k), MN_B: B as k x n (else n x k).
template <bool MN_A, bool MN_B, typename Epilogue>
int launch_product(const Matrix &a, const Matrix &b, const MmaPlan &plan, const Epilogue &epilogue, cudaStream_t st)
{
    CUtensorMap map_a, map_b;
    if (!encode(map_a, a, MN_A ? kStep : kHalf) || !encode(map_b, b, MN_B ? kStep : kHalf)) return PS_ERR_CUDA;
    const auto kernel = softsync::mma_kernel<Epilogue, MN_A, MN_B>;
    static std::atomic<bool> ready[64] = {};
    int device = 0;
    if (cudaGetDevice(&device) != cudaSuccess || device < 0 || device >= 64) return PS_ERR_CUDA;
    if (!ready[device].load(std::memory_order_relaxed)) {
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, softsync::kMmaShared) != cudaSuccess) return PS_ERR_CUDA;
        ready[device].store(true, std::memory_order_relaxed);
    }
    const int64_t tiles = div_up(plan.m, kTile) * div_up(plan.n, kTile) * plan.splits;
    const int64_t pairs = std::min<int64_t>(tiles, pairs_on_device());
    if (pairs < 1) return PS_ERR_CUDA;
    kernel<<<static_cast<unsigned>(2 * pairs), softsync::kMmaThreads, softsync::kMmaShared, st>>>(map_a, map_b, plan, epilogue);
    return launched();
}

// Parts of the contraction, so that few tiles still fill the GPU: the number, at most 16 and a stage for each at least, with the least
// of rounds x stages.
int splits_of(int64_t tiles, int64_t steps)
{
    int best = 1;
    int64_t cost = div_up(tiles, kPairs) * steps;
    for (int s = 2; s <= 16 && s * 4 <= steps; ++s) {
        const int64_t c = div_up(tiles * s, kPairs) * div_up(steps, s) + s;             // and the sums of each have to be read again
        if (c < cost) { cost = c; best = s; }
    }
    return best;
}
int group_of(int64_t tiles_m) { return static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(tiles_m, 16))); }

// ---- workspaces --------------------------------------------------------------------------------------------------------
struct Places {
    int64_t bytes = 0;
    char *base;
    explicit Places(void *p) : base(static_cast<char *>(p)) {}
    template <typename T> void take(T *&out, int64_t count)
    {
        out = reinterpret_cast<T *>(base + bytes);
        bytes += round_up(count * static_cast<int64_t>(sizeof(T)), 256);
    }
};

bool matrix_aligned(const void *p, int64_t rows, int64_t stride) { return aligned_to(p, 16) && (rows <= 1 || stride % 8 == 0); }

struct HeadPlan : Places {
    int64_t rows, width, vocab, rows_padded, width_padded, pieces, piece, tiles_n, parts;
    bool copy_head, copy_hidden;
    int splits;                            // of dhidden's product
    // statistics
    float2 *stat = nullptr;
    float *picked = nullptr, *inverse = nullptr, *sum = nullptr;
    double *sums = nullptr;
    int *order = nullptr, *place = nullptr, *live = nullptr;
    bf16 *hidden = nullptr, *head = nullptr;
    // gradients
    bf16 *g = nullptr;
    float *part = nullptr;
    HeadPlan(const ps_head &h, bool grad, bool listed, void *p) : Places(p), rows(h.rows), width(h.width), vocab(h.vocab)
    {
        rows_padded = round_up(rows, kStep);
        width_padded = round_up(width, 8);
        copy_head = !matrix_aligned(h.head_dev, vocab, h.head_stride);
        copy_hidden = listed || !matrix_aligned(h.hidden_dev, rows, h.hidden_stride);
        tiles_n = div_up(vocab, kTile);
        parts = div_up(vocab, kHalf);
        const int64_t budget = std::max(kPieceBytes, rows * width * 2);
        const int64_t most = std::max<int64_t>(kTile, budget / (2 * rows_padded) / kTile * kTile);
        pieces = div_up(vocab, most);
        piece = std::min(most, round_up(div_up(vocab, pieces), kTile));
        pieces = div_up(vocab, piece);
        splits = splits_of(div_up(rows, kTile) * div_up(width, kTile), div_up(std::min(piece, vocab), kStep));
        take(inverse, 1);
        take(sum, 1);
        take(live, 1);
        take(order, rows);
        take(place, rows);
        take(picked, rows);
        take(sums, div_up(rows, 32));
        if (copy_hidden) take(hidden, rows_padded * width_padded);
        if (copy_head) take(head, round_up(vocab, kStep) * width_padded);
        const int64_t shared = bytes;                       // the statistics are done with before a piece of G is written
        take(stat, parts * rows);
        if (!grad) return;
        const int64_t after_stat = bytes;
        bytes = shared;
        take(g, rows_padded * piece);
        take(part, splits * rows * width_padded);
        bytes = std::max(bytes, after_stat);
    }
};

int check_head(const ps_head *h)
{
    if (!h || h->rows < 0 || h->rows > kMaxRows || h->width < 1 || h->width > kMaxWidth || h->vocab < 1 || h->vocab > kMaxVocab) return PS_ERR_INVALID_ARG;
    if (!(h->temperature > 0.f) || !std::isfinite(h->temperature) || !std::isfinite(1.f / h->temperature)) return PS_ERR_INVALID_ARG;
    if (h->rows == 0) return PS_OK;
    if (!h->hidden_dev || !h->head_dev || !h->tokens_dev || !aligned_to(h->hidden_dev, 2) || !aligned_to(h->head_dev, 2) || !aligned_to(h->tokens_dev, 8)) return PS_ERR_INVALID_ARG;
    const int64_t most = int64_t{1} << 38;                  // elements of a stride: the loads take 2^40 bytes
    if (h->rows > 1 && (h->hidden_stride < h->width || h->hidden_stride > most)) return PS_ERR_INVALID_ARG;
    if (h->vocab > 1 && (h->head_stride < h->width || h->head_stride > most)) return PS_ERR_INVALID_ARG;
    return PS_OK;
}

// One call: the rows that take part, their statistics, the gradients.
struct HeadCall {
    const ps_head &h;
    HeadPlan w;
    cudaStream_t st;
    bool listed;
    Matrix hidden, head;
    const long long *tokens;
    float scale, inv_temperature;

    HeadCall(const ps_head &head_, bool grad, bool listed_, void *workspace, cudaStream_t stream)
        : h(head_), w(head_, grad, listed_, workspace), st(stream), listed(listed_), tokens(reinterpret_cast<const long long *>(head_.tokens_dev)),
          scale(static_cast<float>(1.4426950408889634 / static_cast<double>(head_.temperature))), inv_temperature(1.f / head_.temperature)
    {
        const auto given = [](const void *p, int64_t rows, int64_t cols, int64_t stride) { return Matrix{static_cast<const bf16 *>(p), rows, cols, rows > 1 ? stride : round_up(cols, 8)}; };
        hidden = w.copy_hidden ? Matrix{w.hidden, w.rows_padded, w.width, w.width_padded} : given(h.hidden_dev, h.rows, h.width, h.hidden_stride);
        head = w.copy_head ? Matrix{w.head, h.vocab, h.width, w.width_padded} : given(h.head_dev, h.vocab, h.width, h.head_stride);
    }
    const int *order() const { return listed ? w.order : nullptr; }
    const int *live() const { return listed ? w.live : nullptr; }

    int begin(const float *factors, float *zero_a, float *zero_b)
    {
        int status = PS_OK;
        if (listed) {
            softsync::order_kernel<<<1, softsync::kOrderThreads, 0, st>>>(factors, static_cast<int>(h.rows), {w.order, w.place, w.live, w.inverse, w.sum, zero_a, zero_b});
            status = launched();
        }
        const auto copy = [&](const void *from, int64_t rows, int64_t padded, int64_t stride, const int *ord, const int *n, bf16 *to) {
            softsync::gather_kernel<<<static_cast<unsigned>(padded), 128, 0, st>>>(static_cast<const bf16 *>(from), static_cast<int>(rows), static_cast<int>(h.width), stride, ord, n,
                                                                                  matrix_aligned(from, rows, stride), to, static_cast<int>(w.width_padded));
            return launched();
        };
        if (status == PS_OK && w.copy_hidden) status = copy(h.hidden_dev, h.rows, w.rows_padded, h.hidden_stride, order(), live(), w.hidden);
        if (status == PS_OK && w.copy_head) status = copy(h.head_dev, h.vocab, round_up(h.vocab, kStep), h.head_stride, nullptr, nullptr, w.head);
        return status;
    }
    int statistics(const float *weights, float *logp, float *lse, bool sums)
    {
        softsync::StatsEpilogue ep{};
        ep.order = order(); ep.tokens = tokens; ep.rows = static_cast<int>(h.rows); ep.vocab = static_cast<int>(h.vocab); ep.live = live(); ep.scale = scale;
        ep.parts = w.stat; ep.part_stride = h.rows; ep.picked = w.picked;
        MmaPlan plan{static_cast<int>(h.rows), static_cast<int>(h.vocab), static_cast<int>(h.width), live(), 0, 1, group_of(div_up(h.rows, kTile))};
        const int status = launch_product<false, false>(hidden, head, plan, ep, st);
        if (status != PS_OK) return status;
        softsync::JoinIn in{w.stat, h.rows, static_cast<int>(w.parts), w.picked, tokens, order(), live(), weights, ep.rows, ep.vocab, scale, inv_temperature, logp, lse,
                            sums ? w.sums : nullptr};
        softsync::join_kernel<<<static_cast<unsigned>(div_up(h.rows, 32)), 32 * softsync::kJoinWarps, 0, st>>>(in);
        return launched();
    }
    // coef: of every row, or null for 1; alpha times *alpha_dev: of both gradients
    int gradients(const float *lse, const float *coef, float sign, float alpha, const float *alpha_dev, void *dhidden, void *dhead)
    {
        int status = PS_OK;
        const int rows = static_cast<int>(h.rows), width = static_cast<int>(h.width);
        for (int64_t first = 0; first < h.vocab && status == PS_OK; first += w.piece) {
            const int n = static_cast<int>(std::min(w.piece, h.vocab - first));
            const Matrix entries{head.data + first * head.stride, n, h.width, head.stride};
            softsync::GradEpilogue ge{};
            ge.order = order(); ge.tokens = tokens; ge.lse = lse; ge.coef = coef; ge.sign = sign; ge.rows = rows; ge.vocab = static_cast<int>(h.vocab); ge.live = live(); ge.scale = scale;
            ge.first = static_cast<int>(first); ge.width = n; ge.g = w.g; ge.g_stride = w.piece;
            MmaPlan plan{rows, n, width, live(), 0, 1, group_of(div_up(rows, kTile))};
            if ((status = launch_product<false, false>(hidden, entries, plan, ge, st)) != PS_OK) break;
            const Matrix g{w.g, w.rows_padded, n, w.piece};
            if (dhidden) {
                softsync::StoreEpilogue se{};
                se.rows = rows; se.cols = width;
                se.part = w.part; se.part_stride = w.width_padded; se.part_rows = h.rows * w.width_padded; se.add = first > 0;
                MmaPlan p{rows, width, n, live(), 0, w.splits, group_of(div_up(rows, kTile))};
                if ((status = launch_product<false, true>(g, entries, p, se, st)) != PS_OK) break;
            }
            if (dhead) {
                softsync::StoreEpilogue se{};
                se.rows = n; se.cols = width; se.alpha = alpha; se.alpha_dev = alpha_dev;
                se.out = static_cast<bf16 *>(dhead) + first * h.width; se.out_bf16 = 1; se.vectors = h.width % 8 == 0; se.stride = h.width;
                MmaPlan p{n, width, rows, live(), 1, 1, group_of(div_up(n, kTile))};
                status = launch_product<true, true>(g, hidden, p, se, st);
            }
        }
        if (status != PS_OK || !dhidden) return status;
        softsync::SplitSum in{w.part, w.width_padded, h.rows * w.width_padded, w.splits, listed ? w.place : nullptr, rows, width, alpha, alpha_dev, nullptr, 0, dhidden, 1,
                              h.width % 8 == 0, h.width};
        softsync::split_sum_kernel<<<static_cast<unsigned>(rows), 128, 0, st>>>(in);
        return launched();
    }
};

int no_rows(const ps_head *h, float *stats, void *dhead, cudaStream_t st)
{
    if (stats && cudaMemsetAsync(stats, 0, 2 * sizeof(float), st) != cudaSuccess) return PS_ERR_CUDA;
    if (dhead && cudaMemsetAsync(dhead, 0, static_cast<size_t>(h->vocab * h->width * 2), st) != cudaSuccess) return PS_ERR_CUDA;
    return PS_OK;
}

}  // namespace

extern "C" {

int ps_head_workspace(const ps_head *head, int grad, int64_t *bytes)
{
    const int bad = check_head(head);
    if (bad != PS_OK || !bytes) return PS_ERR_INVALID_ARG;
    *bytes = head->rows ? HeadPlan(*head, grad != 0, true, nullptr).bytes : 0;
    return PS_OK;
}

int ps_head_logprob(const ps_head *head, const float *weights_dev, float *logp_dev, float *lse_dev, void *workspace_dev, int64_t workspace_bytes, void *stream)
{
    const int bad = check_head(head);
    if (bad != PS_OK) return bad;
    if (head->rows == 0) return PS_OK;
    if (!logp_dev || !lse_dev || !aligned_to(logp_dev, 4) || !aligned_to(lse_dev, 4) || !aligned_to(weights_dev, 4)) return PS_ERR_INVALID_ARG;
    HeadCall call(*head, false, weights_dev != nullptr, workspace_dev, static_cast<cudaStream_t>(stream));
    if (!workspace_dev || !aligned_to(workspace_dev, 256) || workspace_bytes < call.w.bytes) return PS_ERR_INVALID_ARG;
    const int status = call.begin(weights_dev, logp_dev, lse_dev);
    return status == PS_OK ? call.statistics(nullptr, logp_dev, lse_dev, false) : status;
}

int ps_head_logprob_grad(const ps_head *head, const float *lse_dev, const float *dlogp_dev, void *dhidden_dev, void *dhead_dev, void *workspace_dev,
                         int64_t workspace_bytes, void *stream)
{
    const int bad = check_head(head);
    if (bad != PS_OK) return bad;
    if (!aligned_to(dhidden_dev, 16) || !aligned_to(dhead_dev, 16)) return PS_ERR_INVALID_ARG;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (head->rows == 0) return no_rows(head, nullptr, dhead_dev, st);
    if (!lse_dev || !dlogp_dev || !aligned_to(lse_dev, 4) || !aligned_to(dlogp_dev, 4)) return PS_ERR_INVALID_ARG;
    if (!dhidden_dev && !dhead_dev) return PS_OK;
    HeadCall call(*head, true, true, workspace_dev, st);
    if (!workspace_dev || !aligned_to(workspace_dev, 256) || workspace_bytes < call.w.bytes) return PS_ERR_INVALID_ARG;
    const int status = call.begin(dlogp_dev, nullptr, nullptr);
    return status == PS_OK ? call.gradients(lse_dev, dlogp_dev, -1.f, call.inv_temperature, nullptr, dhidden_dev, dhead_dev) : status;
}

int ps_head_cross_entropy(const ps_head *head, const float *weights_dev, float *stats_dev, float *logp_dev, float *lse_dev, void *dhidden_dev, void *dhead_dev,
                          void *workspace_dev, int64_t workspace_bytes, void *stream)
{
    const int bad = check_head(head);
    if (bad != PS_OK) return bad;
    if (!stats_dev || !aligned_to(stats_dev, 4) || !aligned_to(dhidden_dev, 16) || !aligned_to(dhead_dev, 16)) return PS_ERR_INVALID_ARG;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (head->rows == 0) return no_rows(head, stats_dev, dhead_dev, st);
    if (!logp_dev || !lse_dev || !aligned_to(logp_dev, 4) || !aligned_to(lse_dev, 4) || !aligned_to(weights_dev, 4)) return PS_ERR_INVALID_ARG;
    const bool grad = dhidden_dev || dhead_dev, listed = weights_dev != nullptr;
    HeadCall call(*head, grad, listed, workspace_dev, st);
    if (!workspace_dev || !aligned_to(workspace_dev, 256) || workspace_bytes < call.w.bytes) return PS_ERR_INVALID_ARG;
    int status = call.begin(weights_dev, logp_dev, lse_dev);
    if (status == PS_OK) status = call.statistics(weights_dev, logp_dev, lse_dev, true);
    if (status != PS_OK) return status;
    const int rows = static_cast<int>(head->rows);
    softsync::loss_kernel<<<1, 256, 0, st>>>(call.w.sums, static_cast<int>(div_up(rows, 32)), listed ? call.w.sum : nullptr, rows, stats_dev);
    if ((status = launched()) != PS_OK || !grad) return status;
    return call.gradients(lse_dev, weights_dev, 1.f, listed ? call.inv_temperature : call.inv_temperature / static_cast<float>(rows), listed ? call.w.inverse : nullptr, dhidden_dev, dhead_dev);
}

}  // extern "C"

// ---- weight gradient from packed activations -----------------------------------------------------------------------------
namespace {

struct PackedPlan : Places {
    int64_t outs_padded, cols_padded;
    bool copy_dout;
    int splits;
    bf16 *dout = nullptr, *values = nullptr;
    float *part = nullptr;
    PackedPlan(const ps_packed_grad &a, void *p) : Places(p), outs_padded(round_up(a.outs, 8)), cols_padded(round_up(a.cols, 8))
    {
        copy_dout = !matrix_aligned(a.dout_dev, a.rows, a.dout_stride);
        splits = splits_of(div_up(a.outs, kTile) * div_up(a.cols, kTile), div_up(a.rows, kStep));
        if (copy_dout) take(dout, round_up(a.rows, kStep) * outs_padded);
        take(values, a.rows * cols_padded);
        if (splits > 1) take(part, splits * a.outs * cols_padded);
    }
};

int check_packed(const ps_packed_grad *a)
{
    const auto is_dtype = [](int t) { return t == PS_GRAD_FP32 || t == PS_GRAD_BF16; };
    if (!a || a->rows < 0 || a->rows > kMaxRows || a->outs < 1 || a->outs > kMaxVocab || a->cols < 1 || a->cols > kMaxWidth || !is_dtype(a->out_dtype)) return PS_ERR_INVALID_ARG;
    if (a->gain_dev && (!is_dtype(a->gain_dtype) || !aligned_to(a->gain_dev, a->gain_dtype == PS_GRAD_BF16 ? 2 : 4))) return PS_ERR_INVALID_ARG;
    if (a->rows > 1 && (a->dout_stride < a->outs || a->dout_stride > (int64_t{1} << 38))) return PS_ERR_INVALID_ARG;
    return PS_OK;
}

}  // namespace

extern "C" {

int ps_packed_grad_workspace(const ps_packed_grad *grad, int64_t *bytes)
{
    if (check_packed(grad) != PS_OK || !bytes) return PS_ERR_INVALID_ARG;
    *bytes = grad->rows ? PackedPlan(*grad, nullptr).bytes : 0;
    return PS_OK;
}

int ps_packed_weight_grad(const ps_packed_grad *a, void *workspace_dev, int64_t workspace_bytes, void *stream)
{
    const int bad = check_packed(a);
    if (bad != PS_OK) return bad;
    if (!a->dweight_dev || !aligned_to(a->dweight_dev, 16)) return PS_ERR_INVALID_ARG;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    const int64_t size = a->out_dtype == PS_GRAD_BF16 ? 2 : 4;
    if (a->rows == 0) return cudaMemsetAsync(a->dweight_dev, 0, static_cast<size_t>(a->outs * a->cols * size), st) == cudaSuccess ? PS_OK : PS_ERR_CUDA;
    if (!a->dout_dev || !aligned_to(a->dout_dev, 2) || !a->codes_dev || !a->scales_dev || !aligned_to(a->codes_dev, 16)) return PS_ERR_INVALID_ARG;
    const PackedPlan w(*a, workspace_dev);
    if (!workspace_dev || !aligned_to(workspace_dev, 256) || workspace_bytes < w.bytes) return PS_ERR_INVALID_ARG;
    const int rows = static_cast<int>(a->rows), outs = static_cast<int>(a->outs), cols = static_cast<int>(a->cols);
    Matrix dout{static_cast<const bf16 *>(a->dout_dev), rows, outs, rows > 1 ? a->dout_stride : w.outs_padded};
    int status = PS_OK;
    if (w.copy_dout) {
        softsync::gather_kernel<<<static_cast<unsigned>(round_up(rows, kStep)), 128, 0, st>>>(dout.data, rows, outs, a->dout_stride, nullptr, nullptr, 0, w.dout, static_cast<int>(w.outs_padded));
        status = launched();
        dout = Matrix{w.dout, rows, outs, w.outs_padded};
    }
    if (status == PS_OK) status = ps_unpack8(a->codes_dev, a->scales_dev, rows, cols, w.values, PS_GRAD_BF16, w.cols_padded, stream);
    if (status != PS_OK) return status;
    const Matrix values{w.values, rows, cols, w.cols_padded};
    const int vectors = a->cols % 8 == 0 && aligned_to(a->gain_dev, 16), gain_bf16 = a->gain_dtype == PS_GRAD_BF16, out_bf16 = a->out_dtype == PS_GRAD_BF16;
    softsync::StoreEpilogue se{};
    se.rows = outs; se.cols = cols; se.alpha = 1.f;
    if (w.splits > 1) {
        se.part = w.part; se.part_stride = w.cols_padded; se.part_rows = a->outs * w.cols_padded;
    } else {
        se.gain = a->gain_dev; se.gain_bf16 = gain_bf16; se.out = a->dweight_dev; se.out_bf16 = out_bf16; se.vectors = vectors; se.stride = cols;
    }
    const MmaPlan plan{outs, cols, rows, nullptr, 0, w.splits, group_of(div_up(outs, kTile))};
    if ((status = launch_product<true, true>(dout, values, plan, se, st)) != PS_OK || w.splits == 1) return status;
    softsync::SplitSum in{w.part, w.cols_padded, a->outs * w.cols_padded, w.splits, nullptr, outs, cols, 1.f, nullptr, a->gain_dev, gain_bf16, a->dweight_dev, out_bf16, vectors, cols};
    softsync::split_sum_kernel<<<static_cast<unsigned>(outs), 128, 0, st>>>(in);
    return launched();
}

}  // extern "C"
