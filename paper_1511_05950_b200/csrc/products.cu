// Entry points of softsync_learn.h that are matrix products: losses without logits, and the weight gradient from 8-bit activations.
#include "../../include/softsync_learn.h"
#include "head_kernels.cuh"
#include "host_util.h"

#include <algorithm>
#include <atomic>
#include <cmath>
#include <type_traits>

using softsync::aligned_to;
using softsync::kHalf;
using softsync::kStep;
using softsync::kTile;
using softsync::MmaPlan;
using bf16 = __nv_bfloat16;

namespace {

int64_t round_up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }
int64_t div_up(int64_t x, int64_t by) { return (x + by - 1) / by; }

constexpr int64_t kMaxRows = int64_t{1} << 26, kMaxWidth = int64_t{1} << 20, kMaxVocab = int64_t{1} << 28;
constexpr double kLog2E = 1.4426950408889634;
constexpr int kPairs = 74;                                 // CTA pairs that the GPU holds: sizes of workspaces go by it, launches by the device
// Of G, or the hidden states' own size where that is more.  7168 x 2048 x 131072 takes 11.9 ms with 128 MiB, 11.2 with 256, 10.8 with 512, 10.3 with 1 GiB (half of the products are
// computed once) and 9.5 with 2 GiB (all are): the memory is what the call is for, so it stops at a size that does not grow with the batch.
constexpr int64_t kPieceBytes = int64_t{1} << 30;

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

int slots_on_device() { return std::min(pairs_on_device(), kPairs); }

template <typename... K, typename... A>
int start(void (*kernel)(K...), int64_t blocks, int threads, int shared, bool dependent, cudaStream_t st, const A &...args)
{
    return softsync::launch(kernel, blocks, threads, shared, dependent, st, args...) ? PS_OK : PS_ERR_CUDA;
}

using softsync::Lying;

// D = A B^T; rounded16: the result is, in the end.  L::mn_a: A is given as k x m (else m x k), L::mn_b: B as k x n (else n x k).
template <typename L, typename Epilogue>
bool job_of(softsync::MmaJob<Epilogue> &job, const Matrix &a, const Matrix &b, const MmaPlan &plan, const Epilogue &epilogue, bool rounded16 = true)
{
    job.plan = plan;
    if constexpr (std::is_same_v<Epilogue, softsync::StoreEpilogue>) job.plan.sum_stages = rounded16 ? softsync::kSumStages16 : softsync::kSumStages;
    if (plan.slots && !plan.live) {
        const int64_t rest = div_up(plan.m, kTile) * div_up(plan.n, kTile) % plan.slots;
        job.plan.splits = rest ? softsync::split_count(static_cast<int>(rest), static_cast<int>(div_up(plan.k, kStep)), plan.slots) : 1;
    }
    job.epilogue = epilogue;
    return encode(job.a, a, L::mn_a ? kStep : kHalf) && encode(job.b, b, L::mn_b ? kStep : kHalf);
}

// A launch counts its tiles, and the parts of split ones, in 31 bits.  Asked of a call's extents before its first kernel: a refusal leaves everything as it was.
constexpr int64_t kMostItems = 0x70000000;
bool too_many_tiles(int64_t m, int64_t n) { return div_up(m, kTile) * div_up(n, kTile) > kMostItems - softsync::kMostParts * kPairs; }

// Items of a product (parts of split tiles one by one): exactly, or at most where only the device knows the extents.
int64_t items_of(const MmaPlan &plan)
{
    const int64_t tiles = div_up(plan.m, kTile) * div_up(plan.n, kTile);
    if (!plan.slots) return tiles;
    if (plan.live) return std::max<int64_t>(tiles, plan.slots);
    const int rest = static_cast<int>(tiles % plan.slots);
    return tiles + int64_t{rest} * (plan.splits - 1);
}

// Stages of the longest tile or part, as far as the host knows.
int64_t longest_of(const MmaPlan &plan)
{
    const int64_t steps = div_up(plan.k, kStep);
    if (!plan.slots || plan.live || plan.splits <= 1) return steps;
    return div_up(plan.m, kTile) * div_up(plan.n, kTile) < plan.slots ? div_up(steps, plan.splits) : steps;
}

// One product, or two whose operands are both there: a launch of its own costs 10 us (48 x 256 x 32000: 63 us with two, 53 with one).
template <typename L, typename M, bool LONG, typename Epilogue>
int launch_products_as(const softsync::MmaJob<Epilogue> *jobs, bool dependent, cudaStream_t st)
{
    constexpr int count = std::is_void_v<M> ? 1 : 2;
    const auto kernel = softsync::mma_kernel<Epilogue, L, M, LONG>;
    static std::atomic<bool> ready[64] = {};
    int device = 0;
    if (cudaGetDevice(&device) != cudaSuccess || device < 0 || device >= 64) return PS_ERR_CUDA;
    if (!ready[device].load(std::memory_order_relaxed)) {
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, softsync::kMmaShared) != cudaSuccess) return PS_ERR_CUDA;
        ready[device].store(true, std::memory_order_relaxed);
    }
    int64_t items = 0;
    for (int k = 0; k < count; ++k) {
        const int64_t n = items_of(jobs[k].plan);
        if (n > kMostItems) return PS_ERR_CUDA;
        items += n;
    }
    const int64_t pairs = std::min<int64_t>(items, pairs_on_device());
    if (pairs < 1) return PS_ERR_CUDA;
    return start(kernel, 2 * pairs, softsync::kMmaThreads, softsync::kMmaShared, dependent, st, jobs[0], jobs[count - 1]);
}
template <typename L, typename M = void, typename Epilogue>
int launch_products(const softsync::MmaJob<Epilogue> *jobs, bool dependent, cudaStream_t st)
{
    bool sums = Epilogue::kAllColumns;
    for (int k = 0; k < (std::is_void_v<M> ? 1 : 2) && !sums; ++k) sums = longest_of(jobs[k].plan) > (Epilogue::kSums ? Epilogue::kSums : jobs[k].plan.sum_stages);
    if constexpr (!Epilogue::kAllColumns) {
        if (!sums) return launch_products_as<L, M, false>(jobs, dependent, st);
    }
    return launch_products_as<L, M, true>(jobs, dependent, st);
}

// The sums of up to two products whose last tiles may be split.
int launch_split_sums(const softsync::MmaJob<softsync::StoreEpilogue> *jobs, int count, cudaStream_t st)
{
    softsync::SplitSums in;
    int64_t blocks[2] = {0, 0};
    for (int k = 0; k < count; ++k) {
        const MmaPlan &plan = in.plan[k] = jobs[k].plan;
        in.target[k] = jobs[k].epilogue.target;
        const int64_t tiles = div_up(plan.m, kTile) * div_up(plan.n, kTile), rest = plan.live && !plan.live_is_k ? std::min<int64_t>(tiles, plan.slots - 1) : tiles % plan.slots;
        if (plan.live || plan.splits > 1) blocks[k] = std::min<int64_t>(rest * kTile / 2, 32 * plan.slots);         // rows in turn: 2 to 8 warps each
    }
    in.blocks = static_cast<int>(blocks[0]);
    return blocks[0] + blocks[1] ? start(softsync::split_sum_kernel, blocks[0] + blocks[1], 256, 0, true, st, in) : PS_OK;
}
// A product's rows of `stride` values to where they belong, dense: a launch for every so many rows (of a multiple of eight) as have fewer than 2^32 values.
template <typename T>
int launch_dense_rows(const T *from, int64_t rows, int64_t cols, int64_t stride, T *to, cudaStream_t st)
{
    const int64_t most = ((int64_t{1} << 32) - 4096) / cols / 8 * 8;
    const unsigned long long magic = cols == 1 ? 0 : ~0ull / static_cast<unsigned long long>(cols) + 1;
    for (int64_t first = 0; first < rows; first += most) {
        const int64_t count = std::min(most, rows - first) * cols;
        const int status = start(softsync::dense_rows_kernel<T>, div_up(count, softsync::kDenseThreads * softsync::kUnit), softsync::kDenseThreads, 0, true, st, from + first * stride,
                                 static_cast<long long>(stride), static_cast<unsigned>(count), static_cast<int>(cols), magic, to + first * cols);
        if (status != PS_OK) return status;
    }
    return PS_OK;
}
// Room for the parts of a product's split tiles, whatever the device leaves of its extents: at most kMostParts x kPairs, of fewer tiles than there are pairs, each in parts of four stages at least.
int64_t part_elements(int64_t m, int64_t n, int64_t k)
{
    const int64_t steps = div_up(k, kStep), tiles = div_up(m, kTile) * div_up(n, kTile);
    if (steps < softsync::kLeastSplit) return 0;
    const int64_t each = std::min<int64_t>(softsync::split_choice(softsync::kSplitChoices - 1), steps / softsync::kLeastPart);
    return std::min(int64_t{softsync::kMostParts} * kPairs, std::min<int64_t>(tiles, kPairs - 1) * each) * kTile * kTile;
}

// Row tiles that take turns before the next column tile's: as many as leave their operand in the L2 (32 MB of it), so that the other one is read once for all of them
// (7168 x 2048 x 131072: 10.02 ms with 8 MB, 9.93 with 32, 10.26 with 64).
int group_of(int64_t m, int64_t k)
{
    return static_cast<int>(std::max<int64_t>(1, std::min(div_up(m, kTile), (int64_t{32} << 20) / (2 * kTile * std::max<int64_t>(k, 1)))));
}

int64_t gather_blocks(int64_t rows, int64_t stride) { return div_up(rows * div_up(stride, softsync::kGatherColumns), softsync::kGatherThreads / 32); }

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

// The vocabulary in pieces: [first, vocab), the widest, whose exponentials the statistics' pass keeps, so that its logits are computed once; and those
// before it, of `piece` columns each.
struct HeadPlan : Places {
    int64_t rows, width, vocab, rows_padded, width_padded, first, piece, g_stride, parts, part_count;
    bool copy_head, copy_hidden;
    float2 *stat = nullptr, *norms = nullptr;
    float *picked = nullptr, *scales = nullptr;
    double *sum = nullptr, *sums = nullptr;
    unsigned *done = nullptr;
    int *order = nullptr, *place = nullptr, *live = nullptr;
    bf16 *hidden = nullptr, *head = nullptr;
    bf16 *g = nullptr, *dhead = nullptr;   // dhead: a piece's rows, where dense ones allow no vectors
    float *dhidden = nullptr, *split_hidden = nullptr, *split_head = nullptr;
    HeadPlan(const ps_head &h, bool grad, bool listed, void *p) : Places(p), rows(h.rows), width(h.width), vocab(h.vocab)
    {
        rows_padded = round_up(rows, kStep);
        width_padded = round_up(width, kStep);              // of copies: rows of whole lines
        copy_head = !matrix_aligned(h.head_dev, vocab, h.head_stride);
        // Rows that straddle lines of 128 bytes are loaded slowly: 1024 x 2040 x 50257 733 us as they lie, 626 from a copy (log probabilities alone 232 and 176); 512 x 1000 196 and 199 (62
        // and 52), 1024 x 200 151 and 163.  The head stays: its copy would cost as much memory as the call is to save.
        copy_hidden = listed || !matrix_aligned(h.hidden_dev, rows, h.hidden_stride) || (h.hidden_stride % kStep && rows > 2 * kTile && width > 2 * kTile);
        part_count = div_up(vocab, kHalf);
        const int64_t most = std::max<int64_t>(kTile, std::max(kPieceBytes, rows * width * 2) / (2 * rows_padded) / kTile * kTile);
        first = vocab > most ? round_up(vocab - most, kTile) : 0;
        piece = first ? round_up(div_up(first, div_up(first, most)), kTile) : 0;
        g_stride = round_up(std::max(piece, vocab - first), kTile);
        take(scales, 3);
        take(sum, 1);
        take(live, 1);
        take(done, 1);
        take(order, rows);
        take(place, rows);
        take(picked, rows);
        take(norms, rows);
        take(sums, div_up(rows, softsync::kJoinRows));
        if (copy_hidden) take(hidden, rows_padded * width_padded);
        if (copy_head) take(head, round_up(vocab, kStep) * width_padded);
        take(stat, part_count * rows);
        if (!grad) return;
        take(g, rows_padded * g_stride);
        const int64_t widest = std::max(piece, vocab - first);
        take(split_hidden, part_elements(rows, width, widest));
        take(split_head, part_elements(widest, width, rows));
        if (first) take(dhidden, rows * width_padded);
        if (width % 8) take(dhead, widest * width_padded);
    }
};

int check_head(const ps_head *h)
{
    if (!h || h->rows < 0 || h->rows > kMaxRows || h->width < 1 || h->width > kMaxWidth || h->vocab < 1 || h->vocab > kMaxVocab) return PS_ERR_INVALID_ARG;
    // 1 / T, and log2(e) / T: the exponentials' scale
    if (!(h->temperature > 0.f) || !std::isfinite(h->temperature) || !std::isfinite(static_cast<float>(kLog2E / h->temperature))) return PS_ERR_INVALID_ARG;
    if (too_many_tiles(h->rows, h->vocab) || too_many_tiles(h->rows, h->width) || too_many_tiles(h->vocab, h->width)) return PS_ERR_INVALID_ARG;
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
          scale(static_cast<float>(kLog2E / head_.temperature)), inv_temperature(1.f / head_.temperature)
    {
        const auto given = [](const void *p, int64_t rows, int64_t cols, int64_t stride) { return Matrix{static_cast<const bf16 *>(p), rows, cols, rows > 1 ? stride : round_up(cols, 8)}; };
        hidden = w.copy_hidden ? Matrix{w.hidden, w.rows_padded, w.width, w.width_padded} : given(h.hidden_dev, h.rows, h.width, h.hidden_stride);
        head = w.copy_head ? Matrix{w.head, h.vocab, h.width, w.width_padded} : given(h.head_dev, h.vocab, h.width, h.head_stride);
    }
    const int *order() const { return listed ? w.order : nullptr; }
    const int *live() const { return listed ? w.live : nullptr; }

    bool started = false;                  // a kernel of this call is under way
    bool dependent() { const bool d = started; started = true; return d; }

    int begin(const float *factors, float *zero_a, float *zero_b, void *dhidden)
    {
        int status = PS_OK;
        if (listed)
            status = start(softsync::order_kernel, 1, softsync::kOrderThreads, 0, dependent(), st, factors, static_cast<int>(h.rows),
                            softsync::OrderOut{w.order, w.place, w.live, w.sum, w.scales, zero_a, zero_b});
        softsync::GatherIn in{};
        in.width = static_cast<int>(h.width); in.out_stride = static_cast<int>(w.width_padded);
        if (status == PS_OK && w.copy_head) {
            in.x = static_cast<const bf16 *>(h.head_dev); in.rows = static_cast<int>(h.vocab); in.stride = h.head_stride; in.out = w.head;
            status = start(softsync::gather_kernel, gather_blocks(round_up(h.vocab, kStep), w.width_padded), softsync::kGatherThreads, 0, dependent(), st, in);
        }
        if (status == PS_OK && w.copy_hidden) {
            in.x = static_cast<const bf16 *>(h.hidden_dev); in.rows = static_cast<int>(h.rows); in.stride = h.hidden_stride; in.out = w.hidden;
            in.aligned = matrix_aligned(h.hidden_dev, h.rows, h.hidden_stride);
            if (listed) { in.order = w.order; in.place = w.place; in.live = w.live; in.zeros = static_cast<bf16 *>(dhidden); }
            status = start(softsync::gather_kernel, gather_blocks(w.rows_padded, w.width_padded), softsync::kGatherThreads, 0, dependent(), st, in);
        }
        return status;
    }
    // stats: loss and sum of the weights, or null.  keep: the exponentials of the columns from w.first on.
    int statistics(const float *weights, float *logp, float *lse, float *stats, bool keep)
    {
        softsync::StatsEpilogue ep{};
        ep.order = order(); ep.tokens = tokens; ep.rows = static_cast<int>(h.rows); ep.vocab = static_cast<int>(h.vocab); ep.live = live(); ep.scale = scale;
        ep.parts = w.stat; ep.part_stride = h.rows; ep.picked = w.picked; ep.done = w.done;
        if (keep) { ep.kept = reinterpret_cast<uint16_t *>(w.g); ep.kept_stride = w.g_stride; ep.first = static_cast<int>(w.first); }
        const MmaPlan plan{static_cast<int>(h.rows), static_cast<int>(h.vocab), static_cast<int>(h.width), 0, live(), 0, 0, group_of(h.rows, h.width)};
        softsync::MmaJob<softsync::StatsEpilogue> job;
        if (!job_of<Lying<false, false>>(job, hidden, head, plan, ep)) return PS_ERR_CUDA;
        const int status = launch_products<Lying<false, false>>(&job, dependent(), st);
        if (status != PS_OK) return status;
        softsync::JoinIn in{};
        in.parts = w.stat; in.part_stride = h.rows; in.count = static_cast<int>(w.part_count); in.picked = w.picked; in.tokens = tokens; in.order = order(); in.live = live();
        in.weights = weights; in.rows = ep.rows; in.vocab = ep.vocab; in.scale = scale; in.inv_temperature = inv_temperature; in.logp = logp; in.lse = lse; in.norms = w.norms;
        in.sums = w.sums; in.done = w.done; in.total = listed ? w.sum : nullptr; in.stats = stats;
        return start(softsync::join_kernel, div_up(h.rows, softsync::kJoinRows), softsync::kJoinThreads, 0, dependent(), st, in);
    }
    // lse: of every row; null after statistics that kept.  coef: of every row, or null for 1; alpha times *alpha_dev: of both gradients.
    int gradients(const float *lse, const float *coef, float sign, float alpha, const float *alpha_dev, void *dhidden, void *dhead)
    {
        const int rows = static_cast<int>(h.rows), width = static_cast<int>(h.width), slots = slots_on_device();
        if (slots < 1) return PS_ERR_CUDA;
        using OfHidden = Lying<false, true>;
        using OfHead = Lying<true, true>;
        const int64_t pieces = 1 + (w.first ? div_up(w.first, w.piece) : 0);
        for (int64_t k = 0; k < pieces; ++k) {                                  // the kept one first: the others take its place
            const int64_t first = k ? (k - 1) * w.piece : w.first;
            const int n = static_cast<int>(k ? std::min(w.piece, w.first - first) : h.vocab - first);
            const Matrix entries{head.data + first * head.stride, n, h.width, head.stride}, g{w.g, w.rows_padded, n, w.g_stride};
            int status;
            if (k == 0 && !lse) {
                softsync::KeptIn in{};
                in.g = reinterpret_cast<uint4 *>(w.g); in.stride = w.g_stride / 8; in.first = static_cast<int>(first); in.width = n;
                in.segments = static_cast<int>(div_up(n, softsync::kKeptColumns)); in.parts = w.stat; in.norms = w.norms; in.part_stride = h.rows; in.tokens = tokens;
                in.order = order(); in.live = live(); in.coef = coef; in.coef_scale = w.scales; in.sign = sign; in.scale = scale; in.rows = rows;
                status = start(softsync::kept_grad_kernel, w.rows_padded * in.segments, softsync::kKeptThreads, 0, dependent(), st, in);
            } else {
                softsync::GradEpilogue ge{};
                ge.order = order(); ge.tokens = tokens; ge.norms = lse ? nullptr : w.norms; ge.lse = lse; ge.coef = coef; ge.coef_scale = w.scales; ge.sign = sign; ge.rows = rows; ge.vocab = static_cast<int>(h.vocab); ge.live = live();
                ge.scale = lse ? inv_temperature : scale; ge.last = lse ? static_cast<float>(kLog2E) : 1.f;
                ge.first = static_cast<int>(first); ge.width = n; ge.g = w.g; ge.g_stride = w.g_stride;
                const MmaPlan plan{rows, n, width, 0, live(), 0, 0, group_of(rows, width)};
                softsync::MmaJob<softsync::GradEpilogue> job;
                status = job_of<Lying<false, false>>(job, hidden, entries, plan, ge) ? launch_products<Lying<false, false>>(&job, dependent(), st) : PS_ERR_CUDA;
            }
            softsync::MmaJob<softsync::StoreEpilogue> jobs[2];
            int count = 0;
            if (status == PS_OK && dhidden) {
                softsync::StoreEpilogue se{};
                softsync::StoreTarget &t = se.target;
                t.rows = rows; t.cols = width; t.live = live(); t.order = order(); t.alpha = alpha; t.alpha_dev = alpha_dev;
                if (k == pieces - 1) { t.out = dhidden; t.out_bf16 = 1; t.vectors = width % 8 == 0; t.stride = width; }
                t.sum = w.dhidden; t.sum_stride = w.width_padded; t.add = k > 0; t.parts = w.split_hidden;
                if (!job_of<OfHidden>(jobs[count++], g, entries, MmaPlan{rows, width, n, 0, live(), 0, slots, group_of(rows, n)}, se)) return PS_ERR_CUDA;
            }
            if (status == PS_OK && dhead) {
                softsync::StoreEpilogue se{};
                softsync::StoreTarget &t = se.target;
                t.rows = n; t.cols = width; t.alpha = alpha; t.alpha_dev = alpha_dev; t.out = w.dhead ? w.dhead : static_cast<bf16 *>(dhead) + first * h.width;
                t.out_bf16 = 1; t.vectors = 1; t.stride = w.dhead ? w.width_padded : h.width; t.parts = w.split_head;
                if (!job_of<OfHead>(jobs[count++], g, hidden, MmaPlan{n, width, rows, 0, live(), 1, slots, group_of(n, rows)}, se)) return PS_ERR_CUDA;
            }
            if (status == PS_OK && count) 
                status = count == 2 ? launch_products<OfHidden, OfHead>(jobs, dependent(), st) : dhidden ? launch_products<OfHidden>(jobs, dependent(), st) : launch_products<OfHead>(jobs, dependent(), st);
            if (status == PS_OK && count) status = launch_split_sums(jobs, count, st);
            if (status == PS_OK && dhead && w.dhead) status = launch_dense_rows(w.dhead, n, h.width, w.width_padded, static_cast<bf16 *>(dhead) + first * h.width, st);
            if (status != PS_OK) return status;
        }
        return PS_OK;
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
    const int status = call.begin(weights_dev, logp_dev, lse_dev, nullptr);
    return status == PS_OK ? call.statistics(nullptr, logp_dev, lse_dev, nullptr, false) : status;
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
    const int status = call.begin(dlogp_dev, nullptr, nullptr, dhidden_dev);
    return status == PS_OK ? call.gradients(lse_dev, dlogp_dev, -1.f, call.inv_temperature, call.w.scales + 1, dhidden_dev, dhead_dev) : status;
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
    int status = call.begin(weights_dev, logp_dev, lse_dev, dhidden_dev);
    if (status == PS_OK) status = call.statistics(weights_dev, logp_dev, lse_dev, stats_dev, grad);
    if (status != PS_OK || !grad) return status;
    return call.gradients(nullptr, weights_dev, 1.f, listed ? call.inv_temperature : call.inv_temperature / static_cast<float>(head->rows), listed ? call.w.scales + 2 : nullptr, dhidden_dev,
                          dhead_dev);
}

}  // extern "C"

// ---- weight gradient from packed activations -----------------------------------------------------------------------------
namespace {

struct PackedPlan : Places {
    int64_t outs_padded, cols_padded;
    bool copy_dout;
    bf16 *dout = nullptr, *values = nullptr;
    void *dweight = nullptr;               // rows of cols_padded values, where dense ones allow no vectors
    float *split = nullptr;
    PackedPlan(const ps_packed_grad &a, void *p) : Places(p), outs_padded(round_up(a.outs, kStep)), cols_padded(round_up(a.cols, kStep))
    {
        copy_dout = !matrix_aligned(a.dout_dev, a.rows, a.dout_stride);
        if (copy_dout) take(dout, round_up(a.rows, kStep) * outs_padded);
        take(values, a.rows * cols_padded);
        take(split, part_elements(a.outs, a.cols, a.rows));
        if (a.cols % 8) {
            char *place;
            take(place, a.outs * cols_padded * (a.out_dtype == PS_GRAD_BF16 ? 2 : 4));
            dweight = place;
        }
    }
};

int check_packed(const ps_packed_grad *a)
{
    const auto is_dtype = [](int t) { return t == PS_GRAD_FP32 || t == PS_GRAD_BF16; };
    if (!a || a->rows < 0 || a->rows > kMaxRows || a->outs < 1 || a->outs > kMaxVocab || a->cols < 1 || a->cols > kMaxWidth || !is_dtype(a->out_dtype)) return PS_ERR_INVALID_ARG;
    if (a->gain_dev && (!is_dtype(a->gain_dtype) || !aligned_to(a->gain_dev, a->gain_dtype == PS_GRAD_BF16 ? 2 : 4))) return PS_ERR_INVALID_ARG;
    if (a->rows > 1 && (a->dout_stride < a->outs || a->dout_stride > (int64_t{1} << 38))) return PS_ERR_INVALID_ARG;
    if (too_many_tiles(a->outs, a->cols)) return PS_ERR_INVALID_ARG;
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
    const int slots = slots_on_device();
    if (slots < 1) return PS_ERR_CUDA;
    Matrix dout{static_cast<const bf16 *>(a->dout_dev), rows, outs, rows > 1 ? a->dout_stride : w.outs_padded};
    int status = PS_OK;
    if (w.copy_dout) {
        softsync::GatherIn in{};
        in.x = dout.data; in.rows = rows; in.width = outs; in.stride = a->dout_stride; in.out = w.dout; in.out_stride = static_cast<int>(w.outs_padded);
        status = start(softsync::gather_kernel, gather_blocks(round_up(rows, kStep), w.outs_padded), softsync::kGatherThreads, 0, false, st, in);
        dout = Matrix{w.dout, rows, outs, w.outs_padded};
    }
    if (status != PS_OK) return status;
    // The codes' values go through memory: turned into bf16 under way (four to eight more warps, from a ring of codes to the tensor cores' one) they took the shared memory's
    // bandwidth from the products (8192 x 8192 x 2048: 285 us, against 10 and 180).
    if ((status = ps_unpack8(a->codes_dev, a->scales_dev, rows, cols, w.values, PS_GRAD_BF16, w.cols_padded, stream)) != PS_OK) return status;
    const Matrix values{w.values, rows, cols, w.cols_padded};
    softsync::StoreEpilogue se{};
    softsync::StoreTarget &t = se.target;
    t.rows = outs; t.cols = cols; t.alpha = 1.f; t.gain = a->gain_dev; t.gain_bf16 = a->gain_dtype == PS_GRAD_BF16; t.out = w.dweight ? w.dweight : a->dweight_dev;
    t.out_bf16 = a->out_dtype == PS_GRAD_BF16; t.vectors = aligned_to(a->gain_dev, 16); t.stride = w.dweight ? w.cols_padded : cols; t.parts = w.split;
    softsync::MmaJob<softsync::StoreEpilogue> job;
    if (!job_of<Lying<true, true>>(job, dout, values, MmaPlan{outs, cols, rows, 0, nullptr, 0, slots, group_of(outs, rows)}, se, t.out_bf16)) return PS_ERR_CUDA;
    status = launch_products<Lying<true, true>>(&job, true, st);
    if (status == PS_OK) status = launch_split_sums(&job, 1, st);
    if (status != PS_OK || !w.dweight) return status;
    return t.out_bf16 ? launch_dense_rows(static_cast<const bf16 *>(w.dweight), outs, cols, w.cols_padded, static_cast<bf16 *>(a->dweight_dev), st)
                      : launch_dense_rows(static_cast<const float *>(w.dweight), outs, cols, w.cols_padded, static_cast<float *>(a->dweight_dev), st);
}

}  // extern "C"
