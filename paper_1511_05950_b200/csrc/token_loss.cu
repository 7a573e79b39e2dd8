// Entry points of softsync_learn.h that work on rows of logits: token log probabilities, policy loss, preference loss.
#include "../../include/softsync_learn.h"
#include "host_util.h"
#include "token_kernels.cuh"

#include <algorithm>
#include <atomic>
#include <cmath>
#include <type_traits>

using softsync::aligned_to;
using softsync::GradBf16;
using softsync::GradFp32;
using softsync::PairTail;
using softsync::PolicyIn;
using softsync::PolicyState;
using softsync::PreferenceIn;
using softsync::RowCoef;
using softsync::RowsIn;
using softsync::RowStat;
using softsync::StatsOut;

namespace {

int64_t round_up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }
int64_t div_up(int64_t x, int64_t by) { return (x + by - 1) / by; }

constexpr int64_t kMaxParts = 1024;       // that the rows of a policy loss are summed in, at most

// Places in the losses' workspace.  Its first word counts finished blocks and is zero between calls.
struct Workspace {
    int64_t bytes = 0;
    unsigned *done = nullptr;
    explicit Workspace(void *p) { take(p, done, 1); }
protected:
    template <typename T> void take(void *p, T *&out, int64_t count)
    {
        out = reinterpret_cast<T *>(static_cast<char *>(p) + bytes);
        bytes += round_up(count * static_cast<int64_t>(sizeof(T)), 256);
    }
};
struct PolicyWorkspace : Workspace {
    PolicyState st{};
    RowStat *stat = nullptr;
    RowCoef *coef = nullptr;
    float *entropy = nullptr;
    PolicyWorkspace(void *p, int64_t rows) : Workspace(p)
    {
        st.done = done;
        take(p, st.inv_weight, 1);
        take(p, st.part_sum, std::min(rows, kMaxParts));
        take(p, stat, rows);
        take(p, coef, rows);
        take(p, entropy, rows);
        take(p, st.order, rows);
        take(p, st.live, 1);
    }
};
struct PreferenceWorkspace : Workspace {
    double (*pairs)[3] = nullptr;          // terms of each pair
    RowStat *stat = nullptr;
    RowCoef *coef = nullptr;
    float *logp = nullptr;
    PreferenceWorkspace(void *p, int64_t rows, int64_t sequences) : Workspace(p)
    {
        take(p, pairs, sequences / 2);
        take(p, stat, rows);
        take(p, coef, rows);
        take(p, logp, rows);
    }
};

constexpr int64_t kMaxRows = 0x7fffffff;

int check_logits(const ps_logits *lg)
{
    if (!lg || (lg->dtype != PS_GRAD_FP32 && lg->dtype != PS_GRAD_BF16)) return PS_ERR_INVALID_ARG;
    if (lg->rows < 0 || lg->rows > kMaxRows || lg->vocab < 1 || lg->vocab > (int64_t{1} << 30) || lg->row_stride < lg->vocab) return PS_ERR_INVALID_ARG;
    if (!(lg->temperature > 0.f) || !std::isfinite(lg->temperature) || !std::isfinite(1.f / lg->temperature)) return PS_ERR_INVALID_ARG;
    if (lg->rows == 0) return PS_OK;
    if (lg->row_stride > (int64_t{1} << 60) / lg->rows) return PS_ERR_INVALID_ARG;
    if (!lg->data_dev || !lg->tokens_dev || !aligned_to(lg->data_dev, lg->dtype == PS_GRAD_BF16 ? 2 : 4)) return PS_ERR_INVALID_ARG;
    if (!aligned_to(lg->tokens_dev, 8) || !aligned_to(lg->weights_dev, 4)) return PS_ERR_INVALID_ARG;
    return PS_OK;
}

// The gradient either replaces the logits element by element or lies wholly elsewhere.
int check_gradient(const ps_logits *lg, const void *dlogits, int64_t stride)
{
    if (!dlogits || lg->rows == 0) return PS_OK;
    const int64_t elem = lg->dtype == PS_GRAD_BF16 ? 2 : 4;
    if (stride < lg->vocab || stride > (int64_t{1} << 60) / lg->rows || !aligned_to(dlogits, elem)) return PS_ERR_INVALID_ARG;
    if (dlogits == lg->data_dev) return stride == lg->row_stride ? PS_OK : PS_ERR_INVALID_ARG;
    const uintptr_t a = reinterpret_cast<uintptr_t>(dlogits), b = reinterpret_cast<uintptr_t>(lg->data_dev);
    const uintptr_t na = static_cast<uintptr_t>(((lg->rows - 1) * stride + lg->vocab) * elem);
    const uintptr_t nb = static_cast<uintptr_t>(((lg->rows - 1) * lg->row_stride + lg->vocab) * elem);
    return a < b + nb && b < a + na ? PS_ERR_INVALID_ARG : PS_OK;
}

RowsIn rows_in(const ps_logits *lg)
{
    RowsIn r;
    r.data = static_cast<const unsigned char *>(lg->data_dev);
    r.rows = lg->rows; r.vocab = lg->vocab; r.stride = lg->row_stride;
    r.tokens = reinterpret_cast<const long long *>(lg->tokens_dev);
    r.weights = lg->weights_dev;
    r.inv_temperature = 1.f / lg->temperature;
    r.scale = static_cast<float>(1.4426950408889634 / static_cast<double>(lg->temperature));
    return r;
}

int launched() { return cudaGetLastError() == cudaSuccess ? PS_OK : PS_ERR_CUDA; }

int sm_count()
{
    static std::atomic<int> cached[64] = {};
    int device = 0;
    if (cudaGetDevice(&device) != cudaSuccess || device < 0 || device >= 64) return 0;
    int n = cached[device].load(std::memory_order_relaxed);
    if (!n && cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, device) == cudaSuccess) cached[device].store(n, std::memory_order_relaxed);
    return n;
}

// `rows` clusters of `cluster` blocks.  dependent: the kernel may start while the one before it on the stream, one of this call's own,
// still runs, and waits for it itself before it touches what that one writes.
template <typename... P, typename... A>
int launch_rows(void (*kernel)(P...), int64_t rows, int cluster, int threads, int smem, bool dependent, cudaStream_t st, A... args)
{
    if (rows * cluster > 0x7fffffff) return PS_ERR_INVALID_ARG;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(rows * cluster));
    cfg.blockDim = dim3(static_cast<unsigned>(threads));
    cfg.dynamicSmemBytes = static_cast<size_t>(smem);
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = static_cast<unsigned>(cluster);
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = dependent ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...) == cudaSuccess ? PS_OK : PS_ERR_CUDA;
}

// Most 16-byte vectors that a row touches.
int64_t row_vectors(const ps_logits *lg)
{
    const int64_t elem = lg->dtype == PS_GRAD_BF16 ? 2 : 4, per = 16 / elem;
    const int64_t phase = lg->rows == 1 || lg->row_stride * elem % 16 == 0 ? (reinterpret_cast<uintptr_t>(lg->data_dev) & 15) / elem : per - 1;
    return div_up(phase + lg->vocab, per);
}

constexpr int kMaxCluster = softsync::kMaxCluster;
constexpr int kWaitLimit = 1 << 20;                    // polls of up to a microsecond each

// Threads of a row's blocks: as few as keep the row's loads under way, since warps without a vector of their own and a wider join cost time.
// Two vectors a thread and batch with 64 threads, four beyond.  Measured on 2.5e8 elements, all with the entropy, 64 | 256 | 512 threads:
// 256 vectors a row (2048 bf16) 344 | 438 | 905 us, 276 (1100 fp32) 716 | 676 | 1348; 6283 vectors (50257 bf16) 197 | 102 | 129, 8192 (65536 bf16)
// 188 | 90 | 88, 25000 (200000 bf16) 284 | 104 | 98; with few rows (256 of 100000 bf16) 76 | 23 | 20.
template <typename GT, bool ENTROPY>
int launch_stats_as(const RowsIn &in, int64_t vectors, const StatsOut &out, cudaStream_t st)
{
    auto go = [&](auto kernel, int threads, int batch) {
        int cluster = 1;                                  // few rows: several blocks each, as long as every one has work
        while (cluster < kMaxCluster && in.rows * cluster * 2 <= 2 * sm_count() && vectors > static_cast<int64_t>(cluster) * threads * batch) cluster *= 2;
        return launch_rows(kernel, in.rows, cluster, threads, 0, false, st, in, out);
    };
    if (vectors <= 256) return go(softsync::row_stats_kernel<GT, 64, 2, ENTROPY>, 64, 2);
    if (vectors < 8192) return go(softsync::row_stats_kernel<GT, 256, 4, ENTROPY>, 256, 4);
    return go(softsync::row_stats_kernel<GT, 512, 4, ENTROPY>, 512, 4);
}
int launch_stats(const ps_logits *lg, const RowsIn &in, const StatsOut &out, bool entropy, cudaStream_t st)
{
    const int64_t n = row_vectors(lg);
    if (lg->dtype == PS_GRAD_BF16) return entropy ? launch_stats_as<GradBf16, true>(in, n, out, st) : launch_stats_as<GradBf16, false>(in, n, out, st);
    return entropy ? launch_stats_as<GradFp32, true>(in, n, out, st) : launch_stats_as<GradFp32, false>(in, n, out, st);
}

int launch_grad(const ps_logits *lg, const RowsIn &in, const RowStat *stat, const RowCoef *coef, const float *entropy, void *out,
                int64_t stride, const PairTail &tail, cudaStream_t st)
{
    const int64_t segments = div_up(row_vectors(lg), softsync::kGradThreads * softsync::kGradVectors);
    const int64_t blocks = lg->rows * segments + (tail.stats ? 1 : 0);
    if (blocks > 0x7fffffff) return PS_ERR_INVALID_ARG;
    const int seg = static_cast<int>(segments);
    auto go = [&](auto kernel) {
        return launch_rows(kernel, blocks, 1, softsync::kGradThreads, 0, true, st, in, stat, coef, entropy, static_cast<unsigned char *>(out),
                           static_cast<long long>(stride), seg, tail);
    };
    if (lg->dtype == PS_GRAD_BF16) return entropy ? go(softsync::row_grad_kernel<GradBf16, true>) : go(softsync::row_grad_kernel<GradBf16, false>);
    return entropy ? go(softsync::row_grad_kernel<GradFp32, true>) : go(softsync::row_grad_kernel<GradFp32, false>);
}

struct PolicyCall {
    RowsIn rows;
    PolicyIn in;
    PolicyState st;
    float *logp, *entropy;
    unsigned char *out;
    int64_t stride, vectors;
};

int launch_totals(const RowsIn &rows, int from, const PolicyState &state, float *logp, float *entropy, cudaStream_t st)
{
    softsync::policy_totals_kernel<<<1, softsync::kTermThreads, 0, st>>>(rows.weights, rows.rows, from, state, logp, entropy);
    return launched();
}

// Clusters of the ring kernel that run at once on the current GPU (asked once for each kernel, cluster size and GPU).
template <typename GT, bool ENTROPY_GRAD, int T>
int resident_clusters(int cluster)
{
    using Shape = softsync::RingShape<T>;
    const auto kernel = softsync::policy_ring_kernel<GT, ENTROPY_GRAD, T>;
    static std::atomic<int> known[64][kMaxCluster + 1] = {};
    int device = 0, n = 0;
    if (cudaGetDevice(&device) != cudaSuccess || device < 0 || device >= 64) return 0;
    if ((n = known[device][cluster].load(std::memory_order_relaxed)) > 0) return n;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape::bytes) != cudaSuccess) return 0;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(cluster));
    cfg.blockDim = dim3(Shape::block);
    cfg.dynamicSmemBytes = Shape::bytes;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = static_cast<unsigned>(cluster);
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess || n < 1) return 0;
    known[device][cluster].store(n, std::memory_order_relaxed);
    return n;
}

template <typename GT, bool ENTROPY_GRAD, int T>
int launch_ring_as(const PolicyCall &k, int cluster, cudaStream_t st)
{
    using Shape = softsync::RingShape<T>;
    auto kernel = softsync::policy_ring_kernel<GT, ENTROPY_GRAD, T>;
    softsync::RingPlan plan;
    plan.vectors = static_cast<int>(div_up(k.vectors, cluster));
    plan.chunks = static_cast<int>(div_up(plan.vectors, Shape::chunk));
    plan.ahead = std::min(plan.chunks, softsync::kRingSlots - plan.chunks);
    plan.wait_limit = kWaitLimit;
    const int64_t resident = resident_clusters<GT, ENTROPY_GRAD, T>(cluster);
    if (resident < 1) return PS_ERR_CUDA;
    const int64_t parts = std::min({static_cast<int64_t>(k.rows.rows), resident, kMaxParts});
    // Weights: a kernel before this one adds them up and lists the rows, unless no cluster gets a second row, and every block adds for itself.
    PolicyState state = k.st;
    const bool listed = k.rows.weights && k.rows.rows > parts;
    if (listed) {
        const int status = launch_totals(k.rows, static_cast<int>(parts), state, k.logp, k.entropy, st);
        if (status != PS_OK) return status;
    } else {
        state.order = nullptr;
    }
    return launch_rows(kernel, parts, cluster, Shape::block, Shape::bytes, listed, st, k.rows, k.in, state, k.logp, k.entropy,
                       k.out, static_cast<long long>(k.stride), plan);
}

// Which ring kernel, and the blocks that a row is spread over; no blocks: the row does not fit.
//
// As few blocks as hold a row: more means more exchange, and a cluster's blocks wait for one another at every row.  A row that fits one
// narrow block has two of them on an SM, in different phases (16384 x 50257 bf16: 629 us, one wide block 715); one that needs more takes one
// or two wide blocks (8192 x 152000 bf16: 937 us with two, 1011 with three narrow ones; 8192 x 65536: 380 with one, 406 with two).  Three
// wide blocks leave more SMs out than five narrow ones (4096 x 128000 fp32: 777 us, 698), so beyond two the narrow ones take over as far
// as they go.  Where rows are so few that the GPU would stay half empty, more narrow blocks share each (48 x 32000 bf16: 11.7 us with four).
struct RingChoice { int threads, cluster; };
RingChoice ring_choice(int64_t vectors, int64_t rows)
{
    if (rows > (int64_t{1} << 30)) return RingChoice{softsync::kNarrow, 0};
    const int64_t narrow = div_up(vectors, softsync::RingShape<softsync::kNarrow>::row), wide = div_up(vectors, softsync::RingShape<softsync::kWide>::row);
    if (narrow > 1 && (wide <= 2 || narrow > kMaxCluster) && (narrow > kMaxCluster || rows * narrow > sm_count()))
        return RingChoice{softsync::kWide, wide <= kMaxCluster ? static_cast<int>(wide) : 0};
    int64_t cluster = narrow;
    while (cluster * 2 <= kMaxCluster && rows * cluster * 2 <= 2 * sm_count() && vectors > cluster * softsync::kNarrow) cluster *= 2;
    return RingChoice{softsync::kNarrow, static_cast<int>(cluster)};
}

int launch_ring(int dtype, const PolicyCall &k, const RingChoice &choice, cudaStream_t st)
{
    const auto go = [&](auto grad, auto ent) {
        using GT = decltype(grad);
        if (choice.threads == softsync::kNarrow) return launch_ring_as<GT, decltype(ent)::value, softsync::kNarrow>(k, choice.cluster, st);
        return launch_ring_as<GT, decltype(ent)::value, softsync::kWide>(k, choice.cluster, st);
    };
    const bool ent = k.in.entropy_coef != 0.f;
    if (dtype == PS_GRAD_BF16) return ent ? go(GradBf16{}, std::true_type{}) : go(GradBf16{}, std::false_type{});
    return ent ? go(GradFp32{}, std::true_type{}) : go(GradFp32{}, std::false_type{});
}

}  // namespace

extern "C" {

int ps_loss_workspace(int64_t rows, int64_t sequences, int64_t *bytes)
{
    if (!bytes || rows < 0 || rows > kMaxRows || sequences < 0 || sequences > (int64_t{1} << 31)) return PS_ERR_INVALID_ARG;
    *bytes = std::max(PolicyWorkspace(nullptr, rows).bytes, PreferenceWorkspace(nullptr, rows, sequences).bytes);
    return PS_OK;
}

int ps_token_logprob(const ps_logits *logits, float *logp_dev, float *lse_dev, float *entropy_dev, void *stream)
{
    const int bad = check_logits(logits);
    if (bad != PS_OK) return bad;
    if (logits->rows == 0) return PS_OK;
    if (!logp_dev || !aligned_to(logp_dev, 4) || !aligned_to(lse_dev, 4) || !aligned_to(entropy_dev, 4)) return PS_ERR_INVALID_ARG;
    return launch_stats(logits, rows_in(logits), StatsOut{logp_dev, lse_dev, entropy_dev, nullptr, nullptr}, entropy_dev != nullptr,
                        static_cast<cudaStream_t>(stream));
}

int ps_policy_loss(const ps_logits *logits, const ps_policy_inputs *in, float *stats_dev, float *logp_dev, float *entropy_dev,
                   void *dlogits_dev, int64_t dlogits_stride, void *workspace_dev, int64_t workspace_bytes, void *stream)
{
    int status = check_logits(logits);
    if (status == PS_OK && (!in || !stats_dev || !aligned_to(stats_dev, 4))) status = PS_ERR_INVALID_ARG;
    if (status == PS_OK) status = check_gradient(logits, dlogits_dev, dlogits_stride);
    if (status != PS_OK) return status;
    if (!(in->clip_low >= 0.f && in->clip_low <= 1.f) || !(in->clip_high >= 0.f) || !std::isfinite(in->clip_high) ||
        !std::isfinite(in->kl_coef) || !std::isfinite(in->entropy_coef))
        return PS_ERR_INVALID_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (logits->rows == 0) return cudaMemsetAsync(stats_dev, 0, 5 * sizeof(float), st) == cudaSuccess ? PS_OK : PS_ERR_CUDA;
    const PolicyWorkspace ws(workspace_dev, logits->rows);
    if (!logp_dev || !in->old_logp_dev || !in->advantages_dev || !workspace_dev || workspace_bytes < ws.bytes ||
        !aligned_to(workspace_dev, 16) || !aligned_to(logp_dev, 4) || !aligned_to(entropy_dev, 4) || !aligned_to(in->old_logp_dev, 4) ||
        !aligned_to(in->advantages_dev, 4) || !aligned_to(in->ref_logp_dev, 4))
        return PS_ERR_INVALID_ARG;
    PolicyCall k;
    k.rows = rows_in(logits);
    k.in = PolicyIn{in->old_logp_dev, in->advantages_dev, in->ref_logp_dev, 1.f - in->clip_low, 1.f + in->clip_high,
                    in->ref_logp_dev ? in->kl_coef : 0.f, in->entropy_coef};
    k.st = ws.st;
    k.st.stats = stats_dev;
    k.logp = logp_dev;
    k.entropy = entropy_dev ? entropy_dev : ws.entropy;
    k.out = static_cast<unsigned char *>(dlogits_dev);
    k.stride = dlogits_stride;
    k.vectors = row_vectors(logits);
    const RingChoice ring = ring_choice(k.vectors, logits->rows);
    if (ring.cluster) return launch_ring(logits->dtype, k, ring, st);
    k.st.order = k.st.live = nullptr;
    if ((status = launch_totals(k.rows, 0, k.st, logp_dev, k.entropy, st)) != PS_OK) return status;
    if ((status = launch_stats(logits, k.rows, StatsOut{logp_dev, nullptr, k.entropy, ws.stat, nullptr}, true, st)) != PS_OK) return status;
    softsync::policy_terms_kernel<<<static_cast<unsigned>(std::min(logits->rows, kMaxParts)), 32, 0, st>>>(k.rows, k.in, k.st, logp_dev, k.entropy,
                                                                                                        dlogits_dev ? ws.coef : nullptr);
    if ((status = launched()) != PS_OK || !dlogits_dev) return status;
    return launch_grad(logits, k.rows, ws.stat, ws.coef, in->entropy_coef != 0.f ? k.entropy : nullptr, dlogits_dev, dlogits_stride, PairTail{}, st);
}

int ps_preference_loss(const ps_logits *logits, const ps_preference_inputs *in, float *stats_dev, float *seq_logp_dev,
                       void *dlogits_dev, int64_t dlogits_stride, void *workspace_dev, int64_t workspace_bytes, void *stream)
{
    int status = check_logits(logits);
    if (status == PS_OK && (!in || !stats_dev || !aligned_to(stats_dev, 4) || in->pairs < 0 || in->pairs > (int64_t{1} << 30))) status = PS_ERR_INVALID_ARG;
    if (status == PS_OK) status = check_gradient(logits, dlogits_dev, dlogits_stride);
    if (status != PS_OK) return status;
    if (!std::isfinite(in->beta) || !(in->label_smoothing >= 0.f && in->label_smoothing <= 1.f)) return PS_ERR_INVALID_ARG;
    if (in->pairs && (!in->offsets_dev || !in->ref_logp_dev || !seq_logp_dev || !aligned_to(in->offsets_dev, 8) ||
                      !aligned_to(in->ref_logp_dev, 4) || !aligned_to(seq_logp_dev, 4)))
        return PS_ERR_INVALID_ARG;
    const PreferenceWorkspace ws(workspace_dev, logits->rows, 2 * in->pairs);
    if (!workspace_dev || workspace_bytes < ws.bytes || !aligned_to(workspace_dev, 16)) return PS_ERR_INVALID_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const RowsIn rows = rows_in(logits);
    const PreferenceIn p{reinterpret_cast<const long long *>(in->offsets_dev), in->ref_logp_dev, in->pairs, in->beta, in->label_smoothing};
    if (logits->rows && (status = launch_stats(logits, rows, StatsOut{ws.logp, nullptr, nullptr, ws.stat, ws.coef}, false, st)) != PS_OK) return status;
    const bool grad = dlogits_dev && logits->rows;
    if (in->pairs)
        status = launch_rows(softsync::preference_terms_kernel, in->pairs, 1, softsync::kPairThreads, 0, logits->rows > 0, st, rows, p, ws.logp, seq_logp_dev,
                             grad ? ws.coef : nullptr, ws.pairs, ws.done, grad ? nullptr : stats_dev);
    else if (cudaMemsetAsync(stats_dev, 0, 3 * sizeof(float), st) != cudaSuccess)
        status = PS_ERR_CUDA;
    if (status != PS_OK || !grad) return status;
    return launch_grad(logits, rows, ws.stat, ws.coef, nullptr, dlogits_dev, dlogits_stride, PairTail{ws.pairs, in->pairs, in->pairs ? stats_dev : nullptr}, st);
}

}  // extern "C"
