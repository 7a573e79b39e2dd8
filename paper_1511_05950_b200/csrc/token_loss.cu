// Entry points of softsync_learn.h that work on rows of logits: token log probabilities, policy loss, preference loss.
#include "../../include/softsync_learn.h"
#include "host_util.h"
#include "token_kernels.cuh"

#include <algorithm>
#include <atomic>
#include <cmath>

using softsync::aligned_to;
using softsync::GradBf16;
using softsync::GradFp32;
using softsync::PolicyIn;
using softsync::PreferenceIn;
using softsync::RowCoef;
using softsync::RowsIn;
using softsync::RowStat;
using softsync::StatsOut;
using softsync::TermsOut;
using softsync::Totals;

namespace {

int64_t round_up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }
int64_t div_up(int64_t x, int64_t by) { return (x + by - 1) / by; }

// Places in the losses' workspace.
struct Workspace {
    Totals *totals = nullptr;
    unsigned *counters = nullptr;
    double (*sums)[5] = nullptr;           // policy loss: of each group of rows
    double (*pairs)[3] = nullptr;          // preference loss: of each pair
    RowStat *stat = nullptr;
    RowCoef *coef = nullptr;
    float (*terms)[5] = nullptr;
    float *entropy = nullptr, *logp = nullptr;
    int64_t bytes = 0;
    Workspace(void *p, int64_t rows, int64_t sequences)
    {
        const int64_t groups = div_up(rows, softsync::kRowGroup);
        take(p, totals, 1);
        take(p, counters, groups + 1);
        take(p, sums, groups);
        take(p, pairs, sequences / 2);
        take(p, stat, rows);
        take(p, coef, rows);
        take(p, terms, rows);
        take(p, entropy, rows);
        take(p, logp, rows);
    }
private:
    template <typename T> void take(void *p, T *&out, int64_t count)
    {
        out = reinterpret_cast<T *>(static_cast<char *>(p) + bytes);
        bytes += round_up(count * static_cast<int64_t>(sizeof(T)), 256);
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

// One cluster of `cluster` blocks per row.  dependent: the kernel may start while the one before it on the stream still runs.
template <typename... P, typename... A>
int launch_rows(void (*kernel)(P...), int64_t rows, int cluster, int threads, bool dependent, cudaStream_t st, A... args)
{
    if (rows * cluster > 0x7fffffff) return PS_ERR_INVALID_ARG;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(rows * cluster));
    cfg.blockDim = dim3(static_cast<unsigned>(threads));
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

int64_t warps(int64_t threads) { return std::min<int64_t>(512, std::max<int64_t>(64, round_up(threads, 32))); }

constexpr int kStatsVectors = 4;
constexpr int kMaxCluster = softsync::kMaxCluster;

template <typename GT, bool ENTROPY>
int launch_stats_as(const RowsIn &in, int64_t vectors, const StatsOut &out, cudaStream_t st)
{
    const int threads = static_cast<int>(warps(div_up(vectors, kStatsVectors)));
    int cluster = 1;                                      // few rows: several blocks each, as long as every one has work
    while (cluster < kMaxCluster && in.rows * cluster * 2 <= 2 * sm_count() && vectors > static_cast<int64_t>(cluster) * threads * kStatsVectors) cluster *= 2;
    return launch_rows(softsync::row_stats_kernel<GT, kStatsVectors, ENTROPY>, in.rows, cluster, threads, false, st, in, out);
}
int launch_stats(const ps_logits *lg, const RowsIn &in, const StatsOut &out, bool entropy, cudaStream_t st)
{
    const int64_t n = row_vectors(lg);
    if (lg->dtype == PS_GRAD_BF16) return entropy ? launch_stats_as<GradBf16, true>(in, n, out, st) : launch_stats_as<GradBf16, false>(in, n, out, st);
    return entropy ? launch_stats_as<GradFp32, true>(in, n, out, st) : launch_stats_as<GradFp32, false>(in, n, out, st);
}

int launch_grad(const ps_logits *lg, const RowsIn &in, const RowStat *stat, const RowCoef *coef, const float *entropy, void *out,
                int64_t stride, cudaStream_t st)
{
    const int64_t segments = div_up(row_vectors(lg), softsync::kGradThreads * softsync::kGradVectors);
    if (lg->rows * segments > 0x7fffffff) return PS_ERR_INVALID_ARG;
    const unsigned grid = static_cast<unsigned>(lg->rows * segments);
    const int seg = static_cast<int>(segments), threads = softsync::kGradThreads;
    unsigned char *dst = static_cast<unsigned char *>(out);
    if (lg->dtype == PS_GRAD_BF16) {
        if (entropy) softsync::row_grad_kernel<GradBf16, true><<<grid, threads, 0, st>>>(in, stat, coef, entropy, dst, stride, seg);
        else softsync::row_grad_kernel<GradBf16, false><<<grid, threads, 0, st>>>(in, stat, coef, entropy, dst, stride, seg);
    } else {
        if (entropy) softsync::row_grad_kernel<GradFp32, true><<<grid, threads, 0, st>>>(in, stat, coef, entropy, dst, stride, seg);
        else softsync::row_grad_kernel<GradFp32, false><<<grid, threads, 0, st>>>(in, stat, coef, entropy, dst, stride, seg);
    }
    return launched();
}

// How a row is spread for the kernel that keeps it in registers; vectors == 0: it does not fit.
struct RowShape { int cluster, threads, vectors; };
RowShape row_shape(int64_t n, int64_t rows)
{
    int cluster = 1, most = 512;
    while (cluster < kMaxCluster && n > static_cast<int64_t>(cluster) * 512 * 8) cluster *= 2;
    if (n > static_cast<int64_t>(cluster) * 512 * 8) most = 1024;
    if (n > static_cast<int64_t>(cluster) * most * 8) return {0, 0, 0};
    while (cluster < kMaxCluster && rows * cluster * 2 <= 2 * sm_count() && n > cluster * 512) cluster *= 2;      // few rows
    const int64_t mine = div_up(n, cluster);
    const int64_t threads = most == 1024 ? 1024 : warps(div_up(mine, 4));
    return {cluster, static_cast<int>(threads), static_cast<int>(div_up(mine, threads))};
}

struct PolicyCall {
    RowsIn rows;
    PolicyIn in;
    TermsOut terms;
    float *logp, *entropy;
    unsigned char *out;
    int64_t stride;
};
template <typename GT, bool ENTROPY_GRAD>
int launch_policy_as(const RowShape &sh, const PolicyCall &k, cudaStream_t st)
{
    auto go = [&](auto kernel) {
        return launch_rows(kernel, k.rows.rows, sh.cluster, sh.threads, true, st, k.rows, k.in, k.terms, k.logp, k.entropy, k.out, static_cast<long long>(k.stride));
    };
    switch (sh.vectors) {
    case 1: case 2: return go(softsync::policy_row_kernel<GT, 2, ENTROPY_GRAD>);
    case 3: case 4: return go(softsync::policy_row_kernel<GT, 4, ENTROPY_GRAD>);
    case 5: return go(softsync::policy_row_kernel<GT, 5, ENTROPY_GRAD>);
    case 6: return go(softsync::policy_row_kernel<GT, 6, ENTROPY_GRAD>);
    case 7: return go(softsync::policy_row_kernel<GT, 7, ENTROPY_GRAD>);
    default: return go(softsync::policy_row_kernel<GT, 8, ENTROPY_GRAD>);
    }
}
int launch_policy(int dtype, const RowShape &sh, const PolicyCall &k, cudaStream_t st)
{
    const bool ent = k.in.entropy_coef != 0.f;
    if (dtype == PS_GRAD_BF16) return ent ? launch_policy_as<GradBf16, true>(sh, k, st) : launch_policy_as<GradBf16, false>(sh, k, st);
    return ent ? launch_policy_as<GradFp32, true>(sh, k, st) : launch_policy_as<GradFp32, false>(sh, k, st);
}

}  // namespace

extern "C" {

int ps_loss_workspace(int64_t rows, int64_t sequences, int64_t *bytes)
{
    if (!bytes || rows < 0 || rows > kMaxRows || sequences < 0 || sequences > (int64_t{1} << 31)) return PS_ERR_INVALID_ARG;
    *bytes = Workspace(nullptr, rows, sequences).bytes;
    return PS_OK;
}

int ps_token_logprob(const ps_logits *logits, float *logp_dev, float *lse_dev, float *entropy_dev, void *stream)
{
    const int bad = check_logits(logits);
    if (bad != PS_OK) return bad;
    if (logits->rows == 0) return PS_OK;
    if (!logp_dev || !aligned_to(logp_dev, 4) || !aligned_to(lse_dev, 4) || !aligned_to(entropy_dev, 4)) return PS_ERR_INVALID_ARG;
    return launch_stats(logits, rows_in(logits), StatsOut{logp_dev, lse_dev, entropy_dev, nullptr, nullptr, nullptr}, entropy_dev != nullptr,
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
    const Workspace ws(workspace_dev, logits->rows, 0);
    if (!logp_dev || !in->old_logp_dev || !in->advantages_dev || !workspace_dev || workspace_bytes < ws.bytes ||
        !aligned_to(workspace_dev, 16) || !aligned_to(logp_dev, 4) || !aligned_to(entropy_dev, 4) || !aligned_to(in->old_logp_dev, 4) ||
        !aligned_to(in->advantages_dev, 4) || !aligned_to(in->ref_logp_dev, 4))
        return PS_ERR_INVALID_ARG;
    PolicyCall k;
    k.rows = rows_in(logits);
    k.in = PolicyIn{in->old_logp_dev, in->advantages_dev, in->ref_logp_dev, 1.f - in->clip_low, 1.f + in->clip_high,
                    in->ref_logp_dev ? in->kl_coef : 0.f, in->entropy_coef};
    k.terms = TermsOut{ws.totals, ws.counters, ws.terms, ws.sums, stats_dev};
    k.logp = logp_dev;
    k.entropy = entropy_dev ? entropy_dev : ws.entropy;
    k.out = static_cast<unsigned char *>(dlogits_dev);
    k.stride = dlogits_stride;
    const int64_t groups = div_up(logits->rows, softsync::kRowGroup);
    const RowShape shape = row_shape(row_vectors(logits), logits->rows);
    const bool one_read = shape.vectors != 0;
    if (!one_read &&
        (status = launch_stats(logits, k.rows, StatsOut{logp_dev, nullptr, k.entropy, ws.stat, nullptr, nullptr}, true, st)) != PS_OK)
        return status;
    softsync::policy_totals_kernel<<<1, softsync::kTermThreads, 0, st>>>(logits->weights_dev, logits->rows, ws.totals, ws.counters, static_cast<int>(groups));
    if ((status = launched()) != PS_OK) return status;
    if (one_read) return launch_policy(logits->dtype, shape, k, st);
    softsync::policy_terms_kernel<<<static_cast<unsigned>(div_up(logits->rows, 8)), 256, 0, st>>>(k.rows, k.in, k.terms, logp_dev, k.entropy,
                                                                                                dlogits_dev ? ws.coef : nullptr);
    if ((status = launched()) != PS_OK || !dlogits_dev) return status;
    return launch_grad(logits, k.rows, ws.stat, ws.coef, in->entropy_coef != 0.f ? k.entropy : nullptr, dlogits_dev, dlogits_stride, st);
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
    const Workspace ws(workspace_dev, logits->rows, 2 * in->pairs);
    if (!workspace_dev || workspace_bytes < ws.bytes || !aligned_to(workspace_dev, 16)) return PS_ERR_INVALID_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const RowsIn rows = rows_in(logits);
    const PreferenceIn p{reinterpret_cast<const long long *>(in->offsets_dev), in->ref_logp_dev, in->pairs, in->beta, in->label_smoothing};
    if (logits->rows) status = launch_stats(logits, rows, StatsOut{ws.logp, nullptr, nullptr, ws.stat, ws.coef, ws.counters}, false, st);
    else if (cudaMemsetAsync(ws.counters, 0, sizeof *ws.counters, st) != cudaSuccess) status = PS_ERR_CUDA;
    if (status != PS_OK) return status;
    if (in->pairs) {
        softsync::preference_terms_kernel<<<static_cast<unsigned>(in->pairs), softsync::kPairThreads, 0, st>>>(
            rows, p, ws.logp, seq_logp_dev, dlogits_dev ? ws.coef : nullptr, ws.pairs, ws.counters, stats_dev);
        status = launched();
    } else if (cudaMemsetAsync(stats_dev, 0, 3 * sizeof(float), st) != cudaSuccess) {
        status = PS_ERR_CUDA;
    }
    if (status != PS_OK || !dlogits_dev || !logits->rows) return status;
    return launch_grad(logits, rows, ws.stat, ws.coef, nullptr, dlogits_dev, dlogits_stride, st);
}

}  // extern "C"
