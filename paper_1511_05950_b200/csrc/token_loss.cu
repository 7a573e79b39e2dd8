// Entry points of softsync_learn.h that work on rows of logits: token log probabilities, policy loss, preference loss.
#include "../../include/softsync_learn.h"
#include "host_util.h"
#include "token_kernels.cuh"

#include <cmath>

using softsync::aligned_to;
using softsync::GradBf16;
using softsync::GradFp32;
using softsync::PolicyIn;
using softsync::PreferenceIn;
using softsync::RowCoef;
using softsync::RowsIn;
using softsync::RowStat;

namespace {

int64_t round_up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

// Places in the losses' workspace.
struct Workspace {
    RowStat *stat;
    RowCoef *coef;
    float *entropy, *logp;
    static int64_t bytes(int64_t rows) { return round_up(rows * 8, 256) * 2 + round_up(rows * 4, 256) * 2 + 256; }
    Workspace(void *p, int64_t rows)
    {
        char *at = static_cast<char *>(p);
        stat = reinterpret_cast<RowStat *>(at); at += round_up(rows * 8, 256);
        coef = reinterpret_cast<RowCoef *>(at); at += round_up(rows * 8, 256);
        entropy = reinterpret_cast<float *>(at); at += round_up(rows * 4, 256);
        logp = reinterpret_cast<float *>(at);
    }
};

constexpr int64_t kMaxRows = 0x7fffffff;

int check_logits(const ps_logits *lg)
{
    if (!lg || (lg->dtype != PS_GRAD_FP32 && lg->dtype != PS_GRAD_BF16)) return PS_ERR_INVALID_ARG;
    if (lg->rows < 0 || lg->rows > kMaxRows || lg->vocab < 1 || lg->vocab > (int64_t{1} << 31) || lg->row_stride < lg->vocab) return PS_ERR_INVALID_ARG;
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

int launch_stats(const ps_logits *lg, const RowsIn &in, float *logp, float *lse, float *entropy, RowStat *stat, cudaStream_t st)
{
    const unsigned grid = static_cast<unsigned>(lg->rows);
    if (lg->dtype == PS_GRAD_BF16) softsync::row_stats_kernel<GradBf16><<<grid, 512, 0, st>>>(in, logp, lse, entropy, stat);
    else softsync::row_stats_kernel<GradFp32><<<grid, 512, 0, st>>>(in, logp, lse, entropy, stat);
    return launched();
}

int launch_grad(const ps_logits *lg, const RowsIn &in, const RowStat *stat, const RowCoef *coef, const float *entropy, void *out,
                int64_t stride, cudaStream_t st)
{
    const unsigned grid = static_cast<unsigned>(lg->rows);
    unsigned char *dst = static_cast<unsigned char *>(out);
    if (lg->dtype == PS_GRAD_BF16) softsync::row_grad_kernel<GradBf16><<<grid, 512, 0, st>>>(in, stat, coef, entropy, dst, stride);
    else softsync::row_grad_kernel<GradFp32><<<grid, 512, 0, st>>>(in, stat, coef, entropy, dst, stride);
    return launched();
}

}  // namespace

extern "C" {

int ps_loss_workspace(int64_t rows, int64_t sequences, int64_t *bytes)
{
    if (!bytes || rows < 0 || rows > kMaxRows || sequences < 0) return PS_ERR_INVALID_ARG;
    *bytes = Workspace::bytes(rows);
    return PS_OK;
}

int ps_token_logprob(const ps_logits *logits, float *logp_dev, float *lse_dev, float *entropy_dev, void *stream)
{
    const int bad = check_logits(logits);
    if (bad != PS_OK) return bad;
    if (logits->rows == 0) return PS_OK;
    if (!logp_dev || !aligned_to(logp_dev, 4) || !aligned_to(lse_dev, 4) || !aligned_to(entropy_dev, 4)) return PS_ERR_INVALID_ARG;
    return launch_stats(logits, rows_in(logits), logp_dev, lse_dev, entropy_dev, nullptr, static_cast<cudaStream_t>(stream));
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
    if (!logp_dev || !in->old_logp_dev || !in->advantages_dev || !workspace_dev || workspace_bytes < Workspace::bytes(logits->rows) ||
        !aligned_to(workspace_dev, 16) || !aligned_to(logp_dev, 4) || !aligned_to(entropy_dev, 4) || !aligned_to(in->old_logp_dev, 4) ||
        !aligned_to(in->advantages_dev, 4) || !aligned_to(in->ref_logp_dev, 4))
        return PS_ERR_INVALID_ARG;
    const Workspace ws(workspace_dev, logits->rows);
    const RowsIn rows = rows_in(logits);
    float *entropy = entropy_dev ? entropy_dev : ws.entropy;
    const PolicyIn p{in->old_logp_dev, in->advantages_dev, in->ref_logp_dev, 1.f - in->clip_low, 1.f + in->clip_high,
                     in->ref_logp_dev ? in->kl_coef : 0.f, in->entropy_coef};
    if ((status = launch_stats(logits, rows, logp_dev, nullptr, entropy, ws.stat, st)) != PS_OK) return status;
    softsync::policy_terms_kernel<<<1, softsync::kTermThreads, 0, st>>>(rows, p, logp_dev, entropy, dlogits_dev ? ws.coef : nullptr, stats_dev);
    if ((status = launched()) != PS_OK || !dlogits_dev) return status;
    return launch_grad(logits, rows, ws.stat, ws.coef, entropy, dlogits_dev, dlogits_stride, st);
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
    if (logits->rows && (!workspace_dev || workspace_bytes < Workspace::bytes(logits->rows) || !aligned_to(workspace_dev, 16))) return PS_ERR_INVALID_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const Workspace ws(workspace_dev, logits->rows);
    const RowsIn rows = rows_in(logits);
    const PreferenceIn p{reinterpret_cast<const long long *>(in->offsets_dev), in->ref_logp_dev, in->pairs, in->beta, in->label_smoothing};
    if (logits->rows) {
        if ((status = launch_stats(logits, rows, ws.logp, nullptr, nullptr, ws.stat, st)) != PS_OK) return status;
        if (dlogits_dev && cudaMemsetAsync(ws.coef, 0, static_cast<size_t>(logits->rows) * sizeof(RowCoef), st) != cudaSuccess) return PS_ERR_CUDA;
    }
    softsync::preference_terms_kernel<<<1, softsync::kTermThreads, 0, st>>>(rows, p, ws.logp, seq_logp_dev, dlogits_dev && logits->rows ? ws.coef : nullptr, stats_dev);
    if ((status = launched()) != PS_OK || !dlogits_dev || !logits->rows) return status;
    return launch_grad(logits, rows, ws.stat, ws.coef, nullptr, dlogits_dev, dlogits_stride, st);
}

}  // extern "C"
