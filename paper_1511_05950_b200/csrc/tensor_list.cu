// Entry points of softsync_learn.h that work on a list of tensors: global gradient norm, AdamW.
#include "../../include/softsync_learn.h"
#include "host_util.h"
#include "tensor_kernels.cuh"

#include <algorithm>
#include <cmath>
#include <cstring>
#include <mutex>
#include <new>
#include <type_traits>
#include <unordered_set>
#include <utility>
#include <vector>

using softsync::AdamwParams;
using softsync::aligned_to;
using softsync::DeviceSwitch;
using softsync::GradBf16;
using softsync::GradFp32;
using softsync::GradTable;
using softsync::kChunk;
using softsync::kListThreads;
using softsync::kStateBlock;
using softsync::ListTables;
using softsync::NormTail;
using softsync::StepTable;
using softsync::TensorRec;

static_assert(kStateBlock == PS_STATE_BLOCK, "the header's block is the kernels'");

namespace {

constexpr int kNormBlocksPerSm = 3;         // one wave: as many as the registers let run at once
constexpr int kNormMaxBlocks = 4096;
// Gradient pointers one launch carries: what fits the 32,764 bytes of its parameters, with a step's coefficients or without, and less.
constexpr int kSmallTable = 32, kMediumTable = 512, kLargeTable = 3840, kLargeStepTable = 1920;

}  // namespace

struct ps_tensors {
    int device = 0, sm_count = 0;
    std::vector<TensorRec> recs;
    int64_t chunks = 0, state_elems = 0;
    TensorRec *recs_dev = nullptr;
    int *chunk_tensor_dev = nullptr;
    double *partial_dev = nullptr;
    unsigned *done_dev = nullptr;
    int state_bits = 0;                   // 0: nothing bound
    void *m = nullptr, *v = nullptr;
    uint8_t *m_scale = nullptr, *v_scale = nullptr;
};

namespace {

std::mutex g_lists_mutex;
std::unordered_set<ps_tensors *> g_lists;

bool is_live(ps_tensors *list)
{
    if (!list) return false;
    std::lock_guard<std::mutex> lock(g_lists_mutex);
    return g_lists.count(list) != 0;
}

#define PS_CATCH_ALL catch (const std::bad_alloc &) { return PS_ERR_NOMEM; } catch (...) { return PS_ERR_INVALID_ARG; }

int64_t round_up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

struct Layout {
    int64_t state_elems = 0, chunks = 0;
    int64_t recs_at = 0, map_at = 0, partial_at = 0, done_at = 0, bytes = 0;   // places in the workspace
};

// False for sizes that are negative or too many.
bool lay_out(int count, const int64_t *sizes, Layout &out)
{
    if (count < 1 || !sizes) return false;
    for (int k = 0; k < count; ++k) {
        if (sizes[k] < 0 || sizes[k] > (int64_t{1} << 44)) return false;
        out.state_elems += round_up(sizes[k], PS_STATE_BLOCK);
        out.chunks += (sizes[k] + kChunk - 1) / kChunk;
        if (out.chunks > 0x7fffffff) return false;
    }
    out.recs_at = 0;
    out.map_at = round_up(static_cast<int64_t>(count) * sizeof(TensorRec), 256);
    out.partial_at = round_up(out.map_at + out.chunks * 4, 256);
    out.done_at = out.partial_at + kNormMaxBlocks * 8;
    out.bytes = out.done_at + 256;
    return true;
}

struct Range { uintptr_t lo, hi; };
bool disjoint(std::vector<Range> &r)
{
    std::sort(r.begin(), r.end(), [](const Range &a, const Range &b) { return a.lo < b.lo; });
    for (size_t k = 1; k < r.size(); ++k)
        if (r[k].lo < r[k - 1].hi) return false;
    return true;
}
Range range_of(const void *p, int64_t bytes) { return {reinterpret_cast<uintptr_t>(p), reinterpret_cast<uintptr_t>(p) + static_cast<uintptr_t>(bytes)}; }

// What is wrong with a call's gradients: PS_OK if nothing.
int check_gradients(const ps_tensors *list, const void *const *grads, int c, const float *scales, int dtype)
{
    if (!grads || c < 1 || c > PS_LIST_MAX_GRADS) return PS_ERR_INVALID_ARG;
    if (dtype != PS_GRAD_FP32 && dtype != PS_GRAD_BF16) return PS_ERR_INVALID_ARG;
    const uintptr_t elem = dtype == PS_GRAD_BF16 ? 2 : 4;
    const size_t n = list->recs.size();
    for (int l = 0; l < c; ++l) {
        if (scales && !std::isfinite(scales[l])) return PS_ERR_INVALID_ARG;
        for (size_t k = 0; k < n; ++k)
            if (list->recs[k].n && (!grads[l * n + k] || !aligned_to(grads[l * n + k], elem))) return PS_ERR_INVALID_ARG;
    }
    return PS_OK;
}

// Calls launch(tables, gradient table) for consecutive ranges of tensors whose gradient pointers fit one launch; coef(tensor) gives a
// step's coefficients.
template <typename Table, typename Coef, typename Launch>
int for_each_range(const ps_tensors *list, const void *const *grads, int c, const float *scales, Coef coef, Launch launch)
{
    const int n = static_cast<int>(list->recs.size());
    const int most = Table::kPointers / c;
    Table tab;
    std::memset(tab.s, 0, sizeof tab.s);
    for (int l = 0; l < c; ++l) tab.s[l] = scales ? scales[l] : 1.f;
    tab.c = c;
    for (int t0 = 0; t0 < n; t0 += most) {
        const int t1 = std::min(n, t0 + most);
        for (int t = t0; t < t1; ++t) {
            for (int l = 0; l < c; ++l) tab.g[(t - t0) * c + l] = grads[static_cast<size_t>(l) * n + t];
            coef(tab, t - t0, list->recs[t]);
        }
        tab.t0 = t0;
        ListTables lt;
        lt.recs = list->recs_dev;
        lt.chunk_tensor = list->chunk_tensor_dev;
        lt.chunk0 = list->recs[t0].first_chunk;
        lt.nchunks = (t1 < n ? list->recs[t1].first_chunk : static_cast<unsigned>(list->chunks)) - lt.chunk0;
        const int status = launch(lt, tab, t0 == 0, t1 == n);
        if (status != PS_OK) return status;
    }
    return PS_OK;
}

// The smallest of three parameter blocks that carries the whole call, else the largest, several times: a launch's cost grows
// with its parameters, which the small lists feel and the large ones do not.
template <template <int> class Table, int LARGE, typename Coef, typename Launch>
int launch_ranges(const ps_tensors *list, const void *const *grads, int c, const float *scales, Coef coef, Launch launch)
{
    const int64_t pointers = static_cast<int64_t>(list->recs.size()) * c;
    if (pointers <= kSmallTable) return for_each_range<Table<kSmallTable>>(list, grads, c, scales, coef, launch);
    if (pointers <= kMediumTable) return for_each_range<Table<kMediumTable>>(list, grads, c, scales, coef, launch);
    return for_each_range<Table<LARGE>>(list, grads, c, scales, coef, launch);
}

uint32_t step_key(uint64_t seed, uint64_t step)          // SplitMix64's finaliser over the seed's step-th place
{
    uint64_t x = seed + step * 0x9E3779B97F4A7C15ull;
    x = (x ^ (x >> 30)) * 0xBF58476D1CE4E5B9ull;
    x = (x ^ (x >> 27)) * 0x94D049BB133111EBull;
    return static_cast<uint32_t>(x ^ (x >> 31));
}

}  // namespace

extern "C" {

int ps_tensors_sizes(int num_tensors, const int64_t *sizes_host, int64_t *state_elems, int64_t *workspace_bytes)
{
    Layout lay;
    if (!lay_out(num_tensors, sizes_host, lay)) return PS_ERR_INVALID_ARG;
    if (state_elems) *state_elems = lay.state_elems;
    if (workspace_bytes) *workspace_bytes = lay.bytes;
    return PS_OK;
}

int ps_tensors_create(ps_tensors_t **out, int num_tensors, const int64_t *sizes_host, void *workspace_dev, int64_t workspace_bytes,
                      void *stream)
{
  try {
    if (!out) return PS_ERR_INVALID_ARG;
    *out = nullptr;
    Layout lay;
    if (!lay_out(num_tensors, sizes_host, lay)) return PS_ERR_INVALID_ARG;
    if (!workspace_dev || !aligned_to(workspace_dev, 16) || workspace_bytes < lay.bytes) return PS_ERR_INVALID_ARG;
    ps_tensors *list = new ps_tensors;
    struct Undo { ps_tensors *p; ~Undo() { delete p; } } undo{list};
    if (cudaGetDevice(&list->device) != cudaSuccess) return PS_ERR_CUDA;
    if (cudaDeviceGetAttribute(&list->sm_count, cudaDevAttrMultiProcessorCount, list->device) != cudaSuccess) return PS_ERR_CUDA;
    list->recs.resize(num_tensors);
    std::vector<int> map(static_cast<size_t>(lay.chunks));
    int64_t chunk = 0, state = 0;
    for (int k = 0; k < num_tensors; ++k) {
        TensorRec &r = list->recs[k];
        r = TensorRec{nullptr, nullptr, sizes_host[k], static_cast<unsigned long long>(state), static_cast<unsigned>(chunk), 0, 1.f, 1.f};
        const int64_t n = (sizes_host[k] + kChunk - 1) / kChunk;
        std::fill(map.begin() + chunk, map.begin() + chunk + n, k);
        chunk += n;
        state += round_up(sizes_host[k], PS_STATE_BLOCK);
    }
    list->chunks = lay.chunks;
    list->state_elems = lay.state_elems;
    char *ws = static_cast<char *>(workspace_dev);
    list->recs_dev = reinterpret_cast<TensorRec *>(ws + lay.recs_at);
    list->chunk_tensor_dev = reinterpret_cast<int *>(ws + lay.map_at);
    list->partial_dev = reinterpret_cast<double *>(ws + lay.partial_at);
    list->done_dev = reinterpret_cast<unsigned *>(ws + lay.done_at);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (cudaMemcpyAsync(list->recs_dev, list->recs.data(), list->recs.size() * sizeof(TensorRec), cudaMemcpyHostToDevice, st) != cudaSuccess ||
        (!map.empty() && cudaMemcpyAsync(list->chunk_tensor_dev, map.data(), map.size() * 4, cudaMemcpyHostToDevice, st) != cudaSuccess) ||
        cudaMemsetAsync(list->done_dev, 0, 256, st) != cudaSuccess || cudaStreamSynchronize(st) != cudaSuccess)
        return PS_ERR_CUDA;
    {
        std::lock_guard<std::mutex> lock(g_lists_mutex);
        g_lists.insert(list);
    }
    undo.p = nullptr;
    *out = list;
    return PS_OK;
  } PS_CATCH_ALL
}

int ps_tensors_destroy(ps_tensors_t *list)
{
  try {
    std::lock_guard<std::mutex> lock(g_lists_mutex);
    if (!list || !g_lists.erase(list)) return PS_ERR_INVALID_ARG;
    delete list;
    return PS_OK;
  } PS_CATCH_ALL
}

int ps_tensors_bind_adamw(ps_tensors_t *list, float *const *weights_host, void *const *mirrors_host,
                          const float *lr_mult_host, const float *decay_mult_host, int state_bits,
                          void *m_dev, void *v_dev, uint8_t *m_scale_dev, uint8_t *v_scale_dev, void *stream)
{
  try {
    if (!is_live(list) || !weights_host || (state_bits != 32 && state_bits != 8)) return PS_ERR_INVALID_ARG;
    if (!aligned_to(m_dev, 16) || !aligned_to(v_dev, 16)) return PS_ERR_INVALID_ARG;
    if (list->state_elems && (!m_dev || !v_dev || (state_bits == 8 && (!m_scale_dev || !v_scale_dev)))) return PS_ERR_INVALID_ARG;
    std::vector<Range> ranges;
    const int64_t state_bytes = list->state_elems * (state_bits / 8);
    ranges.push_back(range_of(m_dev, state_bytes));
    ranges.push_back(range_of(v_dev, state_bytes));
    if (state_bits == 8) {
        ranges.push_back(range_of(m_scale_dev, list->state_elems / PS_STATE_BLOCK));
        ranges.push_back(range_of(v_scale_dev, list->state_elems / PS_STATE_BLOCK));
    }
    std::vector<TensorRec> recs = list->recs;
    for (size_t k = 0; k < recs.size(); ++k) {
        TensorRec &r = recs[k];
        r.w = weights_host[k];
        r.mirror = mirrors_host ? static_cast<unsigned short *>(mirrors_host[k]) : nullptr;
        r.lr_mult = lr_mult_host ? lr_mult_host[k] : 1.f;
        r.decay_mult = decay_mult_host ? decay_mult_host[k] : 1.f;
        r.on_grid = aligned_to(r.w, 16) && aligned_to(r.mirror, 8);
        if (!std::isfinite(r.lr_mult) || !std::isfinite(r.decay_mult)) return PS_ERR_INVALID_ARG;
        if (!r.n) continue;
        if (!r.w || !aligned_to(r.w, 4) || !aligned_to(r.mirror, 2)) return PS_ERR_INVALID_ARG;
        ranges.push_back(range_of(r.w, r.n * 4));
        if (r.mirror) ranges.push_back(range_of(r.mirror, r.n * 2));
    }
    if (!disjoint(ranges)) return PS_ERR_INVALID_ARG;
    DeviceSwitch guard(list->device);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (cudaMemcpyAsync(list->recs_dev, recs.data(), recs.size() * sizeof(TensorRec), cudaMemcpyHostToDevice, st) != cudaSuccess ||
        cudaStreamSynchronize(st) != cudaSuccess)
        return PS_ERR_CUDA;
    list->recs.swap(recs);
    list->state_bits = state_bits;
    list->m = m_dev; list->v = v_dev; list->m_scale = m_scale_dev; list->v_scale = v_scale_dev;
    return PS_OK;
  } PS_CATCH_ALL
}

int ps_grad_norm(ps_tensors_t *list, const void *const *grads_host, int c, const float *scales_host, int grad_dtype,
                 float max_norm, float *out_dev, void *stream)
{
  try {
    if (!is_live(list) || !out_dev || !aligned_to(out_dev, 4) || !(max_norm > 0.f)) return PS_ERR_INVALID_ARG;
    const int bad = check_gradients(list, grads_host, c, scales_host, grad_dtype);
    if (bad != PS_OK) return bad;
    DeviceSwitch guard(list->device);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const int grid = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>({list->chunks, static_cast<int64_t>(kNormBlocksPerSm) * list->sm_count, kNormMaxBlocks})));
    const auto none = [](auto &, int, const TensorRec &) {};
    return launch_ranges<GradTable, kLargeTable>(list, grads_host, c, scales_host, none, [&](const ListTables &lt, const auto &tab, bool first, bool last) {
        constexpr int MAXP = std::decay_t<decltype(tab)>::kPointers;
        const NormTail tail{list->partial_dev, list->done_dev, out_dev, max_norm, first ? 0 : 1, last ? 1 : 0};
        const auto go = [&](auto kernel) { kernel<<<grid, softsync::kNormThreads, 0, st>>>(lt, tab, tail); };
        if (grad_dtype == PS_GRAD_BF16) c == 1 ? go(softsync::grad_norm_kernel<GradBf16, true, MAXP>) : go(softsync::grad_norm_kernel<GradBf16, false, MAXP>);
        else c == 1 ? go(softsync::grad_norm_kernel<GradFp32, true, MAXP>) : go(softsync::grad_norm_kernel<GradFp32, false, MAXP>);
        return cudaGetLastError() == cudaSuccess ? PS_OK : PS_ERR_CUDA;
    });
  } PS_CATCH_ALL
}

int ps_adamw_check(const ps_adamw_config *config)
{
    if (!config) return PS_ERR_INVALID_ARG;
    const ps_adamw_config &k = *config;
    if (!std::isfinite(k.lr) || k.lr < 0 || !(k.beta1 >= 0 && k.beta1 < 1) || !(k.beta2 >= 0 && k.beta2 < 1)) return PS_ERR_INVALID_ARG;
    if (!std::isfinite(k.eps) || k.eps < 0 || !std::isfinite(k.weight_decay) || k.step < 1) return PS_ERR_INVALID_ARG;
    return PS_OK;
}

int ps_adamw_step(ps_tensors_t *list, const void *const *grads_host, int c, const float *scales_host, int grad_dtype,
                  const ps_adamw_config *config, const float *clip_dev, void *stream)
{
  try {
    if (!is_live(list) || !config) return PS_ERR_INVALID_ARG;
    if (!list->state_bits) return PS_ERR_NO_STATE;
    const ps_adamw_config &k = *config;
    int bad = ps_adamw_check(config);
    if (bad == PS_OK && !aligned_to(clip_dev, 4)) bad = PS_ERR_INVALID_ARG;
    if (bad == PS_OK) bad = check_gradients(list, grads_host, c, scales_host, grad_dtype);
    if (bad != PS_OK) return bad;
    const double t = static_cast<double>(k.step);
    AdamwParams p;
    p.m = list->m; p.v = list->v; p.m_scale = list->m_scale; p.v_scale = list->v_scale;
    p.clip = clip_dev;
    const double lr_decay = k.lr * k.weight_decay, step_size = k.lr / (1.0 - std::pow(k.beta1, t));
    const auto twice = [](double x) { return make_float2(static_cast<float>(x), static_cast<float>(x)); };
    p.beta1 = twice(k.beta1);
    p.one_minus_beta1 = twice(1.0 - k.beta1);
    p.beta2 = twice(k.beta2);
    p.one_minus_beta2 = twice(1.0 - k.beta2);
    p.root_scale = static_cast<float>(1.0 / std::sqrt(1.0 - std::pow(k.beta2, t)));
    p.eps = static_cast<float>(k.eps);
    p.short_forms = p.eps >= 0x1p-40f && p.root_scale <= 0x1p10f;
    p.key = step_key(k.seed, static_cast<uint64_t>(k.step));
    DeviceSwitch guard(list->device);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const auto coef = [&](auto &tab, int i, const TensorRec &r) {
        tab.coef[i] = make_float2(static_cast<float>(1.0 - lr_decay * (static_cast<double>(r.lr_mult) * r.decay_mult)), static_cast<float>(step_size * r.lr_mult));
    };
    return launch_ranges<StepTable, kLargeStepTable>(list, grads_host, c, scales_host, coef, [&](const ListTables &lt, const auto &tab, bool, bool) {
        constexpr int MAXP = std::decay_t<decltype(tab)>::kPointers;
        if (lt.nchunks == 0) return static_cast<int>(PS_OK);
        const auto go = [&](auto kernel) { kernel<<<lt.nchunks, kListThreads, 0, st>>>(lt, tab, p); };
        const auto with = [&](auto grad, auto bits) {
            using GT = decltype(grad);
            if (c == 1) go(softsync::adamw_kernel<GT, decltype(bits)::value, true, MAXP>);
            else go(softsync::adamw_kernel<GT, decltype(bits)::value, false, MAXP>);
        };
        using Bits8 = std::integral_constant<int, 8>;
        using Bits32 = std::integral_constant<int, 32>;
        if (list->state_bits == 32) grad_dtype == PS_GRAD_BF16 ? with(GradBf16{}, Bits32{}) : with(GradFp32{}, Bits32{});
        else grad_dtype == PS_GRAD_BF16 ? with(GradBf16{}, Bits8{}) : with(GradFp32{}, Bits8{});
        return cudaGetLastError() == cudaSuccess ? static_cast<int>(PS_OK) : static_cast<int>(PS_ERR_CUDA);
    });
  } PS_CATCH_ALL
}

int ps_adamw_moments(ps_tensors_t *list, void *m_bf16_dev, void *v_bf16_dev, void *stream)
{
  try {
    if (!is_live(list)) return PS_ERR_INVALID_ARG;
    if (list->state_bits != 8) return PS_ERR_NO_STATE;
    const int64_t eights = list->state_elems / 8;
    if (!eights) return PS_OK;
    if (!m_bf16_dev || !v_bf16_dev || m_bf16_dev == v_bf16_dev || !aligned_to(m_bf16_dev, 16) || !aligned_to(v_bf16_dev, 16)) return PS_ERR_INVALID_ARG;
    if ((eights + 255) / 256 > 0x7fffffff) return PS_ERR_INVALID_ARG;
    DeviceSwitch guard(list->device);
    softsync::moments_kernel<<<static_cast<unsigned>((eights + 255) / 256), 256, 0, static_cast<cudaStream_t>(stream)>>>(
        static_cast<const uint2 *>(list->m), static_cast<const uint2 *>(list->v), list->m_scale, list->v_scale,
        static_cast<uint4 *>(m_bf16_dev), static_cast<uint4 *>(v_bf16_dev), eights);
    return cudaGetLastError() == cudaSuccess ? PS_OK : PS_ERR_CUDA;
  } PS_CATCH_ALL
}

}  // extern "C"
