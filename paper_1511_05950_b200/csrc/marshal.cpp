// Argument checks, output tensors and workspaces of the calls in learn.py, as a CPython extension over torch's C++ tensors: what a
// call costs on the host is most of what a short one takes.  The work is done by the entry points of softsync_learn.h, whose
// addresses learn.py hands over once (bind); a call returns their status for learn.py to raise.
#include "../../include/softsync_learn.h"

#include <Python.h>
#include <ATen/ATen.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <map>
#include <tuple>

namespace {

decltype(&ps_loss_workspace) loss_workspace;
decltype(&ps_token_logprob) call_token_logprob;
decltype(&ps_policy_loss) call_policy_loss;
decltype(&ps_preference_loss) call_preference_loss;
decltype(&ps_head_workspace) head_workspace;
decltype(&ps_head_logprob) call_head_logprob;
decltype(&ps_head_logprob_grad) call_head_logprob_grad;
decltype(&ps_head_cross_entropy) call_head_cross_entropy;
decltype(&ps_pack8) call_pack8;
decltype(&ps_unpack8) call_unpack8;
decltype(&ps_rms_norm) call_rms_norm;
decltype(&ps_norm_grad_workspace) norm_grad_workspace;
decltype(&ps_rms_norm_grad) call_rms_norm_grad;
decltype(&ps_packed_grad_workspace) packed_grad_workspace;
decltype(&ps_packed_weight_grad) call_packed_weight_grad;

const at::Tensor &tensor_of(PyObject *o, const char *what)
{
    TORCH_CHECK_TYPE(THPVariable_Check(o), what, " must be a tensor, got ", Py_TYPE(o)->tp_name);
    return THPVariable_Unpack(o);
}

int grad_dtype(at::ScalarType t) { return t == at::kFloat ? PS_GRAD_FP32 : t == at::kBFloat16 ? PS_GRAD_BF16 : -1; }

// One value for each of `count` rows, on the logits' GPU; null for None where that is allowed.
template <typename T>
const T *per_row(PyObject *o, int64_t count, const char *what, const at::Tensor &logits, bool optional = false)
{
    if (optional && o == Py_None) return nullptr;
    const at::Tensor &t = tensor_of(o, what);
    constexpr at::ScalarType want = std::is_same_v<T, float> ? at::kFloat : at::kLong;
    TORCH_CHECK_TYPE(t.scalar_type() == want, what, " must be ", want, ", got ", t.scalar_type());
    TORCH_CHECK_VALUE(t.dim() == 1 && t.numel() == count && t.is_contiguous(), what, ": ", count, " values one behind the other, got shape ", t.sizes(),
                      " with strides ", t.strides());
    TORCH_CHECK_VALUE(t.device() == logits.device(), what, " is on ", t.device(), ", the logits on ", logits.device());
    return static_cast<const T *>(t.const_data_ptr());
}

double number(PyObject *o)
{
    const double x = PyFloat_AsDouble(o);
    if (x == -1.0 && PyErr_Occurred()) throw python_error();
    return x;
}

struct Logits {
    const at::Tensor &t;
    ps_logits c;
    Logits(PyObject *logits, PyObject *tokens, PyObject *weights, PyObject *temperature) : t(tensor_of(logits, "logits"))
    {
        const int dtype = grad_dtype(t.scalar_type());
        TORCH_CHECK_TYPE(dtype >= 0, "logits must be fp32 or bf16, got ", t.scalar_type());
        TORCH_CHECK_VALUE(t.dim() == 2 && (t.stride(1) == 1 || t.size(1) <= 1), "logits must be rows x vocabulary with the vocabulary contiguous");
        TORCH_CHECK_VALUE(t.is_cuda(), "logits must live on the GPU");
        const int64_t rows = t.size(0), vocab = t.size(1);
        c.data_dev = t.const_data_ptr();
        c.dtype = dtype;
        c.rows = rows;
        c.vocab = vocab;
        c.row_stride = rows > 1 ? t.stride(0) : std::max<int64_t>(vocab, 1);
        c.tokens_dev = per_row<int64_t>(tokens, rows, "tokens", t);
        c.weights_dev = per_row<float>(weights, rows, "weights", t, true);
        c.temperature = static_cast<float>(number(temperature));
    }
    at::Tensor floats(int64_t n) const { return at::empty({n}, t.options().dtype(at::kFloat)); }
};

// Tells autograd that a tensor's values have changed: a backward pass that saved it then raises instead of using the new ones.
void changed(const at::Tensor &t)
{
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

// Where the gradient goes: True (a new tensor), False or None (nowhere), "inplace" (over the logits) or a tensor.
struct Gradient {
    at::Tensor t;
    void *data = nullptr;
    int64_t stride = 0;
    bool given = false;                   // written over values that somebody may have saved
    Gradient(PyObject *grad, const Logits &lg)
    {
        if (grad == Py_False || grad == Py_None) return;
        if (grad == Py_True) {
            t = at::empty(lg.t.sizes(), lg.t.options());
        } else {
            given = true;
            if (PyUnicode_Check(grad)) {
                TORCH_CHECK_VALUE(PyUnicode_CompareWithASCIIString(grad, "inplace") == 0, "grad is True, False, 'inplace' or a tensor");
                t = lg.t.detach();
            } else {
                t = tensor_of(grad, "grad");
            }
            TORCH_CHECK_VALUE(t.sizes() == lg.t.sizes() && t.scalar_type() == lg.t.scalar_type() && t.device() == lg.t.device() && (t.stride(1) == 1 || t.size(1) <= 1),
                              "the gradient's buffer must have the logits' shape, type and device, with the vocabulary contiguous");
        }
        data = t.data_ptr();
        stride = t.size(0) > 1 ? t.stride(0) : std::max<int64_t>(t.size(1), 1);
    }
    void written(int status) const { if (given && status == PS_OK) changed(t); }
};

// A workspace for one call on this stream.  Calls on one stream follow one another, whichever thread makes them (each holds the interpreter's
// lock from here to its last launch), and share theirs, which keeps what the library asks of it (a zero at its front) from call to call; a
// captured graph gets its own.  A program that keeps making streams gets new ones now and then: what is given up goes back to
// its stream's part of the allocator, behind the work that uses it.
at::Tensor workspace(int64_t rows, int64_t sequences, const at::Tensor &like, cudaStream_t stream)
{
    constexpr size_t most = 128;          // torch's own pools have 64 streams a GPU
    static auto *kept = new std::map<std::tuple<int, cudaStream_t>, at::Tensor>;      // never destroyed: CUDA goes first at exit
    int64_t need = 0;
    TORCH_CHECK_VALUE(loss_workspace(rows, sequences, &need) == PS_OK, "too many rows or sequences");
    cudaStreamCaptureStatus capture = cudaStreamCaptureStatusNone;
    C10_CUDA_CHECK(cudaStreamIsCapturing(stream, &capture));
    const auto fresh = [&] { return at::zeros({std::max<int64_t>(need, 1 << 16)}, like.options().dtype(at::kByte)); };
    if (capture != cudaStreamCaptureStatusNone) return fresh();
    const std::tuple<int, cudaStream_t> key{like.get_device(), stream};
    if (kept->size() >= most && !kept->count(key)) kept->clear();
    at::Tensor &ws = (*kept)[key];
    if (!ws.defined() || ws.numel() < need) ws = fresh();
    return ws;
}

PyObject *result(int status, std::initializer_list<at::Tensor> tensors)
{
    PyObject *out = PyTuple_New(1 + static_cast<Py_ssize_t>(tensors.size()));
    if (!out) throw python_error();
    PyTuple_SET_ITEM(out, 0, PyLong_FromLong(status));
    Py_ssize_t k = 1;
    for (const at::Tensor &t : tensors) PyTuple_SET_ITEM(out, k++, t.defined() ? THPVariable_Wrap(t) : (Py_INCREF(Py_None), Py_None));
    return out;
}

void expect(Py_ssize_t got, Py_ssize_t want) { TORCH_CHECK_TYPE(got == want, "expected ", want, " arguments, got ", got); }

// (addresses of the entry points, in the order of this list)
PyObject *bind(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    expect(n, 15);
    Py_ssize_t k = 0;
    const auto take = [&](auto &f) {
        void *p = PyLong_AsVoidPtr(a[k++]);
        if (!p) throw python_error();
        f = reinterpret_cast<std::remove_reference_t<decltype(f)>>(p);
    };
    take(loss_workspace); take(call_token_logprob); take(call_policy_loss); take(call_preference_loss);
    take(head_workspace); take(call_head_logprob); take(call_head_logprob_grad); take(call_head_cross_entropy);
    take(call_pack8); take(call_unpack8); take(call_rms_norm); take(norm_grad_workspace); take(call_rms_norm_grad);
    take(packed_grad_workspace); take(call_packed_weight_grad);
    Py_RETURN_NONE;
    END_HANDLE_TH_ERRORS
}

// (logits, tokens, weights, temperature) -> (status, logp, lse, entropy)
PyObject *token_logprob(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    expect(n, 4);
    const Logits lg(a[0], a[1], a[2], a[3]);
    const c10::cuda::CUDAGuard guard(lg.t.device());
    const at::Tensor logp = lg.floats(lg.c.rows), lse = lg.floats(lg.c.rows), entropy = lg.floats(lg.c.rows);
    const int status = call_token_logprob(&lg.c, static_cast<float *>(logp.data_ptr()), static_cast<float *>(lse.data_ptr()), static_cast<float *>(entropy.data_ptr()),
                                          c10::cuda::getCurrentCUDAStream().stream());
    return result(status, {logp, lse, entropy});
    END_HANDLE_TH_ERRORS
}

// (logits, tokens, weights, temperature, old_logp, advantages, ref_logp, clip_low, clip_high, kl_coef, entropy_coef, grad)
// -> (status, stats, logp, entropy, dlogits)
PyObject *policy_loss(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    expect(n, 12);
    const Logits lg(a[0], a[1], a[2], a[3]);
    ps_policy_inputs in;
    in.old_logp_dev = per_row<float>(a[4], lg.c.rows, "old_logp", lg.t);
    in.advantages_dev = per_row<float>(a[5], lg.c.rows, "advantages", lg.t);
    in.ref_logp_dev = per_row<float>(a[6], lg.c.rows, "ref_logp", lg.t, true);
    in.clip_low = static_cast<float>(number(a[7]));
    in.clip_high = static_cast<float>(number(a[8]));
    in.kl_coef = static_cast<float>(number(a[9]));
    in.entropy_coef = static_cast<float>(number(a[10]));
    const c10::cuda::CUDAGuard guard(lg.t.device());
    const Gradient grad(a[11], lg);
    const at::Tensor stats = lg.floats(5), logp = lg.floats(lg.c.rows), entropy = lg.floats(lg.c.rows);
    const cudaStream_t stream = c10::cuda::getCurrentCUDAStream().stream();
    const at::Tensor ws = workspace(lg.c.rows, 0, lg.t, stream);
    const int status = call_policy_loss(&lg.c, &in, static_cast<float *>(stats.data_ptr()), static_cast<float *>(logp.data_ptr()),
                                        static_cast<float *>(entropy.data_ptr()), grad.data, grad.stride, ws.data_ptr(), ws.numel(), stream);
    grad.written(status);
    return result(status, {stats, logp, entropy, grad.t});
    END_HANDLE_TH_ERRORS
}

// (logits, tokens, weights, temperature, offsets, ref_logp, beta, label_smoothing, grad) -> (status, stats, seq_logp, dlogits)
PyObject *preference_loss(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    expect(n, 9);
    const Logits lg(a[0], a[1], a[2], a[3]);
    const at::Tensor &offsets = tensor_of(a[4], "offsets");
    TORCH_CHECK_VALUE(offsets.dim() == 1 && offsets.numel() % 2 == 1, "offsets holds 2 * pairs + 1 row numbers");
    const int64_t sequences = offsets.numel() - 1;
    ps_preference_inputs in;
    in.offsets_dev = per_row<int64_t>(a[4], sequences + 1, "offsets", lg.t);
    in.ref_logp_dev = per_row<float>(a[5], sequences, "ref_logp", lg.t);
    in.pairs = sequences / 2;
    in.beta = static_cast<float>(number(a[6]));
    in.label_smoothing = static_cast<float>(number(a[7]));
    const c10::cuda::CUDAGuard guard(lg.t.device());
    const Gradient grad(a[8], lg);
    const at::Tensor stats = lg.floats(3), seq_logp = lg.floats(sequences);
    const cudaStream_t stream = c10::cuda::getCurrentCUDAStream().stream();
    const at::Tensor ws = workspace(lg.c.rows, sequences, lg.t, stream);
    const int status = call_preference_loss(&lg.c, &in, static_cast<float *>(stats.data_ptr()), static_cast<float *>(seq_logp.data_ptr()), grad.data, grad.stride,
                                            ws.data_ptr(), ws.numel(), stream);
    grad.written(status);
    return result(status, {stats, seq_logp, grad.t});
    END_HANDLE_TH_ERRORS
}

struct Fast {                             // a list or tuple, whatever sequence was given
    PyObject *o;
    Fast(PyObject *seq, const char *what) : o(PySequence_Fast(seq, what)) { if (!o) throw python_error(); }
    ~Fast() { Py_DECREF(o); }
    Fast(const Fast &) = delete;
    Py_ssize_t size() const { return PySequence_Fast_GET_SIZE(o); }
    PyObject *operator[](Py_ssize_t k) const { return PySequence_Fast_GET_ITEM(o, k); }
};

// (gradients, address of the list's sizes, tensors in the list, device index, address of c * tensors pointers to fill, c)
// -> ps_grad_dtype.  gradients: c sequences of one contiguous tensor for each tensor of the list.
PyObject *gradients(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    expect(n, 6);
    const auto *sizes = static_cast<const int64_t *>(PyLong_AsVoidPtr(a[1]));
    const Py_ssize_t tensors = PyLong_AsSsize_t(a[2]);
    const long device = PyLong_AsLong(a[3]);
    auto **out = static_cast<const void **>(PyLong_AsVoidPtr(a[4]));
    const Py_ssize_t c = PyLong_AsSsize_t(a[5]);
    if (PyErr_Occurred()) throw python_error();
    const Fast grads(a[0], "gradients must be a sequence of sequences of tensors");
    TORCH_CHECK_VALUE(grads.size() == c, "expected ", c, " gradients, got ", grads.size());
    int dtype = -1;
    for (Py_ssize_t l = 0; l < c; ++l) {
        const Fast row(grads[l], "a gradient must be a sequence of tensors");
        TORCH_CHECK_VALUE(row.size() == tensors, "a gradient has ", row.size(), " tensors, the list ", tensors);
        for (Py_ssize_t k = 0; k < tensors; ++k) {
            const at::Tensor &g = tensor_of(row[k], "a gradient's tensor");
            const int d = grad_dtype(g.scalar_type());
            TORCH_CHECK_TYPE(d >= 0 && (dtype < 0 || d == dtype), "gradients must all be fp32 or all bf16");
            dtype = d;
            TORCH_CHECK_VALUE(g.numel() == sizes[k] && g.is_contiguous(), "gradient tensor ", k, " must be contiguous with ", sizes[k], " elements");
            TORCH_CHECK_VALUE(g.is_cuda() && g.get_device() == device, "gradient tensor ", k, " is on ", g.device(), ", the list on GPU ", device);
            out[l * tensors + k] = g.const_data_ptr();
        }
    }
    return PyLong_FromLong(dtype);
    END_HANDLE_TH_ERRORS
}

// (sequence of tensors): all of them have been written to
PyObject *written(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    expect(n, 1);
    const Fast tensors(a[0], "a sequence of tensors");
    for (Py_ssize_t k = 0; k < tensors.size(); ++k) changed(tensor_of(tensors[k], "a written tensor"));
    Py_RETURN_NONE;
    END_HANDLE_TH_ERRORS
}

// ---- losses without logits, norm, activations in 8 bits ----------------------------------------------------------------------
// A new tensor on the GPU of another one, past the dispatcher (a third of its time, and a call of the norm makes five).
at::Tensor fresh(at::IntArrayRef sizes, at::ScalarType type, const at::Tensor &like) { return at::detail::empty_cuda(sizes, type, like.device(), std::nullopt); }
bool rows_fine(const at::Tensor &t) { return t.dim() == 2 && (t.stride(1) == 1 || t.size(1) <= 1 || t.size(0) == 0); }       // without rows any strides will do
int64_t row_stride(const at::Tensor &t) { return t.size(0) > 1 ? t.stride(0) : std::max<int64_t>(t.size(1), 1); }
template <typename T> T *data(const at::Tensor &t) { return t.defined() ? static_cast<T *>(t.data_ptr()) : nullptr; }
template <typename T> const T *const_data(const at::Tensor &t) { return t.defined() ? static_cast<const T *>(t.const_data_ptr()) : nullptr; }
at::Tensor scratch(int64_t bytes, const at::Tensor &like) { return fresh({std::max<int64_t>(bytes, 16)}, at::kByte, like); }

// Rows of activations on the GPU, fp32 or bf16.
const at::Tensor &rows_of(PyObject *o, const char *what)
{
    const at::Tensor &t = tensor_of(o, what);
    TORCH_CHECK_TYPE(grad_dtype(t.scalar_type()) >= 0, what, " must be fp32 or bf16, got ", t.scalar_type());
    TORCH_CHECK_VALUE(rows_fine(t), what, " must be rows x columns with the columns contiguous");
    TORCH_CHECK_VALUE(t.is_cuda(), what, " must live on the GPU");
    return t;
}
// Rows of the same shape, type and GPU; undefined for None.
at::Tensor rows_like(PyObject *o, const char *what, const at::Tensor &like)
{
    if (o == Py_None) return at::Tensor();
    const at::Tensor &t = tensor_of(o, what);
    TORCH_CHECK_TYPE(t.scalar_type() == like.scalar_type(), what, " must be ", like.scalar_type(), ", got ", t.scalar_type());
    TORCH_CHECK_VALUE(rows_fine(t) && t.sizes() == like.sizes(), what, " must be ", like.size(0), " x ", like.size(1), " with the columns contiguous, got shape ", t.sizes(),
                      " with strides ", t.strides());
    TORCH_CHECK_VALUE(t.device() == like.device(), what, " is on ", t.device(), ", expected ", like.device());
    return t;
}
// A factor for each column; undefined for None.
at::Tensor gain_of(PyObject *o, int64_t cols, const at::Tensor &like)
{
    if (o == Py_None) return at::Tensor();
    const at::Tensor &t = tensor_of(o, "gain");
    TORCH_CHECK_TYPE(grad_dtype(t.scalar_type()) >= 0, "gain must be fp32 or bf16, got ", t.scalar_type());
    TORCH_CHECK_VALUE(t.dim() == 1 && t.numel() == cols && t.is_contiguous(), "gain: ", cols, " values one behind the other, got shape ", t.sizes(), " with strides ", t.strides());
    TORCH_CHECK_VALUE(t.device() == like.device(), "gain is on ", t.device(), ", expected ", like.device());
    return t;
}

int64_t padded(int64_t cols) { return (cols + PS_PACK_BLOCK - 1) / PS_PACK_BLOCK * PS_PACK_BLOCK; }

struct Packed {
    at::Tensor codes, scales;
    int64_t rows = 0, cols = 0;
    Packed() = default;
    Packed(int64_t r, int64_t c, const at::Tensor &like) : rows(r), cols(c)
    {
        codes = fresh({r, padded(c)}, at::kChar, like);
        scales = fresh({r, padded(c) / PS_PACK_BLOCK}, at::kByte, like);
    }
    Packed(PyObject *codes_, PyObject *scales_, PyObject *cols_) : codes(tensor_of(codes_, "codes")), scales(tensor_of(scales_, "scales"))
    {
        cols = PyLong_AsLongLong(cols_);
        if (cols == -1 && PyErr_Occurred()) throw python_error();
        TORCH_CHECK_TYPE(codes.scalar_type() == at::kChar && scales.scalar_type() == at::kByte, "codes must be int8 and scales uint8, got ", codes.scalar_type(), " and ",
                         scales.scalar_type());
        TORCH_CHECK_VALUE(cols >= 1 && codes.dim() == 2 && codes.is_contiguous() && codes.size(1) == padded(cols), "codes of ", cols, " columns must be rows x ", padded(cols),
                          ", contiguous, got shape ", codes.sizes(), " with strides ", codes.strides());
        rows = codes.size(0);
        TORCH_CHECK_VALUE(scales.dim() == 2 && scales.is_contiguous() && scales.size(0) == rows && scales.size(1) == padded(cols) / PS_PACK_BLOCK, "scales must be ", rows, " x ",
                          padded(cols) / PS_PACK_BLOCK, ", contiguous, got shape ", scales.sizes(), " with strides ", scales.strides());
        TORCH_CHECK_VALUE(codes.is_cuda() && codes.device() == scales.device(), "codes and scales must live on one GPU, got ", codes.device(), " and ", scales.device());
    }
};

struct Head {
    const at::Tensor &hidden, &head;
    ps_head c;
    Head(PyObject *hidden_, PyObject *head_, PyObject *tokens, PyObject *temperature) : hidden(tensor_of(hidden_, "hidden")), head(tensor_of(head_, "head"))
    {
        TORCH_CHECK_TYPE(hidden.scalar_type() == at::kBFloat16 && head.scalar_type() == at::kBFloat16, "hidden and head must be bf16, got ", hidden.scalar_type(), " and ",
                         head.scalar_type());
        TORCH_CHECK_VALUE(rows_fine(hidden) && rows_fine(head), "hidden must be rows x width and head vocabulary x width, with the width contiguous");
        TORCH_CHECK_VALUE(hidden.size(1) == head.size(1), "hidden has width ", hidden.size(1), ", head ", head.size(1));
        TORCH_CHECK_VALUE(hidden.is_cuda() && hidden.device() == head.device(), "hidden and head must live on one GPU, got ", hidden.device(), " and ", head.device());
        c.hidden_dev = hidden.const_data_ptr();
        c.head_dev = head.const_data_ptr();
        c.rows = hidden.size(0);
        c.width = hidden.size(1);
        c.vocab = head.size(0);
        c.hidden_stride = row_stride(hidden);
        c.head_stride = row_stride(head);
        c.tokens_dev = per_row<int64_t>(tokens, c.rows, "tokens", hidden);
        c.temperature = static_cast<float>(number(temperature));
    }
    at::Tensor floats(int64_t n) const { return fresh({n}, at::kFloat, hidden); }
    at::Tensor workspace(bool grad) const
    {
        int64_t need = 0;
        TORCH_CHECK_VALUE(head_workspace(&c, grad, &need) == PS_OK, "no such call: ", c.rows, " rows of width ", c.width, " (strides ", c.hidden_stride, ", ", c.head_stride, "), ", c.vocab,
                          " entries, temperature ", c.temperature);
        return scratch(need, hidden);
    }
};

// Which gradients: True, False or None, "hidden", "head".
struct Wanted {
    bool hidden = false, head = false;
    explicit Wanted(PyObject *o)
    {
        if (o == Py_False || o == Py_None) return;
        if (o == Py_True) { hidden = head = true; return; }
        TORCH_CHECK_VALUE(PyUnicode_Check(o), "grad is True, False, 'hidden' or 'head'");
        hidden = PyUnicode_CompareWithASCIIString(o, "hidden") == 0;
        head = PyUnicode_CompareWithASCIIString(o, "head") == 0;
        TORCH_CHECK_VALUE(hidden || head, "grad is True, False, 'hidden' or 'head'");
    }
    at::Tensor of_hidden(const Head &h) const { return hidden ? fresh({h.c.rows, h.c.width}, at::kBFloat16, h.hidden) : at::Tensor(); }
    at::Tensor of_head(const Head &h) const { return head ? fresh({h.c.vocab, h.c.width}, at::kBFloat16, h.head) : at::Tensor(); }
};

// (hidden, head, tokens, weights, temperature) -> (status, logp, lse)
PyObject *head_logprob(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    expect(n, 5);
    const Head h(a[0], a[1], a[2], a[4]);
    const float *weights = per_row<float>(a[3], h.c.rows, "weights", h.hidden, true);
    const c10::cuda::CUDAGuard guard(h.hidden.device());
    const at::Tensor logp = h.floats(h.c.rows), lse = h.floats(h.c.rows), ws = h.workspace(false);
    const int status = call_head_logprob(&h.c, weights, data<float>(logp), data<float>(lse), ws.data_ptr(), ws.numel(), c10::cuda::getCurrentCUDAStream().stream());
    return result(status, {logp, lse});
    END_HANDLE_TH_ERRORS
}

// (hidden, head, tokens, lse, dlogp, temperature, grad) -> (status, dhidden, dhead)
PyObject *head_logprob_grad(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    expect(n, 7);
    const Head h(a[0], a[1], a[2], a[5]);
    const float *lse = per_row<float>(a[3], h.c.rows, "lse", h.hidden), *dlogp = per_row<float>(a[4], h.c.rows, "dlogp", h.hidden);
    const Wanted want(a[6]);
    const c10::cuda::CUDAGuard guard(h.hidden.device());
    const at::Tensor dhidden = want.of_hidden(h), dhead = want.of_head(h), ws = h.workspace(true);
    const int status = call_head_logprob_grad(&h.c, lse, dlogp, data<void>(dhidden), data<void>(dhead), ws.data_ptr(), ws.numel(), c10::cuda::getCurrentCUDAStream().stream());
    return result(status, {dhidden, dhead});
    END_HANDLE_TH_ERRORS
}

// (hidden, head, tokens, weights, temperature, grad) -> (status, stats, logp, lse, dhidden, dhead)
PyObject *head_cross_entropy(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    expect(n, 6);
    const Head h(a[0], a[1], a[2], a[4]);
    const float *weights = per_row<float>(a[3], h.c.rows, "weights", h.hidden, true);
    const Wanted want(a[5]);
    const c10::cuda::CUDAGuard guard(h.hidden.device());
    const at::Tensor stats = h.floats(2), logp = h.floats(h.c.rows), lse = h.floats(h.c.rows), dhidden = want.of_hidden(h), dhead = want.of_head(h),
                     ws = h.workspace(want.hidden || want.head);
    const int status = call_head_cross_entropy(&h.c, weights, data<float>(stats), data<float>(logp), data<float>(lse), data<void>(dhidden), data<void>(dhead), ws.data_ptr(), ws.numel(),
                                               c10::cuda::getCurrentCUDAStream().stream());
    return result(status, {stats, logp, lse, dhidden, dhead});
    END_HANDLE_TH_ERRORS
}

// (x) -> (status, codes, scales)
PyObject *pack8(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    expect(n, 1);
    const at::Tensor &x = rows_of(a[0], "x");
    const c10::cuda::CUDAGuard guard(x.device());
    const Packed p(x.size(0), x.size(1), x);
    const int status = call_pack8(x.const_data_ptr(), grad_dtype(x.scalar_type()), p.rows, p.cols, row_stride(x), data<int8_t>(p.codes), data<uint8_t>(p.scales),
                                  c10::cuda::getCurrentCUDAStream().stream());
    return result(status, {p.codes, p.scales});
    END_HANDLE_TH_ERRORS
}

// (codes, scales, cols, whether bf16) -> (status, values)
PyObject *unpack8(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    expect(n, 4);
    const Packed p(a[0], a[1], a[2]);
    const c10::cuda::CUDAGuard guard(p.codes.device());
    const bool half = a[3] == Py_True;
    const at::Tensor out = fresh({p.rows, p.cols}, half ? at::kBFloat16 : at::kFloat, p.codes);
    const int status = call_unpack8(const_data<int8_t>(p.codes), const_data<uint8_t>(p.scales), p.rows, p.cols, out.data_ptr(), half ? PS_GRAD_BF16 : PS_GRAD_FP32, p.cols,
                                    c10::cuda::getCurrentCUDAStream().stream());
    return result(status, {out});
    END_HANDLE_TH_ERRORS
}

// (x, gain, residual, eps, whether out, whether codes, whether the total replaces the residual) -> (status, out, total, codes, scales, rstd)
PyObject *rms_norm(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    expect(n, 7);
    const at::Tensor &x = rows_of(a[0], "x");
    const int64_t rows = x.size(0), cols = x.size(1);
    const at::Tensor gain = gain_of(a[1], cols, x), residual = rows_like(a[2], "residual", x);
    const bool want_out = a[4] == Py_True, want_codes = a[5] == Py_True, inplace = a[6] == Py_True;
    TORCH_CHECK_VALUE(!inplace || residual.defined(), "inplace needs a residual to replace");
    const c10::cuda::CUDAGuard guard(x.device());
    ps_norm c{};
    c.eps = static_cast<float>(number(a[3]));
    at::Tensor total = residual.defined() ? inplace ? residual : fresh({rows, cols}, x.scalar_type(), x) : at::Tensor(), out;
    if (want_out) out = fresh({rows, cols}, x.scalar_type(), x);
    const Packed p = want_codes ? Packed(rows, cols, x) : Packed();
    const at::Tensor rstd = fresh({rows}, at::kFloat, x);
    c.x_dev = x.const_data_ptr(); c.residual_dev = const_data<void>(residual); c.gain_dev = const_data<void>(gain);
    c.dtype = grad_dtype(x.scalar_type());
    c.gain_dtype = gain.defined() ? grad_dtype(gain.scalar_type()) : c.dtype;
    c.rows = rows; c.cols = cols; c.x_stride = row_stride(x);
    c.residual_stride = residual.defined() ? row_stride(residual) : cols;
    c.total_stride = total.defined() ? row_stride(total) : cols;
    c.total_dev = data<void>(total); c.out_dev = data<void>(out);
    c.codes_dev = data<int8_t>(p.codes); c.scales_dev = data<uint8_t>(p.scales); c.rstd_dev = data<float>(rstd);
    const int status = call_rms_norm(&c, c10::cuda::getCurrentCUDAStream().stream());
    if (inplace && status == PS_OK) changed(residual);
    return result(status, {out, total, p.codes, p.scales, rstd});
    END_HANDLE_TH_ERRORS
}

// (dout, codes or total, scales or None, rstd, gain, dtotal, whether the gain's gradient) -> (status, dx, dgain)
PyObject *rms_norm_grad(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    expect(n, 7);
    const at::Tensor &dout = rows_of(a[0], "dout");
    const int64_t rows = dout.size(0), cols = dout.size(1);
    Packed p;
    at::Tensor total;
    if (a[2] != Py_None) {
        PyObject *wanted = PyLong_FromLongLong(cols);
        if (!wanted) throw python_error();
        const struct Drop { PyObject *o; ~Drop() { Py_DECREF(o); } } drop{wanted};
        p = Packed(a[1], a[2], wanted);
        TORCH_CHECK_VALUE(p.rows == rows && p.codes.device() == dout.device(), "codes of ", p.rows, " rows on ", p.codes.device(), ", dout has ", rows, " on ", dout.device());
    } else {
        total = rows_like(a[1], "total", dout);
        TORCH_CHECK_TYPE(total.defined(), "what the norm kept: a Packed8 or the total");
    }
    const float *rstd = per_row<float>(a[3], rows, "rstd", dout);
    const at::Tensor gain = gain_of(a[4], cols, dout), dtotal = rows_like(a[5], "dtotal", dout);
    const bool want_gain = a[6] == Py_True && gain.defined();
    const c10::cuda::CUDAGuard guard(dout.device());
    const at::Tensor dx = fresh({rows, cols}, dout.scalar_type(), dout), dgain = want_gain ? fresh({cols}, gain.scalar_type(), gain) : at::Tensor();
    int64_t need = 0;
    TORCH_CHECK_VALUE(norm_grad_workspace(rows, cols, &need) == PS_OK, "too many rows or columns, or none: ", rows, " x ", cols);
    const at::Tensor ws = scratch(want_gain ? need : 0, dout);
    ps_norm_grad c{};
    c.dout_dev = dout.const_data_ptr(); c.total_dev = const_data<void>(total); c.gain_dev = const_data<void>(gain); c.dtotal_dev = const_data<void>(dtotal);
    c.codes_dev = const_data<int8_t>(p.codes); c.scales_dev = const_data<uint8_t>(p.scales); c.rstd_dev = rstd;
    c.dtype = grad_dtype(dout.scalar_type());
    c.gain_dtype = gain.defined() ? grad_dtype(gain.scalar_type()) : c.dtype;
    c.rows = rows; c.cols = cols; c.dout_stride = row_stride(dout);
    c.total_stride = total.defined() ? row_stride(total) : cols;
    c.dtotal_stride = dtotal.defined() ? row_stride(dtotal) : cols;
    c.dx_dev = dx.data_ptr(); c.dgain_dev = data<void>(dgain);
    const int status = call_rms_norm_grad(&c, ws.data_ptr(), ws.numel(), c10::cuda::getCurrentCUDAStream().stream());
    return result(status, {dx, dgain});
    END_HANDLE_TH_ERRORS
}

// (dout, codes, scales, cols, gain, whether fp32) -> (status, dweight)
PyObject *packed_weight_grad(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    expect(n, 6);
    const at::Tensor &dout = rows_of(a[0], "dout");
    TORCH_CHECK_TYPE(dout.scalar_type() == at::kBFloat16, "dout must be bf16, got ", dout.scalar_type());
    const Packed p(a[1], a[2], a[3]);
    TORCH_CHECK_VALUE(p.rows == dout.size(0) && p.codes.device() == dout.device(), "codes of ", p.rows, " rows on ", p.codes.device(), ", dout has ", dout.size(0), " on ", dout.device());
    const at::Tensor gain = gain_of(a[4], p.cols, dout);
    const bool wide = a[5] == Py_True;
    const c10::cuda::CUDAGuard guard(dout.device());
    const at::Tensor dweight = fresh({dout.size(1), p.cols}, wide ? at::kFloat : at::kBFloat16, dout);
    ps_packed_grad c{};
    c.dout_dev = dout.const_data_ptr(); c.gain_dev = const_data<void>(gain); c.codes_dev = const_data<int8_t>(p.codes); c.scales_dev = const_data<uint8_t>(p.scales);
    c.gain_dtype = gain.defined() ? grad_dtype(gain.scalar_type()) : PS_GRAD_FP32;
    c.out_dtype = wide ? PS_GRAD_FP32 : PS_GRAD_BF16;
    c.rows = p.rows; c.outs = dout.size(1); c.cols = p.cols; c.dout_stride = row_stride(dout);
    c.dweight_dev = dweight.data_ptr();
    int64_t need = 0;
    TORCH_CHECK_VALUE(packed_grad_workspace(&c, &need) == PS_OK, "no such product: ", c.rows, " rows of ", c.outs, " (stride ", c.dout_stride, ") and ", c.cols);
    const at::Tensor ws = scratch(need, dout);
    const int status = call_packed_weight_grad(&c, ws.data_ptr(), ws.numel(), c10::cuda::getCurrentCUDAStream().stream());
    return result(status, {dweight});
    END_HANDLE_TH_ERRORS
}

#define SOFTSYNC_FAST(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    SOFTSYNC_FAST(bind), SOFTSYNC_FAST(token_logprob), SOFTSYNC_FAST(policy_loss), SOFTSYNC_FAST(preference_loss), SOFTSYNC_FAST(gradients),
    SOFTSYNC_FAST(written), SOFTSYNC_FAST(head_logprob), SOFTSYNC_FAST(head_logprob_grad), SOFTSYNC_FAST(head_cross_entropy), SOFTSYNC_FAST(pack8),
    SOFTSYNC_FAST(unpack8), SOFTSYNC_FAST(rms_norm), SOFTSYNC_FAST(rms_norm_grad), SOFTSYNC_FAST(packed_weight_grad),
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }
