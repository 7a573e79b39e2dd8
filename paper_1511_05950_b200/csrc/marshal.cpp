// Argument checks, output tensors and workspaces of the calls in learn.py, as a CPython extension over torch's C++ tensors: what a
// call costs on the host is most of what a short one takes.  The work is done by the entry points of softsync_learn.h, whose
// addresses learn.py hands over once (bind); a call returns their status for learn.py to raise.
#include "../../include/softsync_learn.h"

#include <Python.h>
#include <ATen/ATen.h>
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

// (addresses of ps_loss_workspace, ps_token_logprob, ps_policy_loss, ps_preference_loss)
PyObject *bind(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    expect(n, 4);
    void *p[4];
    for (int k = 0; k < 4; ++k) {
        p[k] = PyLong_AsVoidPtr(a[k]);
        if (!p[k]) throw python_error();
    }
    loss_workspace = reinterpret_cast<decltype(loss_workspace)>(p[0]);
    call_token_logprob = reinterpret_cast<decltype(call_token_logprob)>(p[1]);
    call_policy_loss = reinterpret_cast<decltype(call_policy_loss)>(p[2]);
    call_preference_loss = reinterpret_cast<decltype(call_preference_loss)>(p[3]);
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

#define SOFTSYNC_FAST(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    SOFTSYNC_FAST(bind), SOFTSYNC_FAST(token_logprob), SOFTSYNC_FAST(policy_loss), SOFTSYNC_FAST(preference_loss), SOFTSYNC_FAST(gradients),
    SOFTSYNC_FAST(written),
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }
