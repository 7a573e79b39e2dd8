"""Operators around the parameter server for language models (include/softsync_learn.h): on the learner the token log
probabilities, the clipped policy loss and the preference loss with their gradients with respect to the logits; on the server
the global norm of weighted gradients and AdamW over many tensors with moments in 32 or 8 bits.

As in `binding`, Python checks and marshals arguments and allocates outputs; the work is done by the library on torch's
current stream of the tensors' device.
"""
from __future__ import annotations

import ctypes as C
import functools
import itertools
import threading
from typing import List, NamedTuple, Optional, Sequence, Union

import torch

from . import binding as B

_DTYPES = {torch.float32: B.PS_GRAD_FP32, torch.bfloat16: B.PS_GRAD_BF16}
INPLACE = "inplace"
_numel, _is_contiguous, _get_device, _data_ptr = (torch.Tensor.numel, torch.Tensor.is_contiguous, torch.Tensor.get_device, torch.Tensor.data_ptr)


def _stream(device: torch.device) -> int:
    return torch._C._cuda_getCurrentRawStream(device.index)


def _on(device: torch.device):
    """Makes `device` current for a call that has no handle to remember it."""
    return _HERE if torch._C._cuda_getDevice() == device.index else torch.cuda.device(device)


_HERE = B._NullCtx()


def _cuda_device(device) -> torch.device:
    device = torch.device("cuda" if device is None else device)
    if device.type != "cuda":
        raise ValueError("the operators run on a CUDA device, got %s" % device)
    return device if device.index is not None else torch.device("cuda", torch.cuda.current_device())


# ---- a list of tensors ------------------------------------------------------------------------------------------------

class TensorList:
    """A list of tensors by their sizes, for the global norm of their gradients.  One list's calls go to one stream at a time."""

    def __init__(self, sizes: Sequence[int], device=None):
        self._h = C.c_void_p()
        self.device = _cuda_device(device)
        self.sizes = [int(n) for n in sizes]
        self._sizes = (C.c_int64 * max(1, len(self.sizes)))(*self.sizes)
        elems, need = C.c_int64(), C.c_int64()
        B._check(B.ps_tensors_sizes(len(self.sizes), self._sizes, C.byref(elems), C.byref(need)), "ps_tensors_sizes")
        self.state_elems = elems.value
        self._workspace = torch.empty(need.value, dtype=torch.uint8, device=self.device)
        with _on(self.device):
            B._check(B.ps_tensors_create(C.byref(self._h), len(self.sizes), self._sizes, self._workspace.data_ptr(), need.value,
                                         _stream(self.device)), "ps_tensors_create")
        self._pointers = {}                       # ctypes arrays by the number of gradients, reused from call to call

    def destroy(self) -> None:
        if self._h:
            B._check(B.ps_tensors_destroy(self._h), "ps_tensors_destroy")
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass

    def state_offsets(self) -> List[int]:
        """First element of each tensor in a state array."""
        at, out = 0, []
        for n in self.sizes:
            out.append(at)
            at += -(-n // B.PS_STATE_BLOCK) * B.PS_STATE_BLOCK
        return out

    def _gradients(self, grads, scales):
        """(pointers, c, scales, dtype) of c gradients, each a list of one contiguous tensor per entry of the list."""
        if len(grads) and isinstance(grads[0], torch.Tensor):
            grads = [grads]
        c, n = len(grads), len(self.sizes)
        if not 1 <= c <= B.PS_LIST_MAX_GRADS:
            raise ValueError("between 1 and %d gradients, got %d" % (B.PS_LIST_MAX_GRADS, c))
        if scales is not None and len(scales) != c:
            raise ValueError("one scale for each of the %d gradients, got %d" % (c, len(scales)))
        if c not in self._pointers:
            self._pointers[c] = ((C.c_void_p * (c * n))(), (C.c_float * c)())
        ptrs, factors = self._pointers[c]
        flat = list(itertools.chain.from_iterable(grads))
        if [len(gradient) for gradient in grads] != [n] * c or list(map(_numel, flat)) != self.sizes * c:
            raise ValueError("each gradient must have the list's %d tensors with the same numbers of elements" % n)
        if not all(map(_is_contiguous, flat)):
            raise ValueError("gradient tensors must be contiguous")
        if set(map(_get_device, flat)) != {self.device.index}:
            raise ValueError("gradient tensors must live on the list's GPU, %s" % self.device)
        dtypes = {g.dtype for g in flat}
        dtype = dtypes.pop()
        if dtypes or dtype not in _DTYPES:
            raise TypeError("gradients must all be fp32 or all bf16")
        ptrs[:] = list(map(_data_ptr, flat))
        factors[:] = [1.0] * c if scales is None else scales
        return ptrs, c, factors, _DTYPES[dtype]

    def grad_norm(self, grads, scales: Optional[Sequence[float]] = None, max_norm: float = float("inf"),
                  out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """(|g|, clipping factor) of g = sum_l scales[l] * grads[l], as two fp32 values on the device: the factor is max_norm / |g|
        where |g| is larger than max_norm, else 1.  grads: a list of tensors, or a list of c such lists."""
        ptrs, c, factors, dtype = self._gradients(grads, scales)
        if out is None:
            out = torch.empty(2, dtype=torch.float32, device=self.device)
        else:
            B.require_tensor(out, torch.float32, 2, "norm output", on_gpu=True, device=self.device)
        B._check(B.ps_grad_norm(self._h, ptrs, c, factors, dtype, max_norm, out.data_ptr(), _stream(self.device)), "ps_grad_norm")
        return out


class AdamW(TensorList):
    """AdamW over a list of fp32 parameter tensors, one pass over all of them, moments in 32 or 8 bits.

    params: contiguous fp32 tensors on one GPU (views of a flat vector are fine), updated in place.  mirrors: bf16 tensors (or
    None) that every step rewrites with the rounded parameters.  lr_mult, decay_mult: a multiplier for each tensor.  state: (m, v) fp32 state
    arrays of `state_elems` elements (each tensor's part starts at `state_offsets`), or (m, v, m_scale, v_scale) byte arrays, the scales with
    one byte for each PS_STATE_BLOCK elements; zeros when not given.  step: how many steps the state has behind it.  seed: of the random
    rounding of 8-bit moments."""

    def __init__(self, params: Sequence[torch.Tensor], lr: float = 1e-3, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay: float = 0.01,
                 state_bits: int = 32, lr_mult=None, decay_mult=None, mirrors=None, state=None, step: int = 0, seed: int = 0):
        params = list(params)
        if not params:
            raise ValueError("at least one parameter tensor")
        if state_bits not in (8, 32):
            raise ValueError("moments have 8 or 32 bits, not %r" % (state_bits,))
        super().__init__([p.numel() for p in params], params[0].device)
        n = len(params)
        for p in params:
            B.require_tensor(p, torch.float32, p.numel(), "parameter", on_gpu=True, device=self.device)
        mirrors = [None] * n if mirrors is None else list(mirrors)
        for what, x in (("mirror", mirrors), ("learning-rate multiplier", lr_mult), ("decay multiplier", decay_mult)):
            if x is not None and len(x) != n:
                raise ValueError("one %s for each of the %d tensors, got %d" % (what, n, len(x)))
        for p, t in zip(params, mirrors):
            if t is not None:
                B.require_tensor(t, torch.bfloat16, p.numel(), "mirror", on_gpu=True, device=self.device)
        blocks = self.state_elems // B.PS_STATE_BLOCK
        shapes = [(torch.float32, self.state_elems)] * 2 if state_bits == 32 else [(torch.uint8, self.state_elems)] * 2 + [(torch.uint8, blocks)] * 2
        if state is None:
            state = [torch.zeros(max(1, k), dtype=d, device=self.device) for d, k in shapes]
        if len(state) != len(shapes):
            raise ValueError("state of %d-bit moments has %d arrays, got %d" % (state_bits, len(shapes), len(state)))
        for t, (d, k) in zip(state, shapes):
            B.require_tensor(t, d, k, "state array", on_gpu=True, device=self.device)
        self.params, self.mirrors, self.state, self.state_bits = params, mirrors, tuple(state), state_bits
        self.lr, self.betas, self.eps, self.weight_decay, self.steps, self.seed = lr, betas, eps, weight_decay, step, seed
        p_arr = (C.c_void_p * n)(*[p.data_ptr() for p in params])
        m_arr = (C.c_void_p * n)(*[None if t is None else t.data_ptr() for t in mirrors])
        f_arr = [None if x is None else (C.c_float * n)(*[float(y) for y in x]) for x in (lr_mult, decay_mult)]
        s_ptr = [t.data_ptr() for t in self.state] + [None] * (4 - len(self.state))
        B._check(B.ps_tensors_bind_adamw(self._h, p_arr, m_arr, f_arr[0], f_arr[1], state_bits, *s_ptr, _stream(self.device)),
                 "ps_tensors_bind_adamw")
        self._config = B.AdamwConfig()

    def step(self, grads, scales: Optional[Sequence[float]] = None, clip: Optional[torch.Tensor] = None) -> None:
        """One step with g = sum_l scales[l] * grads[l] (times clip[1] if `clip`, the result of grad_norm, is given: where its norm is not
        finite nothing changes).  The step is counted in `steps` either way."""
        ptrs, c, factors, dtype = self._gradients(grads, scales)
        if clip is not None:
            B.require_tensor(clip, torch.float32, 2, "clip", on_gpu=True, device=self.device)
        k = self._config
        k.lr, (k.beta1, k.beta2), k.eps, k.weight_decay = self.lr, self.betas, self.eps, self.weight_decay
        k.step, k.seed = self.steps + 1, self.seed
        B._check(B.ps_adamw_step(self._h, ptrs, c, factors, dtype, C.byref(k), None if clip is None else clip.data_ptr(),
                                 _stream(self.device)), "ps_adamw_step")
        self.steps += 1

    def moments(self):
        """(m, v) as state arrays: the fp32 arrays themselves, or the 8-bit moments' values in bf16 (exactly; new tensors)."""
        if self.state_bits == 32:
            return self.state
        m, v = (torch.empty(self.state_elems, dtype=torch.bfloat16, device=self.device) for _ in range(2))
        B._check(B.ps_adamw_moments(self._h, m.data_ptr(), v.data_ptr(), _stream(self.device)), "ps_adamw_moments")
        return m, v


# ---- losses from logits -----------------------------------------------------------------------------------------------

class TokenLogprob(NamedTuple):
    logp: torch.Tensor
    lse: torch.Tensor
    entropy: torch.Tensor


class PolicyLoss(NamedTuple):
    stats: torch.Tensor                  # loss, clipped term, KL term, entropy, share of clipped tokens
    logp: torch.Tensor
    entropy: torch.Tensor
    dlogits: Optional[torch.Tensor]


class PreferenceLoss(NamedTuple):
    stats: torch.Tensor                  # loss, share of positive margins, mean margin
    seq_logp: torch.Tensor
    dlogits: Optional[torch.Tensor]


def _logits(logits: torch.Tensor, tokens: torch.Tensor, weights: Optional[torch.Tensor], temperature: float) -> B.Logits:
    dtype = _DTYPES.get(logits.dtype)
    if dtype is None:
        raise TypeError("logits must be fp32 or bf16, got %s" % logits.dtype)
    if logits.dim() != 2 or (logits.stride(1) != 1 and logits.shape[1] > 1):
        raise ValueError("logits must be rows x vocabulary with the vocabulary contiguous")
    if not logits.is_cuda:
        raise ValueError("logits must live on the GPU")
    rows, vocab = logits.shape
    _per_row(tokens, rows, "tokens", logits, torch.int64)
    _per_row(weights, rows, "weights", logits)
    stride = logits.stride(0) if rows > 1 else max(vocab, 1)
    return B.Logits(logits.data_ptr(), dtype, rows, vocab, stride, tokens.data_ptr(), None if weights is None else weights.data_ptr(), temperature)


def _per_row(t: Optional[torch.Tensor], rows: int, what: str, logits: torch.Tensor, dtype: torch.dtype = torch.float32) -> None:
    if t is None:
        return
    if t.dtype is not dtype:
        raise TypeError("%s must be %s, got %s" % (what, dtype, t.dtype))
    if t.dim() != 1 or t.numel() != rows or not t.is_contiguous():
        raise ValueError("%s: %d values one behind the other, got shape %s with strides %s" % (what, rows, tuple(t.shape), t.stride()))
    if t.get_device() != logits.get_device():
        raise ValueError("%s is on %s, the logits on %s" % (what, t.device, logits.device))


def _gradient_buffer(logits: torch.Tensor, grad: Union[bool, str, torch.Tensor]):
    """(tensor or None, row stride) the gradient goes to."""
    rows, vocab = logits.shape
    if grad is False or grad is None:
        return None, vocab
    if grad is True:
        return torch.empty((rows, vocab), dtype=logits.dtype, device=logits.device), max(vocab, 1)
    if isinstance(grad, str):
        if grad != INPLACE:
            raise ValueError("grad is True, False, %r or a tensor" % INPLACE)
        grad = logits.detach()
    if grad.shape != logits.shape or grad.dtype != logits.dtype or grad.device != logits.device or (grad.stride(1) != 1 and vocab > 1):
        raise ValueError("the gradient's buffer must have the logits' shape, type and device, with the vocabulary contiguous")
    return grad, grad.stride(0) if rows > 1 else max(vocab, 1)


_workspaces = {}                          # (device, stream, thread): a workspace that such calls use one after the other


@functools.lru_cache(maxsize=1024)
def _workspace_bytes(rows: int, sequences: int) -> int:
    need = C.c_int64()
    B._check(B.ps_loss_workspace(rows, sequences, C.byref(need)), "ps_loss_workspace")
    return need.value


def _workspace(rows: int, sequences: int, device: torch.device, stream: int) -> torch.Tensor:
    need = _workspace_bytes(rows, sequences)
    capturing = torch._C._cuda_isCurrentStreamCapturing()               # a graph keeps its own
    key = (device.index, stream, threading.get_ident())
    ws = None if capturing else _workspaces.get(key)
    if ws is None or ws.numel() < need:
        ws = torch.zeros(max(need, 1 << 16), dtype=torch.uint8, device=device)
        if not capturing:
            _workspaces[key] = ws
    return ws


def token_logprob(logits: torch.Tensor, tokens: torch.Tensor, weights: Optional[torch.Tensor] = None, temperature: float = 1.0) -> TokenLogprob:
    """Log probability of each row's token, log normaliser and entropy, from one pass over the logits (rows x vocabulary, fp32 or bf16).
    Rows of weight zero are not read and give zeros."""
    lg = _logits(logits, tokens, weights, temperature)
    logp, lse, entropy = (torch.empty(lg.rows, dtype=torch.float32, device=logits.device) for _ in range(3))
    with _on(logits.device):
        B._check(B.ps_token_logprob(C.byref(lg), logp.data_ptr(), lse.data_ptr(), entropy.data_ptr(), _stream(logits.device)), "ps_token_logprob")
    return TokenLogprob(logp, lse, entropy)


def policy_loss(logits: torch.Tensor, tokens: torch.Tensor, old_logp: torch.Tensor, advantages: torch.Tensor,
                weights: Optional[torch.Tensor] = None, ref_logp: Optional[torch.Tensor] = None, clip_low: float = 0.2, clip_high: float = 0.2,
                kl_coef: float = 0.0, entropy_coef: float = 0.0, temperature: float = 1.0, grad: Union[bool, str, torch.Tensor] = True) -> PolicyLoss:
    """The clipped policy loss with a KL and an entropy term (formulas: include/softsync_learn.h) and its gradient with respect to the
    logits: `logits.backward(result.dlogits)` continues into the model.  grad: True (a new tensor), a tensor to write to, "inplace" (the
    gradient replaces the logits), or False."""
    lg = _logits(logits, tokens, weights, temperature)
    for what, t in (("old_logp", old_logp), ("advantages", advantages), ("ref_logp", ref_logp)):
        _per_row(t, lg.rows, what, logits)
    device = logits.device
    dlogits, stride = _gradient_buffer(logits, grad)
    stats = torch.empty(5, dtype=torch.float32, device=device)
    logp, entropy = (torch.empty(lg.rows, dtype=torch.float32, device=device) for _ in range(2))
    k = B.PolicyInputs(old_logp.data_ptr(), advantages.data_ptr(), None if ref_logp is None else ref_logp.data_ptr(),
                       clip_low, clip_high, kl_coef, entropy_coef)
    with _on(device):
        stream = _stream(device)
        ws = _workspace(lg.rows, 0, device, stream)
        B._check(B.ps_policy_loss(C.byref(lg), C.byref(k), stats.data_ptr(), logp.data_ptr(), entropy.data_ptr(),
                                  None if dlogits is None else dlogits.data_ptr(), stride, ws.data_ptr(), ws.numel(), stream), "ps_policy_loss")
    return PolicyLoss(stats, logp, entropy, dlogits)


def preference_loss(logits: torch.Tensor, tokens: torch.Tensor, offsets: torch.Tensor, ref_logp: torch.Tensor,
                    weights: Optional[torch.Tensor] = None, beta: float = 0.1, label_smoothing: float = 0.0, temperature: float = 1.0,
                    grad: Union[bool, str, torch.Tensor] = True) -> PreferenceLoss:
    """The preference loss over pairs of sequences (formulas: include/softsync_learn.h) and its gradient with respect to the logits.
    offsets: 2 * pairs + 1 ascending row numbers (int64, on the GPU); sequences 2i and 2i + 1 are pair i's preferred and other answer.  ref_logp: 2 *
    pairs.  grad: as in policy_loss."""
    lg = _logits(logits, tokens, weights, temperature)
    if offsets.dim() != 1 or offsets.numel() % 2 != 1:
        raise ValueError("offsets holds 2 * pairs + 1 row numbers")
    seqs = offsets.numel() - 1
    _per_row(offsets, seqs + 1, "offsets", logits, torch.int64)
    _per_row(ref_logp, seqs, "ref_logp", logits)
    device = logits.device
    dlogits, stride = _gradient_buffer(logits, grad)
    stats = torch.empty(3, dtype=torch.float32, device=device)
    seq_logp = torch.empty(seqs, dtype=torch.float32, device=device)
    k = B.PreferenceInputs(offsets.data_ptr(), ref_logp.data_ptr(), seqs // 2, beta, label_smoothing)
    with _on(device):
        stream = _stream(device)
        ws = _workspace(lg.rows, seqs, device, stream)
        B._check(B.ps_preference_loss(C.byref(lg), C.byref(k), stats.data_ptr(), seq_logp.data_ptr(),
                                      None if dlogits is None else dlogits.data_ptr(), stride, ws.data_ptr(), ws.numel(), stream), "ps_preference_loss")
    return PreferenceLoss(stats, seq_logp, dlogits)
