"""Operators around the parameter server for language models (include/softsync_learn.h): on the learner the token log
probabilities, the clipped policy loss and the preference loss with their gradients with respect to the logits; on the server
the global norm of weighted gradients and AdamW over many tensors with moments in 32 or 8 bits.

As in `binding`, this side checks and marshals arguments and allocates outputs (the losses and gradient lists in the `_marshal`
extension, csrc/marshal.cpp); the work is done by the library on torch's current stream of the tensors' device.
"""
from __future__ import annotations

import ctypes as C
import itertools
import os
from typing import List, NamedTuple, Optional, Sequence, Union

import torch

from . import binding as B, build as _build

if not os.path.exists(_build.MARSHAL):
    raise RuntimeError("_marshal.so is not built (%s). Run `python -m paper_1511_05950_b200.build`." % _build.MARSHAL)
from . import _marshal  # noqa: E402

_marshal.bind(*[C.cast(f, C.c_void_p).value for f in (B.ps_loss_workspace, B.ps_token_logprob, B.ps_policy_loss, B.ps_preference_loss)])
INPLACE = "inplace"


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
    """A list of tensors by their sizes, for the global norm of their gradients.  One list's calls go to one stream at a time; which one
    may change from call to call, and a list may be dropped while its work is under way."""

    def __init__(self, sizes: Sequence[int], device=None):
        self._h = C.c_void_p()
        self.device = _cuda_device(device)
        self.sizes = [int(n) for n in sizes]
        self._sizes = (C.c_int64 * max(1, len(self.sizes)))(*self.sizes)
        elems, need = C.c_int64(), C.c_int64()
        B._check(B.ps_tensors_sizes(len(self.sizes), self._sizes, C.byref(elems), C.byref(need)), "ps_tensors_sizes")
        self.state_elems = elems.value
        self._workspace = torch.empty(need.value, dtype=torch.uint8, device=self.device)
        self._own, self._streams = [self._workspace], {_stream(self.device)}   # memory nobody else knows of; the streams it was used on
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

    def _stream(self) -> int:
        """The current stream.  torch's allocator is told of each, so that it gives the list's own memory, which is that of the stream the list
        was made on, to nobody before the work there is done."""
        stream = _stream(self.device)
        if stream not in self._streams:
            for t in self._own:
                t.record_stream(torch.cuda.current_stream(self.device))
            self._streams.add(stream)
        return stream

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
            self._pointers[c] = ((C.c_void_p * (c * n))(), (C.c_float * c)())      # sized for what the extension writes
        ptrs, factors = self._pointers[c]
        dtype = _marshal.gradients(grads, C.addressof(self._sizes), n, self.device.index, C.addressof(ptrs), c)
        factors[:] = [1.0] * c if scales is None else scales
        return ptrs, c, factors, dtype

    def grad_norm(self, grads, scales: Optional[Sequence[float]] = None, max_norm: float = float("inf"),
                  out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """(|g|, clipping factor) of g = sum_l scales[l] * grads[l], as two fp32 values on the device: the factor is max_norm / |g|
        where |g| is larger than max_norm, else 1.  grads: a list of tensors, or a list of c such lists."""
        ptrs, c, factors, dtype = self._gradients(grads, scales)
        if out is None:
            out = torch.empty(2, dtype=torch.float32, device=self.device)
        else:
            B.require_tensor(out, torch.float32, 2, "norm output", on_gpu=True, device=self.device)
        B._check(B.ps_grad_norm(self._h, ptrs, c, factors, dtype, max_norm, out.data_ptr(), self._stream()), "ps_grad_norm")
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
            self._own += state
        if len(state) != len(shapes):
            raise ValueError("state of %d-bit moments has %d arrays, got %d" % (state_bits, len(shapes), len(state)))
        for t, (d, k) in zip(state, shapes):
            B.require_tensor(t, d, k, "state array", on_gpu=True, device=self.device)
        self._written = params + [t for t in mirrors if t is not None]
        self.params, self.mirrors, self.state, self.state_bits = params, mirrors, tuple(state), state_bits
        self.lr, self.betas, self.eps, self.weight_decay, self.steps, self.seed = lr, betas, eps, weight_decay, step, seed
        p_arr = (C.c_void_p * n)(*[p.data_ptr() for p in params])
        m_arr = (C.c_void_p * n)(*[None if t is None else t.data_ptr() for t in mirrors])
        f_arr = [None if x is None else (C.c_float * n)(*[float(y) for y in x]) for x in (lr_mult, decay_mult)]
        s_ptr = [t.data_ptr() for t in self.state] + [None] * (4 - len(self.state))
        B._check(B.ps_tensors_bind_adamw(self._h, p_arr, m_arr, f_arr[0], f_arr[1], state_bits, *s_ptr, _stream(self.device)),
                 "ps_tensors_bind_adamw")
        self._config = B.AdamwConfig()

    def _configure(self):
        k = self._config
        k.lr, (k.beta1, k.beta2), k.eps, k.weight_decay = self.lr, self.betas, self.eps, self.weight_decay
        k.step, k.seed = self.steps + 1, self.seed
        return k

    def check(self) -> None:
        """Raises if the next step would refuse lr, betas, eps, weight_decay or steps as they are."""
        B._check(B.ps_adamw_check(C.byref(self._configure())), "ps_adamw_check")

    def step(self, grads, scales: Optional[Sequence[float]] = None, clip: Optional[torch.Tensor] = None) -> None:
        """One step with g = sum_l scales[l] * grads[l] (times clip[1] if `clip`, the result of grad_norm, is given: where its norm is not
        finite nothing changes).  The step is counted in `steps` either way."""
        ptrs, c, factors, dtype = self._gradients(grads, scales)
        if clip is not None:
            B.require_tensor(clip, torch.float32, 2, "clip", on_gpu=True, device=self.device)
        k = self._configure()
        B._check(B.ps_adamw_step(self._h, ptrs, c, factors, dtype, C.byref(k), None if clip is None else clip.data_ptr(),
                                 self._stream()), "ps_adamw_step")
        _marshal.written(self._written)
        self.steps += 1

    def moments(self):
        """(m, v) as state arrays: the fp32 arrays themselves, or the 8-bit moments' values in bf16 (exactly; new tensors)."""
        if self.state_bits == 32:
            return self.state
        m, v = (torch.empty(self.state_elems, dtype=torch.bfloat16, device=self.device) for _ in range(2))
        B._check(B.ps_adamw_moments(self._h, m.data_ptr(), v.data_ptr(), self._stream()), "ps_adamw_moments")
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


def token_logprob(logits: torch.Tensor, tokens: torch.Tensor, weights: Optional[torch.Tensor] = None, temperature: float = 1.0) -> TokenLogprob:
    """Log probability of each row's token, log normaliser and entropy, from one pass over the logits (rows x vocabulary, fp32 or bf16).
    Rows of weight zero are not read and give zeros."""
    status, *out = _marshal.token_logprob(logits, tokens, weights, temperature)
    B._check(status, "ps_token_logprob")
    return TokenLogprob(*out)


def policy_loss(logits: torch.Tensor, tokens: torch.Tensor, old_logp: torch.Tensor, advantages: torch.Tensor,
                weights: Optional[torch.Tensor] = None, ref_logp: Optional[torch.Tensor] = None, clip_low: float = 0.2, clip_high: float = 0.2,
                kl_coef: float = 0.0, entropy_coef: float = 0.0, temperature: float = 1.0, grad: Union[bool, str, torch.Tensor] = True) -> PolicyLoss:
    """The clipped policy loss with a KL and an entropy term (formulas: include/softsync_learn.h) and its gradient with respect to the
    logits: `logits.backward(result.dlogits)` continues into the model.  grad: True (a new tensor), a tensor to write to, "inplace" (the
    gradient replaces the logits, which autograd takes as it takes any change in place: not for logits that their producer saved for its
    backward pass, as a soft cap's tanh does), or False."""
    status, *out = _marshal.policy_loss(logits, tokens, weights, temperature, old_logp, advantages, ref_logp, clip_low, clip_high, kl_coef,
                                        entropy_coef, grad)
    B._check(status, "ps_policy_loss")
    return PolicyLoss(*out)


def preference_loss(logits: torch.Tensor, tokens: torch.Tensor, offsets: torch.Tensor, ref_logp: torch.Tensor,
                    weights: Optional[torch.Tensor] = None, beta: float = 0.1, label_smoothing: float = 0.0, temperature: float = 1.0,
                    grad: Union[bool, str, torch.Tensor] = True) -> PreferenceLoss:
    """The preference loss over pairs of sequences (formulas: include/softsync_learn.h) and its gradient with respect to the logits.
    offsets: 2 * pairs + 1 ascending row numbers (int64, on the GPU); sequences 2i and 2i + 1 are pair i's preferred and other answer.  ref_logp: 2 *
    pairs.  grad: as in policy_loss."""
    status, *out = _marshal.preference_loss(logits, tokens, weights, temperature, offsets, ref_logp, beta, label_smoothing, grad)
    B._check(status, "ps_preference_loss")
    return PreferenceLoss(*out)


# ---- an n-softsync server whose update is an AdamW step -------------------------------------------------------------------

class AdamWServer:
    """The n-softsync protocol (Sections 2.1-2.4) with an AdamW step in the place of momentum SGD.

    A `ParameterServer` without parameters keeps the clock: learners `pull` a timestamp, `push` a gradient (a list of one tensor for each
    parameter) with it, and every c = floor(num_learners / n) pushes make a group.  `apply_update` takes the oldest group: g = sum_l s_l g_l
    with s_l = 1 / (c sigma_l) (or the modulation's own penalty over c) in the server's summation order, clipped to max_norm if given, then
    one AdamW step.  The learning rate is AdamW's: a group of equally stale gradients is scaled as a whole, which the step's normalisation
    takes back, so staleness weighs gradients against one another, inside a group and through the moments from group to group.
    Gradients are borrowed until the update that consumes them; all work goes to torch's current stream, which has to come after whatever
    wrote the group's gradients."""

    def __init__(self, params: Sequence[torch.Tensor], num_learners: int, n: int, modulation: str = "inv_staleness",
                 max_norm: Optional[float] = None, **adamw):
        self.optimizer = AdamW(params, **adamw)
        self.max_norm = max_norm
        self._check()
        self._clock = B.ParameterServer(0, num_learners, n, 1.0, modulation=modulation)
        self._token = torch.zeros(1, device=self.optimizer.device)          # stands for a gradient where the clock asks for one
        self._pushed = {}                                                   # (learner, push index): gradient, in the order of the pushes
        self._dtype = None                                                  # of the gradients: the first push's
        self._pushes = [0] * num_learners
        self.c = self._clock.c
        self.last_norm = None                                               # (norm, factor) of the last update, on the device

    def timestamps(self):
        """(applied, logical)."""
        return self._clock.timestamps()

    def pull(self) -> int:
        """The timestamp that a gradient computed on the present parameters must carry.  Complete groups are applied first, so that the
        parameters are those of the timestamp."""
        while self._clock.timestamps()[1] > self._clock.timestamps()[0]:
            self.apply_update()
        return self._clock.pull_weights()

    def push(self, learner: int, grads: Sequence[torch.Tensor], ts: int) -> bool:
        """True if this push completed a group.  All gradients have the first one's type."""
        grads = list(grads)
        dtype = self.optimizer._gradients(grads, None)[3]                   # what the update would refuse is refused here
        if self._dtype not in (None, dtype):
            raise TypeError("gradients must all be fp32 or all bf16; this server's are %s" % ("bf16" if self._dtype == B.PS_GRAD_BF16 else "fp32"))
        ready = self._clock.push_gradient(learner, self._token, ts)
        self._dtype = dtype
        self._pushed[learner, self._pushes[learner]] = grads
        self._pushes[learner] += 1
        return ready

    def _check(self) -> None:
        if self.max_norm is not None and not self.max_norm > 0:
            raise ValueError("max_norm must be above zero, got %r" % (self.max_norm,))
        self.optimizer.check()

    def apply_update(self) -> None:
        """Applies the oldest complete group.  Where the step would refuse it, nothing has changed when this raises."""
        group = list(itertools.islice(self._pushed.values(), self.c))
        if len(group) == self.c:                                            # else the clock refuses
            self._check()
            self.optimizer._gradients(group, None)
        self._clock.apply_update()
        entries = self._clock.update_log(self._clock.timestamps()[0] - 1, 1)
        grads = [self._pushed.pop((int(e["learner"]), int(e["push_index"]))) for e in entries]
        scales = [float(e["scale"]) for e in entries]
        clip = None
        if self.max_norm is not None:
            clip = self.last_norm = self.optimizer.grad_norm(grads, scales, self.max_norm)
        self.optimizer.step(grads, scales, clip=clip)
        stream = torch.cuda.current_stream(self.optimizer.device)
        for g in itertools.chain.from_iterable(grads):                      # they may be dropped now: not before the step has read them
            g.record_stream(stream)

    def staleness_histogram(self):
        return self._clock.staleness_histogram()
