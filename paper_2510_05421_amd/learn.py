"""Learning operators on the caller's tensors: token log-probabilities, the clipped policy loss with its
gradient, and AdamW over many tensors with states in 32 or 8 bits.

Each call runs in the HIP kernels behind the C entry point of its name (include/dvi.h says what it
computes), on the current stream of its tensors' device; nothing waits for the device.  Gradients are
returned by the loss itself: nothing here is recorded by autograd, which does not notice either that a
step, or a gradient written over its logits, has changed a tensor that some graph still needs.
"""
from __future__ import annotations

import ctypes
from typing import Dict, List, NamedTuple, Optional, Sequence, Tuple

import torch

from . import _abi

_DTYPES = {torch.float32: _abi.FP32, torch.bfloat16: _abi.BF16}


def _refuse(msg):
    raise _abi.DVIError(_abi.ERR_ARG, msg)


def _logits(t, name):
    if t.dim() != 2 or t.dtype not in _DTYPES or not t.is_cuda:
        _refuse("%s must be a 2-d float32 or bfloat16 tensor on a GPU" % name)
    if t.shape[1] < 1 or (t.shape[1] > 1 and t.stride(1) != 1):
        _refuse("%s: the vocabulary must be contiguous" % name)
    return t.data_ptr()


def _ld(t):
    """Row stride in elements; a single row's says nothing."""
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _vector(t, name, rows, dtype, device):
    if t is None:
        return None
    if t.dtype != dtype or t.device != device or t.shape != (rows,) or not t.is_contiguous():
        _refuse("%s must be a contiguous %s tensor of %d elements on %s" % (name, dtype, rows, device))
    return t.data_ptr()


_raw_stream = torch._C._cuda_getCurrentRawStream   # the handle alone: a Stream object costs 2 us


def _call(device, fn, *args):
    """fn(*args, stream) on the device's current stream, with the device current."""
    at = device.index
    if torch.cuda.current_device() == at:
        st = fn(*args, _raw_stream(at))
    else:
        with torch.cuda.device(device):
            st = fn(*args, _raw_stream(at))
    if st != _abi.OK:
        raise _abi.DVIError(st, _abi.load().dvi_op_error().decode())


def _workspace(nbytes, device):
    return (torch.empty(nbytes, dtype=torch.uint8, device=device), nbytes) if nbytes else (None, 0)


def token_logprobs(logits: torch.Tensor, tokens: torch.Tensor, temperature: float = 1.0,
                   entropy: bool = False) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """(log softmax(logits / temperature)[token] of every row, the rows' entropies or None), fp32.

    logits [rows, vocab] fp32 or bf16 with contiguous rows of any stride, tokens int32 [rows]; rows whose
    token lies outside the vocabulary (-1, say) give 0."""
    lib = _abi.load()
    ptr = _logits(logits, "logits")
    rows, vocab = logits.shape
    dev = logits.device
    tok = _vector(tokens, "tokens", rows, torch.int32, dev)
    logp = torch.empty(rows, dtype=torch.float32, device=dev)
    ent = torch.empty(rows, dtype=torch.float32, device=dev) if entropy else None
    ws, nbytes = _workspace(lib.dvi_token_logprobs_workspace_bytes(rows, vocab), dev)
    args = _abi.LogprobArgs(rows, vocab, _DTYPES[logits.dtype], ptr, _ld(logits), tok, temperature, logp.data_ptr(),
                            ent.data_ptr() if entropy else None)
    _call(dev, lib.dvi_token_logprobs, args, ws.data_ptr() if nbytes else None, nbytes)
    return logp, ent


class PolicyLoss(NamedTuple):
    """terms: fp32 [5], the weighted sums (loss, policy, kl, entropy, weight of the clipped rows); logp: fp32
    [rows]; grad: d loss / d logits, or None."""
    terms: torch.Tensor
    logp: torch.Tensor
    grad: Optional[torch.Tensor]

    @property
    def loss(self) -> torch.Tensor:
        return self.terms[0]


def policy_loss(logits: torch.Tensor, tokens: torch.Tensor, advantages: torch.Tensor,
                old_logp: Optional[torch.Tensor] = None, weights: Optional[torch.Tensor] = None, *,
                ref_logits: Optional[torch.Tensor] = None, ref_logp: Optional[torch.Tensor] = None,
                temperature: float = 1.0, ref_temperature: float = 1.0, clip_low: float = 0.2, clip_high: float = 0.2,
                c_kl: float = 0.0, c_ent: float = 0.0, grad: bool = True,
                out: Optional[torch.Tensor] = None) -> PolicyLoss:
    """The clipped policy loss of dvi_policy_loss and, unless grad is False, its gradient with respect to
    the logits (into out where given, which may be the logits themselves).

    logits [rows, vocab] fp32 or bf16 with contiguous rows of any stride; tokens int32 [rows]; advantages,
    old_logp, weights and ref_logp fp32 [rows]; ref_logits like logits, or one row of them expanded."""
    lib = _abi.load()
    ptr = _logits(logits, "logits")
    rows, vocab = logits.shape
    dev = logits.device
    if advantages is None:
        _refuse("advantages must be given")
    f32 = torch.float32
    tok, adv = _vector(tokens, "tokens", rows, torch.int32, dev), _vector(advantages, "advantages", rows, f32, dev)
    old, wts = _vector(old_logp, "old_logp", rows, f32, dev), _vector(weights, "weights", rows, f32, dev)
    rlp = _vector(ref_logp, "ref_logp", rows, f32, dev)
    ref = None
    if ref_logits is not None:
        ref = _logits(ref_logits, "ref_logits")
        if ref_logits.shape != logits.shape or ref_logits.dtype != logits.dtype or ref_logits.device != dev:
            _refuse("ref_logits must have the logits' shape, type and device")
    if grad and out is None:
        out = torch.empty((rows, vocab), dtype=logits.dtype, device=dev)
    elif grad:
        _logits(out, "out")
        if out.shape != logits.shape or out.dtype != logits.dtype or out.device != dev:
            _refuse("out must have the logits' shape, type and device")
    elif out is not None:
        _refuse("out is given without grad")
    logp = torch.empty(rows, dtype=torch.float32, device=dev)
    terms = torch.empty(5, dtype=torch.float32, device=dev)
    ws, nbytes = _workspace(lib.dvi_policy_loss_workspace_bytes(rows, vocab), dev)
    args = _abi.PolicyArgs(rows, vocab, _DTYPES[logits.dtype], ptr, _ld(logits), tok, adv, old, wts, ref,
                           _ld(ref_logits) if ref is not None else 0, rlp, temperature, ref_temperature, clip_low,
                           clip_high, c_kl, c_ent, out.data_ptr() if grad else None, _ld(out) if grad else 0,
                           logp.data_ptr(), terms.data_ptr())
    _call(dev, lib.dvi_policy_loss, args, ws.data_ptr() if nbytes else None, nbytes)
    return PolicyLoss(terms, logp, out if grad else None)


class AdamW:
    """AdamW over a list of contiguous parameter tensors (all fp32, or all bf16) of one GPU, which step()
    updates in place; their storage and the states' must stay where they are.

    max_norm > 0 clips the gradients' global norm (grad_norm holds it after a step) and skips a step whose
    norm is not finite.  state_bits 8 keeps the moments in 8 bits with a scale per 256 elements, rounded at
    random from `seed`.  bf16 parameters get fp32 masters unless master is False.

    states: existing state tensors to go on with, lists by name: "m", "v" (32 bits) or "m", "r", "m_scale",
    "r_scale" (8 bits: r holds the square root of v), and "master"; step_count is the number of steps they
    have seen.  Both are attributes, which a checkpoint stores."""

    def __init__(self, params: Sequence[torch.Tensor], lr: float = 1e-3, betas: Tuple[float, float] = (0.9, 0.999),
                 eps: float = 1e-8, weight_decay: float = 0.0, max_norm: float = 0.0, state_bits: int = 32, seed: int = 0,
                 master: bool = True, states: Optional[Dict[str, List[torch.Tensor]]] = None, step_count: int = 0):
        self.params = list(params)
        if not self.params:
            _refuse("no parameters")
        if state_bits not in (8, 32):
            _refuse("state_bits must be 8 or 32")
        first = self.params[0]
        self.device, self.dtype = first.device, first.dtype
        if self.dtype not in _DTYPES or not first.is_cuda:
            _refuse("parameters must be float32 or bfloat16 tensors on a GPU")
        self.lr, self.betas, self.eps, self.weight_decay = lr, tuple(betas), eps, weight_decay
        self.max_norm, self.state_bits, self.seed, self.step_count = max_norm, state_bits, seed, step_count
        master = master and self.dtype == torch.bfloat16
        kinds = ({"m": torch.float32, "v": torch.float32} if state_bits == 32 else
                 {"m": torch.float8_e4m3fn, "r": torch.float8_e4m3fn, "m_scale": torch.float32, "r_scale": torch.float32})
        if master:
            kinds["master"] = torch.float32
        if states is None:
            states = {k: [p.detach().float() if k == "master" else
                          torch.zeros(-(-p.numel() // 256) if k.endswith("scale") else p.numel(), dtype=t, device=self.device)
                          for p in self.params] for k, t in kinds.items()}
        if set(states) != set(kinds):
            _refuse("states must be %s" % ", ".join(sorted(kinds)))
        self.states = states
        spans = []
        for i, p in enumerate(self.params):
            self._array(p, "parameter", i, p.numel(), self.dtype, spans)
            for k, t in kinds.items():
                if len(states[k]) != len(self.params):
                    _refuse("states: one %s for every parameter" % k)
                self._array(states[k][i], k, i, -(-p.numel() // 256) if k.endswith("scale") else p.numel(), t, spans)
        spans.sort()
        if any(a[1] > b[0] for a, b in zip(spans, spans[1:])):
            _refuse("parameters and states must not overlap")
        self.grad_norm = torch.zeros(1, dtype=torch.float32, device=self.device) if max_norm > 0 else None
        lib = _abi.load()
        self._ws, self._ws_bytes = _workspace(lib.dvi_adamw_workspace_bytes(len(self.params)) if max_norm > 0 else 0, self.device)
        self._table = (_abi.AdamwTensor * len(self.params))()
        self._sizes = [p.numel() for p in self.params]
        for i, (e, p) in enumerate(zip(self._table, self.params)):
            s = {k: v[i].data_ptr() for k, v in states.items()}
            e.param, e.master, e.m, e.v = p.data_ptr(), s.get("master"), s["m"], s["r"] if state_bits == 8 else s["v"]
            e.m_scale, e.v_scale = s.get("m_scale"), s.get("r_scale")

    def _array(self, t, name, i, n, dtype, spans):
        if t.dtype != dtype or t.device != self.device or t.numel() != n or not t.is_contiguous():
            _refuse("%s %d must be a contiguous %s tensor of %d elements on %s" % (name, i, dtype, n, self.device))
        if n:
            spans.append((t.data_ptr(), t.data_ptr() + n * t.element_size()))

    def step(self, grads: Sequence[Optional[torch.Tensor]], lr: Optional[float] = None) -> None:
        """One step: grads holds a contiguous gradient (all fp32, or all bf16) for every parameter, or None
        where a parameter and its states stay as they are."""
        if len(grads) != len(self._sizes):
            _refuse("one gradient for every parameter")
        dtype, dev = None, self.device
        for i, (e, g, n) in enumerate(zip(self._table, grads, self._sizes)):
            if g is None:
                e.n = 0
                continue
            if dtype is None:
                dtype = g.dtype
                if dtype not in _DTYPES:
                    _refuse("gradients must be float32 or bfloat16")
            if g.dtype != dtype or g.device != dev or g.numel() != n or not g.is_contiguous():
                _refuse("gradient %d must be a contiguous %s tensor of %d elements on %s" % (i, dtype, n, dev))
            e.n, e.grad = n, g.data_ptr()
        args = _abi.AdamwArgs(_DTYPES[self.dtype], _DTYPES[dtype or self.dtype], self.state_bits, self.step_count + 1,
                              self.lr if lr is None else lr, self.betas[0], self.betas[1], self.eps, self.weight_decay,
                              self.max_norm, self.seed & 0xFFFFFFFFFFFFFFFF,
                              None if self.grad_norm is None else self.grad_norm.data_ptr())
        _call(dev, _abi.load().dvi_adamw, self._table, len(self._sizes), args,
              self._ws.data_ptr() if self._ws_bytes else None, self._ws_bytes)
        self.step_count += 1
