"""What a language model has around its quantized linears: the norm in front of one, and what is done with the logits of the last.

`LayerNorm`, `TokenLogProbs` and `Distillation` own the device buffers of one operator each and call the C ABI of ``qsync.py``; all
arithmetic runs inside libqsync's kernels.  Buffers are allocated once in the constructor for up to `rows` rows: a call on fewer
rows returns the leading part of them, a later call overwrites what an earlier one returned, and nothing is allocated or synchronised.
Like the linear operators, a call runs on `stream` or torch's current stream; tensors that another stream writes or frees are the
caller's to order.

    norm, head, loss = LayerNorm(T, C), QLinear(Q.INT8, T, V, C, ...), Distillation(T, V, k, ...)
    losses, dlogits = loss.forward_backward(head.forward(norm.forward(x, gamma, beta), w), teacher_logp, teacher_index, weight)
    dhidden, dw, _ = head.backward(dlogits)
    dx, dgamma, dbeta = norm.backward(dhidden)
"""
from __future__ import annotations

from typing import Optional

import torch

from . import qsync as Q
from .operator import _scratch

_FLOATS = (torch.float32, torch.float16, torch.bfloat16)
# The checks of the binding: an input's rows (-> its leading dimension), packed matrices and (0 columns) vectors of a kind of elements
_check_rows, _check_packed = Q._native.check_rows, Q._native.check_packed
_FLOAT32, _ANY_FLOAT, _INTEGER = 1, 2, 4


def _float_type(dtype, what: str) -> None:
    if dtype not in _FLOATS:
        raise ValueError(f"{what}: float32, float16 or bfloat16, not {dtype}")


def _sizes(rows: int, cols: int) -> None:
    if rows < 0 or cols < 1:
        raise ValueError("rows must not be negative, cols must be positive")


def _gpu(device) -> int:
    """The index of the GPU that buffers on `device` are on; -1: they are on none, and every call is refused."""
    d = torch.device(device)
    if d.type != "cuda":
        return -1
    return torch.cuda.current_device() if d.index is None else d.index


class LayerNorm:
    """Layer norm over `cols` columns; the weights are handed to `forward`, as a linear operator's are."""

    def __init__(self, rows: int, cols: int, x_dtype=torch.float16, y_dtype=None, dx_dtype=None, eps: float = 1e-5, training: bool = True,
                 collect_y_amax: bool = False, device="cuda"):
        """y_dtype, dx_dtype: x_dtype unless given.  training=False: no buffers for `backward`.  collect_y_amax: `y_amax` collects max |y|
        for an INT8 linear that takes y as its input (`QLinear.forward(y, w, x_amax=norm.y_amax)`, which leaves it at zero)."""
        _sizes(rows, cols)
        y_dtype, dx_dtype = y_dtype or x_dtype, dx_dtype or x_dtype
        for what, dt in (("x_dtype", x_dtype), ("y_dtype", y_dtype), ("dx_dtype", dx_dtype)):
            _float_type(dt, what)
        self.rows, self.cols, self.eps, self.device = rows, cols, float(eps), _gpu(device)
        e = lambda *s, dt=torch.float32: torch.empty(*s, dtype=dt, device=device)
        self.y = e(rows, cols, dt=y_dtype)
        self.y_amax = torch.zeros(1, dtype=torch.float32, device=device) if collect_y_amax else None
        self.training = training
        self._saved = self.mean = self.rstd = None
        if training:
            self.mean, self.rstd = e(rows), e(rows)
            self.dx, self.dgamma, self.dbeta = e(rows, cols, dt=dx_dtype), e(cols), e(cols)
            self.ws = _scratch(Q.qsync_layernorm_bwd_workspace_bytes(rows, cols), device)

    def forward(self, x: torch.Tensor, gamma: Optional[torch.Tensor] = None, beta: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """x [n <= rows, cols], rows at any stride; gamma, beta: float32 or None (1 and 0).  `backward` reads x and gamma again."""
        cols, device = self.cols, self.device
        ld = _check_rows(x, self.rows, cols, device, "x")
        _check_packed(gamma, cols, 0, _FLOAT32, device, "gamma")
        _check_packed(beta, cols, 0, _FLOAT32, device, "beta")
        n = x.shape[0]
        if n:      # (a tensor without elements has no address)
            Q.qsync_layernorm_fwd(x, n, cols, ld, gamma, beta, self.eps, self.y, self.mean, self.rstd, self.y_amax, stream)
        if self.training:
            self._saved = (x, gamma, ld)
        return self.y if n == self.rows else self.y[:n]

    def backward(self, dy: torch.Tensor, stream=None):
        """(dx, dgamma, dbeta) of the last `forward`; dy [n, cols] of the same number of rows."""
        if self._saved is None:
            raise RuntimeError("backward without a forward of an operator with training=True")
        x, gamma, ldx = self._saved
        n = x.shape[0]
        lddy = _check_rows(dy, n, self.cols, self.device, "dy")
        if dy.shape[0] != n:
            raise ValueError(f"dy has {dy.shape[0]} rows, the forward pass had {n}")
        dx = self.dx if n == self.rows else self.dx[:n]
        if n == 0:      # zeros, on the call's stream; the empty tensors have no address, and any will do
            one = self.dgamma
            Q.qsync_layernorm_bwd(one, self.cols, one, 0, self.cols, self.cols, gamma, one, one, None, self.dgamma, self.dbeta, None, stream)
            return dx, self.dgamma, self.dbeta
        Q.qsync_layernorm_bwd(dy, lddy, x, n, self.cols, ldx, gamma, self.mean, self.rstd, dx, self.dgamma, self.dbeta, self.ws, stream)
        return dx, self.dgamma, self.dbeta


class TokenLogProbs:
    """Log probabilities of given tokens, with the entropy and the top alternatives of every position, and their gradient."""

    def __init__(self, rows: int, cols: int, top_k: int = 0, entropy: bool = True, scale: float = 1.0, dlogits_dtype=None, device="cuda"):
        """scale: 1 / temperature.  top_k: alternatives of a position, 0 to 64.  dlogits_dtype: the type of `backward`'s result; None: no
        buffer for it (`backward` then needs `out`)."""
        _sizes(rows, cols)
        if not 0 <= top_k <= min(64, cols):
            raise ValueError("top_k must lie between 0 and 64 and not exceed cols")
        self.rows, self.cols, self.top_k, self.scale, self.device = rows, cols, top_k, float(scale), _gpu(device)
        e = lambda *s, dt=torch.float32: torch.empty(*s, dtype=dt, device=device)
        self.logp, self.stats = e(rows), e(rows, 2)
        self.entropy = e(rows) if entropy else None
        self.top_logp, self.top_index = (e(rows, top_k), e(rows, top_k, dt=torch.int32)) if top_k else (None, None)
        if dlogits_dtype is not None:
            _float_type(dlogits_dtype, "dlogits_dtype")
        self.dlogits = e(rows, cols, dt=dlogits_dtype) if dlogits_dtype is not None else None
        self._saved = None
        self.ws = _scratch(max(Q.qsync_token_logprobs_workspace_bytes(t, rows, cols, top_k) for t in (Q.F32, Q.F16)), device)

    def forward(self, logits: torch.Tensor, tokens: Optional[torch.Tensor] = None, stream=None):
        """(logp, entropy, top_logp, top_index), each None where it is not wanted (logp: without tokens).  logits [n <= rows, cols], rows at
        any stride; tokens: n of int64 or int32, negative where a position has none.  `backward` reads logits and tokens again."""
        ld = _check_rows(logits, self.rows, self.cols, self.device, "logits")
        n = logits.shape[0]
        _check_packed(tokens, n, 0, _INTEGER, self.device, "tokens")
        logp = self.logp if tokens is not None else None
        if n:      # (a tensor without elements has no address)
            Q.qsync_token_logprobs(logits, n, self.cols, ld, self.scale, tokens, logp, self.entropy, self.stats, self.top_k, self.top_logp,
                                   self.top_index, self.ws, stream)
        self._saved = (logits, tokens, ld)
        if n == self.rows:
            return logp, self.entropy, self.top_logp, self.top_index
        return _first(logp, n), _first(self.entropy, n), _first(self.top_logp, n), _first(self.top_index, n)

    def backward(self, dlogp: Optional[torch.Tensor] = None, dentropy: Optional[torch.Tensor] = None, stream=None,
                 out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Gradient of sum(dlogp * logp + dentropy * entropy) of the last `forward`; dlogp, dentropy: n of float32, either may be None.
        out: packed [n, cols], may be the logits themselves."""
        if self._saved is None:
            raise RuntimeError("backward without a forward")
        logits, tokens, ld = self._saved
        n = logits.shape[0]
        if dlogp is None and dentropy is None:
            raise ValueError("dlogp or dentropy is needed")
        if dlogp is not None and tokens is None:
            raise ValueError("dlogp needs a forward with tokens")
        if dentropy is not None and self.entropy is None:
            raise ValueError("dentropy needs an operator with entropy=True")
        _check_packed(dlogp, n, 0, _FLOAT32, self.device, "dlogp")
        _check_packed(dentropy, n, 0, _FLOAT32, self.device, "dentropy")
        out = _output(self, out, n)
        if n:
            Q.qsync_token_logprobs_bwd(logits, n, self.cols, ld, self.scale, tokens, self.stats, None if dentropy is None else self.entropy,
                                       dlogp, dentropy, out, stream)
        return out


class Distillation:
    """Distillation from a teacher's top logits: the loss of every position, and the gradient of their weighted sum."""

    def __init__(self, rows: int, cols: int, k: int, scale: float = 1.0, dlogits_dtype=None, device="cuda"):
        """k: the teacher's entries of a position, 1 to 256.  scale: 1 / temperature.  dlogits_dtype: the type of the gradient; None: no
        buffer for it (`forward_backward` then needs `out`)."""
        _sizes(rows, cols)
        if not 1 <= k <= 256:
            raise ValueError("k must lie between 1 and 256")
        self.rows, self.cols, self.k, self.scale, self.device = rows, cols, k, float(scale), _gpu(device)
        if dlogits_dtype is not None:
            _float_type(dlogits_dtype, "dlogits_dtype")
        self.loss = torch.empty(rows, dtype=torch.float32, device=device)
        self.dlogits = torch.empty(rows, cols, dtype=dlogits_dtype, device=device) if dlogits_dtype is not None else None
        self.ws = _scratch(max(Q.qsync_distill_topk_workspace_bytes(t, rows, cols) for t in (Q.F32, Q.F16)), device)

    def _run(self, logits, teacher, index, weight, out, stream) -> torch.Tensor:
        device = self.device
        ld = _check_rows(logits, self.rows, self.cols, device, "logits")
        n = logits.shape[0]
        _check_packed(teacher, n, self.k, _ANY_FLOAT, device, "teacher")
        _check_packed(index, n, self.k, _INTEGER, device, "index")
        _check_packed(weight, n, 0, _FLOAT32, device, "weight")
        if n:      # (a tensor without elements has no address)
            Q.qsync_distill_topk(logits, n, self.cols, ld, self.scale, teacher, index, self.k, weight, self.loss, out, self.ws, stream)
        return self.loss if n == self.rows else self.loss[:n]

    def forward(self, logits: torch.Tensor, teacher: torch.Tensor, index: torch.Tensor, stream=None) -> torch.Tensor:
        """The losses alone.  logits [n <= rows, cols], rows at any stride; teacher [n, k] logits or log probabilities, index [n, k] their
        columns (int32 or int64, negative: no entry), e.g. top_logp and top_index of a `TokenLogProbs`."""
        return self._run(logits, teacher, index, None, None, stream)

    def forward_backward(self, logits: torch.Tensor, teacher: torch.Tensor, index: torch.Tensor, weight: Optional[torch.Tensor] = None,
                         stream=None, out: Optional[torch.Tensor] = None):
        """(loss, dlogits): the losses and the gradient of sum(weight * loss).  weight: n of float32, or None (1).  out: packed [n, cols],
        may be the logits themselves."""
        out = _output(self, out, logits.shape[0])
        return self._run(logits, teacher, index, weight, out, stream), out


def _first(t: Optional[torch.Tensor], n: int) -> Optional[torch.Tensor]:
    return None if t is None else t[:n]


def _output(op, out: Optional[torch.Tensor], n: int) -> torch.Tensor:
    if out is None:
        if op.dlogits is None:
            raise ValueError("an operator without dlogits_dtype needs `out`")
        return op.dlogits if n == op.rows else op.dlogits[:n]
    _check_packed(out, n, op.cols, _ANY_FLOAT, op.device, "out")
    return out
