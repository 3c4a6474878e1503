"""INT8 linear operators with a scale for each token, and the experts' layers that are made of them.

`TokenLinear` is the linear operator of ``operator.py`` with a scale for each row of the activation and of the gradient instead of one for the
whole of it, so that a wide token costs no other its bits; its backward passes are INT8 products too.  `ExpertRoute` sorts a batch's tokens
by the experts that a router gave them, gathers their rows and combines the experts' rows again; `ExpertLinear` is the `TokenLinear` of the
sorted rows, a weight matrix for each expert.  As in ``head.py``, buffers are allocated once, for up to `rows` rows or `tokens` tokens: a call on
fewer returns the leading part of them, a later call overwrites what an earlier one returned, nothing is allocated or synchronised, and
calls run on `stream` or torch's current stream.

    route = ExpertRoute(T, k, E, C)
    up, down = ExpertLinear(T * k, F, C, E), ExpertLinear(T * k, C, F, E, gather=False)
    route.sort(ids)                                                      # ids, weight [T, k]: the router's
    h = activation(up.forward(x, route, w=w_up))
    y = route.combine(down.forward(h, route, w=w_down), weight)
    dz, dweight = route.combine_backward(dy)
    dh, dw_down, _ = down.backward(dz)
    drows, dw_up, _ = up.backward(activation_backward(dh))
    dx = route.gather_backward(drows)
"""
from __future__ import annotations

from typing import Optional

import torch

from . import qsync as Q
from .head import _ANY_FLOAT, _FLOAT32, _INTEGER, _check_packed, _check_rows, _float_type, _gpu
from .operator import _scratch


_on_device = Q._native.check_device      # a kernel runs on the current device, and its buffers have to be there


class ExpertRoute:
    """Tokens to the experts that a router gave them, and back."""

    def __init__(self, tokens: int, k: int, experts: int, cols: Optional[int] = None, dtype=torch.float16, training: bool = True, device="cuda"):
        """k: experts of a token.  cols, dtype: of the buffers that `gather`, `combine` and their backward passes return; without cols, `sort`
        alone.  training=False: no buffers for the backward passes."""
        if tokens < 0 or not 1 <= k or not 1 <= experts <= 512:
            raise ValueError("tokens must not be negative, k must be positive, experts must lie between 1 and 512")
        if tokens * k > 1 << 23:
            raise ValueError("at most 2^23 rows: tokens times k")
        if cols is not None and cols < 1:
            raise ValueError("cols must be positive")
        _float_type(dtype, "dtype")
        self.tokens, self.k, self.experts, self.cols, self.training, self.device = tokens, k, experts, cols, training, _gpu(device)
        e = lambda *s, dt=torch.int32: torch.empty(*s, dtype=dt, device=device)
        self.offsets, self.source, self.slot = e(experts + 1), e(tokens * k), e(tokens, k)
        self.count = self.offsets[experts:]                    # the rows that have an expert
        self.ws = _scratch(Q.qsync_expert_sort_workspace_bytes(tokens * k, experts), device)
        if cols is not None:
            self.rows_out, self.y = e(tokens * k, cols, dt=dtype), e(tokens, cols, dt=dtype)
            if training:
                self.dz, self.dweight, self.dx = e(tokens * k, cols, dt=dtype), e(tokens, k, dt=torch.float32), e(tokens, cols, dt=dtype)
        self.n, self._rows_of_sort = None, -1                  # tokens and rows of the last sort
        self.sorts = 0
        self._saved = None

    @property
    def rows(self) -> int:
        """Rows of the last `sort`: its tokens times k.  Those from `offsets[experts]` on belong to no expert."""
        if self.n is None:
            raise RuntimeError("a route without a sort")
        return self._rows_of_sort

    def sort(self, ids: torch.Tensor, stream=None) -> torch.Tensor:
        """offsets [experts + 1] (int32): expert e has the rows offsets[e] .. offsets[e+1]-1, in the order of its entries in ids.  ids [n <= tokens, k] of
        int64 or int32; an entry outside of 0 .. experts-1 has no expert.  Also left: `source`, the entry of every row, and `slot`, the row
        of every entry or -1."""
        _on_device(self.device)
        n = len(ids)
        if n > self.tokens:
            raise ValueError(f"ids: at most {self.tokens} tokens expected")
        _check_packed(ids, n, self.k, _INTEGER, self.device, "ids")
        if n:
            Q.qsync_expert_sort(ids, n, self.k, self.experts, self.offsets, self.source, self.slot, self.ws, stream)
        else:      # (a tensor without elements has no address, and any will do)
            Q.qsync_expert_sort(self.offsets, 0, self.k, self.experts, self.offsets, self.offsets, self.offsets, self.ws, stream)
        self.n, self._rows_of_sort, self._saved = n, n * self.k, None
        self.sorts += 1
        return self.offsets

    def gather(self, x: torch.Tensor, stream=None) -> torch.Tensor:
        """The tokens' rows in the experts' order, [rows, cols]; x [n, cols] of the route's dtype, rows at any stride.  Rows that belong to no
        expert are left as they were."""
        ld, n = self._tokens(x, "x"), self.n
        out = self.rows_out
        if x.dtype != out.dtype:
            raise ValueError(f"x: {out.dtype} expected, not {x.dtype}")
        if n:
            Q.qsync_expert_gather(x, n, self.cols, ld, self.source, self.k, self._rows_of_sort, self.count, out, stream)
        return out if n == self.tokens else out[:self._rows_of_sort]

    def gather_backward(self, drows: torch.Tensor, stream=None) -> torch.Tensor:
        """The tokens' gradient, [n, cols]: the sum of their rows'."""
        self._training()
        ld, n = self._rows(drows, "drows"), self.n
        if n:
            Q.qsync_expert_combine(drows, self._rows_of_sort, self.cols, ld, self.slot, n, self.k, None, self.dx, stream)
        return self.dx if n == self.tokens else self.dx[:n]

    def combine(self, z: torch.Tensor, weight: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """[n, cols]: the sum of the tokens' rows in z [rows, cols], times weight [n, k] (float32) or 1.  `combine_backward` reads both again."""
        ld, n = self._rows(z, "z"), self.n
        _check_packed(weight, n, self.k, _FLOAT32, self.device, "weight")
        if n:
            Q.qsync_expert_combine(z, self._rows_of_sort, self.cols, ld, self.slot, n, self.k, weight, self.y, stream)
        self._saved = (z, ld, weight)
        return self.y if n == self.tokens else self.y[:n]

    def combine_backward(self, dy: torch.Tensor, stream=None):
        """(dz [rows, cols], dweight [n, k]) of the last `combine`; dy [n, cols].  Rows that belong to no expert are left as they were."""
        self._training()
        lddy, n = self._tokens(dy, "dy"), self.n
        if self._saved is None:
            raise RuntimeError("combine_backward without a combine since the last sort")
        z, ld, weight = self._saved
        if n:
            Q.qsync_expert_combine_bwd(dy, n, self.cols, lddy, z, self._rows_of_sort, ld, self.slot, self.k, weight, self.dz, self.dweight, stream)
        if n == self.tokens:
            return self.dz, self.dweight
        return self.dz[:self._rows_of_sort], self.dweight[:n]

    def _training(self) -> None:
        if not self.training:
            raise RuntimeError("a backward pass of a route with training=False")

    def _check(self, t: torch.Tensor, rows: int, name: str) -> int:
        """The leading dimension of a matrix of the sorted batch."""
        _on_device(self.device)
        if self.n is None:
            raise RuntimeError("a route without a sort")
        if self.cols is None:
            raise ValueError("a route without cols only sorts")
        ld = _check_rows(t, rows, self.cols, self.device, name)
        if len(t) != rows:
            raise ValueError(f"{name} has {len(t)} rows, the sorted batch {rows}")
        return ld

    def _tokens(self, t: torch.Tensor, name: str) -> int:
        return self._check(t, self.n or 0, name)

    def _rows(self, t: torch.Tensor, name: str) -> int:
        return self._check(t, self._rows_of_sort, name)


class _CodeLinear:
    """Buffers and calls of `TokenLinear` (one set of rows and weights) and `ExpertLinear` (one for each expert)."""

    def __init__(self, rows, N, K, sets, routed, x_dtype, y_dtype, dx_dtype, dw_dtype, dy_round, philox_seed, bias, training, device):
        y_dtype, dx_dtype = y_dtype or x_dtype, dx_dtype or x_dtype
        for what, dt in (("x_dtype", x_dtype), ("y_dtype", y_dtype), ("dx_dtype", dx_dtype), ("dw_dtype", dw_dtype)):
            _float_type(dt, what)
        if rows < 0 or N < 1 or K < 1:
            raise ValueError("rows must not be negative, N and K must be positive")
        if rows > 1 << 23 or N > 1 << 20 or K > 1 << 20 or sets * N > 1 << 23:
            raise ValueError("at most 2^23 rows, 2^20 features, and 2^23 rows of all the weights")
        if dy_round not in (Q.ROUND_NEAREST, Q.ROUND_STOCHASTIC):
            raise ValueError("dy_round: ROUND_NEAREST or ROUND_STOCHASTIC")
        self.rows, self.N, self.K, self.sets, self.training, self.device = rows, N, K, sets, training, _gpu(device)
        self.dy_round, self.seed, self.offset = dy_round, philox_seed, 0
        e = lambda *s, dt=torch.float32: torch.empty(*s, dtype=dt, device=device)
        i8, pad = torch.int8, Q.qsync_token_code_cols
        self.xq, self.sx = e(rows, pad(K), dt=i8), e(rows)
        self.wq, self.sw = e(sets * N, pad(K), dt=i8), e(sets * N)
        self.bias = torch.zeros(*((sets, N) if routed else (N,)), dtype=torch.float32, device=device) if bias else None
        self.y = e(rows, N, dt=y_dtype)
        self.ws = _scratch(0 if routed else Q.qsync_token_linear_workspace_bytes(rows, N, K, sets), device)      # (of K splits, which the experts' have none of)
        self._converted, self._saved = False, None
        if not training:
            return
        positions = Q.qsync_token_code_rows(rows, sets, routed)
        self.wqT, self.swc = e(Q.qsync_token_code_rows(sets * N, sets, False) * K, dt=i8), e(sets, K)
        self.xqT, self.sxc = e(positions * K, dt=i8), e(sets, K)
        self.dyq, self.sdy = e(rows, pad(N), dt=i8), e(rows)
        self.dyqT, self.sdyc = e(positions * N, dt=i8), e(sets, N)
        self.dx, self.dw = e(rows, K, dt=dx_dtype), e(*((sets, N, K) if routed else (N, K)), dt=dw_dtype)
        self.db = e(*((sets, N) if routed else (N,))) if bias else None
        self.ws_x = _scratch(max(Q.qsync_token_quantize_both_workspace_bytes(rows, c, sets, routed) for c in (N, K)), device)
        self.ws_w = _scratch(Q.qsync_token_quantize_both_workspace_bytes(sets * N, K, sets, False), device)
        self.ws_bwd = _scratch(0 if routed else Q.qsync_token_linear_bwd_workspace_bytes(rows, N, K, sets), device)

    def _weights(self, w) -> torch.Tensor:
        if not isinstance(w, torch.Tensor) or w.shape != self.dw_shape:
            raise ValueError(f"w: {list(self.dw_shape)} expected")
        w = w.flatten(0, -2) if w.dim() > 2 and w.is_contiguous() else w
        _check_packed(w, self.sets * self.N, self.K, _ANY_FLOAT, self.device, "w")
        return w

    def convert_w(self, w: torch.Tensor, stream=None) -> None:
        """The codes of the weights, which `forward` and `backward` use until the next conversion."""
        _on_device(self.device)
        w = self._weights(w)
        rows, K = self.sets * self.N, self.K
        if self.training:
            Q.qsync_token_quantize_both(w, rows, K, K, None, 1, rows, self.sets, None, Q.ROUND_NEAREST, 0, 0, self.sw, self.wq, self.swc, self.wqT,
                                        None, self.ws_w, stream)
        else:
            Q.qsync_token_quantize(w, rows, K, K, None, 1, rows, None, Q.ROUND_NEAREST, 0, 0, self.sw, self.wq, stream)
        self._converted = True

    def _forward(self, x, x_rows, ld, w, source, group, n, offsets, stream):
        if w is not None and (not self.training or not n):
            self.convert_w(w, stream)
            w = None
        if w is None and not self._converted:
            raise RuntimeError("forward without weights: w, or convert_w before it")
        if not n:      # (a tensor without elements has no address)
            pass
        elif self.training:
            if w is not None:
                Q.qsync_token_convert(x, x_rows, self.K, ld, source, group, n, self.sets, offsets, self.sx, self.xq, self.sxc, self.xqT,
                                      self._weights(w), self.N, self.sw, self.wq, self.swc, self.wqT, self.ws_x, self.ws_w, stream)
                self._converted = True
            else:
                Q.qsync_token_quantize_both(x, x_rows, self.K, ld, source, group, n, self.sets, offsets, Q.ROUND_NEAREST, 0, 0, self.sx, self.xq,
                                            self.sxc, self.xqT, None, self.ws_x, stream)
            Q.qsync_token_linear_fwd(n, self.N, self.K, self.sets, offsets, self.xq, self.sx, self.wq, self.sw, self.bias, self.y, self.ws, stream)
        else:
            Q.qsync_token_linear(x, x_rows, self.K, ld, source, group, n, self.N, self.sets, offsets, self.wq, self.sw, self.bias, self.y, self.sx,
                                 self.xq, self.ws, stream)
        return self.y if n == self.rows else self.y[:n]

    def _backward(self, dy, n, offsets, stream):
        N, K, sets = self.N, self.K, self.sets
        lddy = _check_rows(dy, n, N, self.device, "dy")
        if dy.shape[0] != n:
            raise ValueError(f"dy has {dy.shape[0]} rows, the forward pass had {n}")
        some = dy if n else self.dw            # (a tensor without elements has no address, and any will do)
        at = lambda t: t if n else self.dw
        Q.qsync_token_quantize_both(some, n, N, lddy, None, 1, n, sets, offsets, self.dy_round, self.seed, self.offset, at(self.sdy), at(self.dyq),
                                    self.sdyc, at(self.dyqT), self.db, self.ws_x, stream)
        if self.dy_round == Q.ROUND_STOCHASTIC:
            self.offset += n * ((N + 7) // 8)
        if n:
            Q.qsync_token_linear_bwd(n, N, K, sets, offsets, self.dyq, self.sdy, self.wqT, self.swc, self.dyqT, self.sdyc, self.xqT, self.sxc, self.dx,
                                     self.dw, self.ws_bwd, stream)
        else:
            Q.qsync_token_linear_wgrad(0, N, K, sets, offsets, self.dw, self.sdyc, self.dw, self.sxc, self.dw, self.ws_bwd, stream)
        return self.dx if n == self.rows else self.dx[:n], self.dw, self.db

    def _check_backward(self) -> None:
        _on_device(self.device)
        if self._saved is None:
            raise RuntimeError("backward without a forward of an operator with training=True")


class TokenLinear(_CodeLinear):
    """y = x w^T + b in 8-bit integers, with a scale for each token of x and each channel of w.  Sums are of 32 bits, as `QLinear`'s: exact for
    contractions of up to 133144, over K, N and, in the weight gradient, the rows of a set."""

    def __init__(self, rows: int, N: int, K: int, x_dtype=torch.float16, y_dtype=None, dx_dtype=None, dw_dtype=torch.float32,
                 dy_round: int = Q.ROUND_STOCHASTIC, philox_seed: int = 0, bias: bool = True, training: bool = True, device="cuda"):
        """x_dtype: the default of y_dtype and dx_dtype (x, w and dy may have any of the three types in any call).  dy_round: of the gradient's
        codes.  training=False: no buffers for `backward`; x is then read once in a forward pass instead of twice."""
        self.dw_shape = (N, K)
        super().__init__(rows, N, K, 1, False, x_dtype, y_dtype, dx_dtype, dw_dtype, dy_round, philox_seed, bias, training, device)

    def forward(self, x: torch.Tensor, w: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """x [n <= rows, K], rows at any stride; w [N, K], or None: the weights that `convert_w` was given last.  `backward` reads neither."""
        _on_device(self.device)
        ld = _check_rows(x, self.rows, self.K, self.device, "x")
        n = len(x)
        y = self._forward(x, n, ld, w, None, 1, n, None, stream)
        if self.training:
            self._saved = n
        return y

    def backward(self, dy: torch.Tensor, stream=None):
        """(dx, dw, db) of the last `forward`, db None without a bias; dy [n, N] of the same number of rows."""
        self._check_backward()
        return self._backward(dy, self._saved, None, stream)


class ExpertLinear(_CodeLinear):
    """The `TokenLinear` of every expert on the rows that a route sorted to it."""

    def __init__(self, rows: int, N: int, K: int, experts: int, x_dtype=torch.float16, y_dtype=None, dx_dtype=None, dw_dtype=torch.float32,
                 dy_round: int = Q.ROUND_STOCHASTIC, philox_seed: int = 0, bias: bool = False, gather: bool = True, training: bool = True,
                 device="cuda"):
        """rows: tokens times k.  gather: x holds the tokens, whose rows the operator takes through the route; False: x holds the sorted rows.  dx
        is the gradient of the sorted rows either way (`ExpertRoute.gather_backward` makes the tokens' of it)."""
        if not 1 <= experts <= 512:
            raise ValueError("experts must lie between 1 and 512")
        self.dw_shape, self.gather = (experts, N, K), gather
        super().__init__(rows, N, K, experts, True, x_dtype, y_dtype, dx_dtype, dw_dtype, dy_round, philox_seed, bias, training, device)

    def forward(self, x: torch.Tensor, route: ExpertRoute, w: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """[route.rows, N], sorted; rows that belong to no expert are left as they were.  x [tokens of the sort, K] (gather=False: [route.rows, K]), rows
        at any stride; w [experts, N, K], or None: the weights that `convert_w` was given last."""
        _on_device(self.device)
        n = route.rows
        if route.experts != self.sets or route.device != self.device or n > self.rows:
            raise ValueError(f"a route of {self.sets} experts and at most {self.rows} rows on the operator's GPU expected")
        have = route.n if self.gather else n
        ld = _check_rows(x, have, self.K, self.device, "x")
        if x.shape[0] != have:
            raise ValueError(f"x has {x.shape[0]} rows, {have} expected")
        y = self._forward(x, have, ld, w, route.source if self.gather else None, route.k if self.gather else 1, n, route.offsets, stream)
        if self.training:
            self._saved = (route, route.sorts, n)
        return y

    def backward(self, dy: torch.Tensor, stream=None):
        """(dx [rows, K], dw [experts, N, K], db) of the last `forward`, db [experts, N] or None without a bias; dy [rows, N], sorted.  The route must not
        have sorted another batch since.  An expert without rows has a gradient of zeros."""
        self._check_backward()
        route, sorts, n = self._saved
        if route.sorts != sorts:
            raise RuntimeError("the route has sorted another batch since the forward pass")
        return self._backward(dy, n, route.offsets, stream)
