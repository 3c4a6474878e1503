"""Layer norm, token log-probabilities and distillation in 64 bits (numpy), and bounds on the error of a computation of them in 32.

A bound counts roundings: `U` (2^-24) for each operation that a value goes through, sums by the longest chain of additions that any order
of theirs may have had, and one rounding of the result to its type."""
import numpy as np
import torch

U = 2.0 ** -24
# half the spacing, relative to a value and of the smallest ones
_ROUNDING = {t: (torch.finfo(t).eps / 2, torch.finfo(t).eps * torch.finfo(t).tiny / 2) for t in (torch.float32, torch.float16, torch.bfloat16)}


def f64(t: torch.Tensor) -> np.ndarray:
    return t.detach().cpu().to(torch.float64).numpy()


def rounded(want: np.ndarray, dtype) -> np.ndarray:
    """Bound of one rounding of values near `want` to dtype."""
    rel, least = _ROUNDING[dtype]
    return rel * np.abs(want) * 1.01 + least


def assert_within(got: torch.Tensor, want: np.ndarray, bound: np.ndarray, what: str):
    g = f64(got)
    assert g.shape == want.shape, (what, g.shape, want.shape)
    want = np.where(np.abs(want) > torch.finfo(got.dtype).max * (1 + torch.finfo(got.dtype).eps), np.copysign(np.inf, want), want)      # (beyond the type)
    assert np.array_equal(np.isnan(g), np.isnan(want)), f"{what}: NaN in other places"
    inf = np.isinf(want)
    assert np.array_equal(g[inf], want[inf]), f"{what}: infinities"
    with np.errstate(invalid="ignore"):
        bad = ~inf & ~np.isnan(want) & ~(np.abs(g - want) <= bound)
    i = np.argwhere(bad)
    assert i.size == 0, f"{what}: {len(i)} of {g.size} outside, first at {tuple(i[0])}: got {g[tuple(i[0])]}, want {want[tuple(i[0])]}, " \
                        f"bound {np.broadcast_to(bound, g.shape)[tuple(i[0])]}"


# ---- layer norm ---------------------------------------------------------------------------------------------------------------

def layernorm(x, gamma, beta, eps):
    mean = x.mean(1, keepdims=True)
    rstd = 1.0 / np.sqrt(((x - mean) ** 2).mean(1, keepdims=True) + eps)
    return (x - mean) * rstd * gamma + beta, mean[:, 0], rstd[:, 0]


def layernorm_grad(dy, x, gamma, eps):
    _, mean, rstd = layernorm(x, 1.0, 0.0, eps)
    xh = (x - mean[:, None]) * rstd[:, None]
    g = dy * gamma
    dx = rstd[:, None] * (g - g.mean(1, keepdims=True) - xh * (g * xh).mean(1, keepdims=True))
    return dx, (dy * xh).sum(0), dy.sum(0)


def _chain(cols):
    """Additions that an element of a row's sum goes through at most: 32 of a lane's own, or its share of a long row; the lanes; the wavefronts."""
    return max(32, cols // 1024 + 8) + 12 + 16


def layernorm_bound(x, gamma, beta, eps):
    """Of y before its rounding.  The mean is off by chain * U of the mean magnitude, which the normalisation multiplies by rstd;
    rstd by half of the variance's relative error; then a handful of operations."""
    k = _chain(x.shape[1])
    y, mean, rstd = layernorm(x, gamma, beta, eps)
    xh = np.abs((x - mean[:, None]) * rstd[:, None])
    off = k * U * (np.abs(x).mean(1, keepdims=True) + np.abs(mean[:, None])) * rstd[:, None]
    return np.abs(gamma) * (off + 4 * U * np.abs(x) * rstd[:, None] + xh * (k + 8) * U + xh * off ** 2) + 4 * U * (np.abs(beta) + np.abs(y))


def layernorm_grad_bound(dy, x, gamma, eps):
    n, cols = x.shape
    k = _chain(cols)
    _, mean, rstd = layernorm(x, 1.0, 0.0, eps)
    xh = (x - mean[:, None]) * rstd[:, None]
    dxh = layernorm_bound(x, 1.0, 0.0, eps)
    g = np.abs(dy * gamma)
    mg, mgx = g.mean(1, keepdims=True), (g * np.abs(xh)).mean(1, keepdims=True)
    slip = (g * dxh).mean(1, keepdims=True)
    dx = rstd[:, None] * ((k + 8) * U * (g + mg + 2 * np.abs(xh) * mgx) + np.abs(xh) * slip + dxh * mgx)
    rows = n + 32                                         # additions over the rows, whatever their order
    return dx, rows * U * np.abs(dy * xh).sum(0) + (np.abs(dy) * dxh).sum(0), rows * U * np.abs(dy).sum(0)


# ---- logits -------------------------------------------------------------------------------------------------------------------

def log_softmax(z, scale):
    """log p with 0 * inf nowhere: rows of -inf alone give -inf."""
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        top = z.max(1, keepdims=True)
        d = np.where(np.isneginf(top) & np.isneginf(z), -np.inf, (z - top) * scale)
        s = np.exp(d).sum(1, keepdims=True)
        return np.where(np.isneginf(top), -np.inf, d - np.log(s))


def _plogp(p, lp):
    with np.errstate(invalid="ignore"):
        return np.where(p == 0, 0.0, p * lp)


def token_logprobs(z, tokens, scale, top_k):
    lp = log_softmax(z, scale)
    p = np.exp(lp)
    n, cols = z.shape
    logp = np.array([0.0 if t < 0 else np.nan if t >= cols else lp[r, t] for r, t in enumerate(tokens)])
    order = np.argsort(-z, axis=1, kind="stable")[:, :top_k]
    return logp, -_plogp(p, lp).sum(1), np.take_along_axis(lp, order, 1), order


def token_logprobs_grad(z, tokens, scale, dlogp, dentropy):
    lp = log_softmax(z, scale)
    p = np.exp(lp)
    h = -_plogp(p, lp).sum(1, keepdims=True)
    n, cols = z.shape
    out = -dentropy[:, None] * (_plogp(p, lp) + p * h)
    empty = np.isneginf(z).all(1)
    for r, t in enumerate(tokens):
        if empty[r]:
            out[r] = 0.0
        elif t >= cols and dlogp[r] is not None:
            out[r] = np.nan
        elif t >= 0:
            out[r] -= dlogp[r] * p[r]
            out[r, t] += dlogp[r]
    return out * scale


def distill(z, teacher, index, scale):
    """(loss, dense teacher probabilities)"""
    lp = log_softmax(z, scale)
    n, cols = z.shape
    loss, q_all = np.zeros(n), np.zeros((n, cols))
    for r in range(n):
        if (index[r] >= cols).any() or np.isnan(teacher[r][index[r] >= 0]).any():
            loss[r], q_all[r] = np.nan, np.nan
            continue
        t = np.where(index[r] >= 0, teacher[r], -np.inf)
        lq = log_softmax(t[None], scale)[0]
        for i in np.flatnonzero(~np.isneginf(lq)):
            q = np.exp(lq[i])
            loss[r] += q * (lq[i] - lp[r, index[r, i]])
            q_all[r, index[r, i]] += q
    return loss, q_all


def distill_grad(z, teacher, index, scale, weight):
    _, q = distill(z, teacher, index, scale)
    p = np.exp(log_softmax(z, scale))
    live = (weight != 0) & ~np.isneginf(z).all(1) & (np.isnan(q).any(1) | (q.sum(1) > 0))
    with np.errstate(invalid="ignore"):
        return np.where(live[:, None], weight[:, None] * scale * (p - q), 0.0)


def logits_bound(z, scale):
    """(relative bound of a probability of every column, absolute one of its logarithm).  The difference to the maximum and its product with
    the scale (which is rounded itself) are off by 3 U of the difference, the exponential by 2 U; the sum by as many roundings as a lane adds
    elements of a row, and the lanes; the logarithm by 2 U of its value."""
    cols = z.shape[1]
    with np.errstate(invalid="ignore"):
        top = z.max(1, keepdims=True)
        d = np.where(np.isfinite(z) & np.isfinite(top), np.abs(z - top) * scale, 0.0)
    lp = log_softmax(z, scale)
    p = np.exp(np.where(np.isnan(lp), -np.inf, lp))
    chain = cols // 256 + 64 + 32
    total = U * (chain + 8 + 4 * (p * d).sum(1, keepdims=True) + 2 * np.log(cols + 1.0))
    return total + U * (6 * d + 6), total + U * (6 * d + 4)
