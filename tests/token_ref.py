"""INT8 linear operators with a scale for each token, and routing to experts, in numpy: codes and scales as they are defined (their
divisions and products rounded to 32 bits), everything behind them in 64 bits, and bounds that count the roundings of 32-bit epilogues and sums."""
import numpy as np

from oracle.qsync_oracle import philox4x32_10
from tests.head_ref import U

TINY = 2.0 ** -100


def draws(rows: int, cols: int, seed: int, offset: int) -> np.ndarray:
    """The 16-bit draws of stochastic rounding: a block of counters for each eight elements of a row, rows one behind the other."""
    per_row = (cols + 7) // 8
    n = np.array([offset + i for i in range(rows * per_row)], dtype=object)
    counter = np.stack([(n >> s) & 0xFFFFFFFF for s in (0, 32, 64, 96)], 1).astype(np.uint32)
    words = philox4x32_10(counter, (seed & 0xFFFFFFFF, seed >> 32)).astype(np.int64)
    return np.stack([words & 0xFFFF, words >> 16], 2).reshape(rows, per_row * 8)[:, :cols]


def codes(x: np.ndarray, axis: int, u=None):
    """(codes int64, scales float32) with a scale for each slice along `axis`; x holds values of 32 bits at most."""
    x = x.astype(np.float32)
    with np.errstate(all="ignore"):
        top = np.abs(x).max(axis, keepdims=True)                     # (NaN where there is one)
        finite, some = np.isfinite(top), top >= np.float32(TINY)
        safe = np.where(finite & some, top, np.float32(1.0))
        scale = np.where(finite, np.where(some, safe / np.float32(127.0), np.float32(1.0)), np.float32(np.nan)).astype(np.float32)
        v = np.where(finite & some, x * (np.float32(127.0) / safe), np.float32(0.0)).astype(np.float32)
    if u is None:
        q = np.rint(v)
    else:
        down = np.floor(v)
        q = down + (u < np.floor((v - down).astype(np.float32) * np.float32(65536.0)))      # (the difference in 32 bits, as in the oracle)
    return np.clip(q, -127, 127).astype(np.int64), np.squeeze(scale, axis)


def product(a, sa, b, sb, bias=None):
    """(Y, bound of a 32-bit epilogue): a [M, K], b [N, K] codes.  float(acc) is one rounding, the fused multiply-add another; sa sb is a
    32-bit product in the definition."""
    acc = (a.astype(np.float64) @ b.astype(np.float64).T)            # (exact: below 2^53)
    with np.errstate(all="ignore"):
        f = (sa.astype(np.float32)[:, None] * sb.astype(np.float32)[None, :]).astype(np.float64)
        y = acc * f
        bound = U * np.abs(y)
        if bias is not None:
            y = y + bias[None, :]
        return y, (bound + U * np.abs(y)) * 1.01 + 2.0 ** -149


def sort(ids: np.ndarray, experts: int):
    """(offsets, source, slot) of int32."""
    flat = ids.reshape(-1)
    here = np.flatnonzero((flat >= 0) & (flat < experts))
    source = here[np.argsort(flat[here], kind="stable")]
    slot = np.full(flat.size, -1)
    slot[source] = np.arange(source.size)
    counts = np.bincount(flat[here].astype(np.int64), minlength=experts)
    return np.concatenate([[0], np.cumsum(counts)]).astype(np.int32), source.astype(np.int32), slot.reshape(ids.shape).astype(np.int32)


def pad(n: int) -> int:
    return (n + 127) // 128 * 128


def transposed_layout(q: np.ndarray, bounds, with_offsets: bool):
    """Where the codes along the rows lie: {set: (start, [cols, pad(len)])}; q [rows, cols], bounds the sets' first rows and the end."""
    out = {}
    for e, (a, b) in enumerate(zip(bounds[:-1], bounds[1:])):
        start = pad(a) + 128 * e if with_offsets else pad(b - a) * e
        m = np.zeros((q.shape[1], pad(b - a)), np.int64)
        m[:, :b - a] = q[a:b].T
        out[e] = (start * q.shape[1], m)
    return out


def assert_within(got, want: np.ndarray, bound: np.ndarray, what: str):
    """As head_ref's, but exact where a type ends: rounding to nearest makes an infinity of everything from the largest value plus half
    its step on (binary16: 65504 + 16 = 65520; head_ref has a whole step, 65568, and calls 65520.8 finite), and a result that may lie
    on either side of that, by its bound, may be either."""
    import torch

    from tests import head_ref
    info = torch.finfo(got.dtype)
    limit = info.max * (1 + info.eps / 2 / (2 - info.eps))               # max = (2 - eps) 2^e, half a step = eps / 2 * 2^e
    with np.errstate(invalid="ignore"):
        over, near = np.abs(want) >= limit, np.abs(np.abs(want) - limit) <= np.broadcast_to(bound, want.shape)
    g = head_ref.f64(got)
    same_side = near & (np.sign(g) == np.sign(want)) & (np.abs(g) >= info.max * (1 - info.eps))
    want = np.where(over, np.copysign(np.inf, want), want)
    head_ref.assert_within(got, np.where(same_side, g, want), bound, what)
