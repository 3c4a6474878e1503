"""Token log-probabilities, their gradient and distillation on the GPU against the 64-bit forms, within bounds that count roundings
(head_ref)."""
import numpy as np
import pytest
import torch

from paper_2407_02327_amd import qsync as Q
from paper_2407_02327_amd.head import Distillation, TokenLogProbs
from tests import head_ref as R
from tests.gpu_util import say

pytestmark = pytest.mark.gpu
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
INF = float("inf")
# one column, a handful, lengths around a vector, a wavefront's and a workgroup's reach, more pieces than one, rows beyond the device's room
SIZES = [(1, 1), (2, 3), (5, 64), (3, 65), (4, 1000), (2, 2048), (3, 2049), (1, 8193), (2, 50021), (1, 131072), (1, 140001), (1100, 77), (1030, 8200)]


def _logits(rows, cols, dtype, seed, pad=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    z = torch.randn(rows, cols + pad, generator=g, device="cuda") * 2.5
    z[:, ::37] += 4.0
    return z.to(dtype)[:, pad // 2:pad // 2 + cols]


def _randn(n, seed):
    return torch.randn(n, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


def _tokens(rows, cols, seed, dtype=torch.int64):
    t = torch.randint(0, cols, (rows,), generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")
    t[::5] = -100
    t[-1] = cols - 1
    return t.to(dtype)


def _check_logprobs(z, tokens, scale, top_k, what, op=None, grad_dtype=None):
    rows, cols = z.shape
    op = op or TokenLogProbs(rows, cols, top_k=top_k, scale=scale, dlogits_dtype=grad_dtype or z.dtype)
    logp, entropy, top_logp, top_index = op.forward(z, tokens)
    torch.cuda.synchronize()
    z64, t = R.f64(z), tokens.cpu().numpy()
    rel, off = R.logits_bound(z64, scale)
    w_logp, w_h, w_tl, w_ti = R.token_logprobs(z64, t, scale, top_k)
    R.assert_within(logp, w_logp, np.array([off[r, max(min(x, cols - 1), 0)] for r, x in enumerate(t)]) + R.rounded(w_logp, F32), what + " logp")
    lp = R.log_softmax(z64, scale)
    p = np.exp(np.where(np.isnan(lp), -np.inf, lp))
    plp = np.abs(R._plogp(p, lp))
    R.assert_within(entropy, w_h, (rel * plp + off * p).sum(1) * 2 + rel.max(1) * 2 + R.rounded(w_h, F32), what + " entropy")
    if top_k:
        assert np.array_equal(top_index.cpu().numpy(), w_ti), what + " alternatives"
        R.assert_within(top_logp, w_tl, np.take_along_axis(off, w_ti, 1) + R.rounded(w_tl, F32), what + " top_logp")
    for with_g, with_h in ((True, True), (True, False), (False, True)):
        g, h = _randn(rows, 11), _randn(rows, 12) * 0.3
        dz = op.backward(g if with_g else None, h if with_h else None)
        torch.cuda.synchronize()
        g64, h64 = R.f64(g) * with_g, R.f64(h) * with_h
        seen = t if with_g else np.full_like(t, -1)
        want = R.token_logprobs_grad(z64, seen, scale, g64, h64)
        at = np.zeros_like(p)
        at[np.arange(rows)[(t >= 0) & (t < cols)], t[(t >= 0) & (t < cols)]] = 1
        size = scale * (np.abs(g64)[:, None] * (p + at) + np.abs(h64)[:, None] * (plp + p * w_h[:, None] + p))
        R.assert_within(dz, want, (2 * rel.max(1, keepdims=True) + 2 * rel) * size + R.rounded(want, dz.dtype) + scale * (np.abs(g64) + np.abs(h64))[:, None] * 2.0 ** -120,
                        f"{what} gradient {with_g} {with_h}")


@pytest.mark.parametrize("rows, cols", SIZES)
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_logprobs_sizes_and_types(rows, cols, dtype):
    say("logprobs", rows, cols, dtype)
    _check_logprobs(_logits(rows, cols, dtype, 1), _tokens(rows, cols, 2), 1.0, min(cols, 7), f"{rows}x{cols}")


@pytest.mark.parametrize("top_k", [0, 1, 2, 31, 63, 64])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_numbers_of_alternatives(top_k, dtype):
    """One workgroup a row, and rows in pieces; bfloat16 logits have many equal values."""
    for rows, cols in ((1200, 300), (3, 300), (2, 40000)):
        say("alternatives", rows, cols, top_k, dtype)
        _check_logprobs(_logits(rows, cols, dtype, top_k), _tokens(rows, cols, 2, torch.int32), 0.7, top_k, f"top {top_k} of {cols}")


@pytest.mark.parametrize("rows, cols", [(2, 9000), (1100, 9000)])
@pytest.mark.parametrize("order", ["equal", "two values", "ascending", "descending", "one lane", "zeros of both signs"])
def test_alternatives_in_any_order(rows, cols, order):
    """Equal logits come by their column; the best in the last, the first and in the places of one lane."""
    say("order", rows, cols, order)
    z = torch.zeros(rows, cols, device="cuda")
    ramp = torch.arange(cols, device="cuda", dtype=torch.float32) / 1000
    if order == "two values":
        z[:, 4500:] = 1.0
        z[:, ::7] = 1.0
    elif order == "ascending":
        z += ramp
    elif order == "descending":
        z -= ramp
    elif order == "one lane":
        z += ramp * 1e-3
        for first in range(0, cols, 1024):
            z[:, first + 40:first + 44] += 5.0 + first
    elif order == "zeros of both signs":
        z[:, ::2] = -0.0
    for dtype in (F32, F16):
        _check_logprobs(z.to(dtype), _tokens(rows, cols, 2), 1.0, 64, f"{order} {dtype}")


@pytest.mark.parametrize("rows, cols, pad", [(3, 1001, 3), (1100, 130, 1), (2, 33000, 7)])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_rows_at_a_stride(rows, cols, pad, dtype):
    say("stride", rows, cols, pad, dtype)
    z = _logits(rows, cols, dtype, 4, pad)
    _check_logprobs(z, _tokens(rows, cols, 2), 1.3, 5, "strided")
    _check_distill(z, 9, 1.3, "strided")


@pytest.mark.parametrize("grad_dtype", [F32, F16, BF16])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_gradients_of_another_type(dtype, grad_dtype):
    z = _logits(4, 1003, dtype, 4)
    _check_logprobs(z, _tokens(4, 1003, 2), 1.0, 0, "types", grad_dtype=grad_dtype)
    _check_distill(z, 5, 1.0, "types", grad_dtype=grad_dtype)


def test_operator_for_fewer_rows_and_other_types():
    """One operator, calls of every number of rows up to its own: the pieces differ, the workspace has room."""
    op, dist = TokenLogProbs(1500, 5000, top_k=9, dlogits_dtype=F32), Distillation(1500, 5000, 6, dlogits_dtype=F32)
    for rows, dtype in ((1500, F16), (1, F32), (2, BF16), (37, F32), (1025, F32)):
        say("fewer rows", rows, dtype)
        z = _logits(rows, 5000, dtype, rows)
        _check_logprobs(z, _tokens(rows, 5000, 2), 1.0, 9, f"{rows} rows", op)
        _check_distill(z, 6, 1.0, f"{rows} rows", dist)


def _masked(rows, cols, dtype, least):
    """Rows with all, nothing but one, few, and the end of the columns masked."""
    z = _logits(rows, cols, dtype, 6).clone()
    z[0] = least
    z[1, 1:] = least
    z[2, :] = least
    z[2, [cols // 3, cols // 2, cols - 1]] = torch.tensor([1.0, 3.0, 2.0], device="cuda", dtype=dtype)
    z[3, cols // 2:] = least
    return z


@pytest.mark.parametrize("rows, cols", [(4, 700), (5, 30000), (1100, 700)])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("least", ["-inf", "lowest"])
@pytest.mark.parametrize("scale", [1.0, 2.5])
def test_masked_logits(rows, cols, dtype, least, scale):
    """-inf and the type's lowest value as masks; a row of nothing else is empty (-inf) or uniform (lowest)."""
    say("masked", rows, cols, dtype, least, scale)
    z = _masked(rows, cols, dtype, -INF if least == "-inf" else torch.finfo(dtype).min)
    _check_logprobs(z, _tokens(rows, cols, 2), scale, 6, least)
    _check_distill(z, 7, scale, least)


@pytest.mark.parametrize("rows, cols", [(4, 5000), (1100, 600)])
def test_rows_with_nan_and_infinity(rows, cols):
    """Such a row's results are NaN, its alternatives columns of the row or -1; the others are what they would be without it."""
    z, tokens = _logits(rows, cols, F16, 1).clone(), _tokens(rows, cols, 2).clamp_(min=0)
    clean = TokenLogProbs(rows, cols, top_k=5, dlogits_dtype=F32)
    good = [t.clone() for t in clean.forward(z, tokens)]
    z[1, 17], z[2, cols - 2] = float("nan"), INF
    z[3, :] = float("nan")
    op = TokenLogProbs(rows, cols, top_k=5, dlogits_dtype=F32)
    got = op.forward(z, tokens)
    for a, b in zip(got, good):
        assert torch.equal(a[0], b[0]) and torch.equal(a[4:], b[4:])
    assert torch.isnan(got[0][1:4]).all() and torch.isnan(got[1][1:4]).all()
    assert ((got[3] >= -1) & (got[3] < cols)).all()
    dz = op.backward(torch.ones(rows, device="cuda"), torch.ones(rows, device="cuda"))
    assert torch.isnan(dz[1:4]).all(1).all() and not torch.isnan(dz[0]).any()
    g = torch.ones(rows, device="cuda")
    g[1:4] = 0
    assert not op.backward(g, None)[1:4].any()             # (nothing is asked of those rows)


def test_tokens_outside_the_vocabulary():
    """Negative: no token.  Too large: NaN, and nothing is read there."""
    z = _logits(4, 500, F32, 1)
    tokens = torch.tensor([3, -1, 500, 2 ** 40], device="cuda")
    op = TokenLogProbs(4, 500, dlogits_dtype=F32)
    logp = op.forward(z, tokens)[0].cpu()
    assert logp[1] == 0 and torch.isnan(logp[2:]).all() and not torch.isnan(logp[:2]).any()
    dz = op.backward(torch.ones(4, device="cuda"))
    assert torch.isnan(dz[2:]).all() and not dz[1].any() and not torch.isnan(dz[0]).any()


# ---- distillation -------------------------------------------------------------------------------------------------------------

def _entries(rows, cols, k, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    index = torch.randint(0, cols, (rows, k), generator=g, device="cuda")
    teacher = torch.randn(rows, k, generator=g, device="cuda") * 2
    if k > 2:
        index[::3, 1] = -1                                 # an absent entry
        teacher[1::3, 2] = -INF                            # one without weight
    index[-1] = index[-1, 0].clone()                               # one column k times
    if rows > 2:
        index[2] = -100                                    # a row without entries
    return teacher, index


def _check_distill(z, k, scale, what, op=None, grad_dtype=None, teacher_dtype=F32, index_dtype=torch.int64):
    rows, cols = z.shape
    op = op or Distillation(rows, cols, k, scale=scale, dlogits_dtype=grad_dtype or z.dtype)
    teacher, index = _entries(rows, cols, k, 5)
    teacher, index = teacher.to(teacher_dtype), index.to(index_dtype)
    weight = _randn(rows, 8)
    weight[rows // 2] = 0.0
    z64, t64, i64, w64 = R.f64(z), R.f64(teacher), index.cpu().numpy(), R.f64(weight)
    want, q = R.distill(z64, t64, i64, scale)
    rel, off = R.logits_bound(z64, scale)
    lp = R.log_softmax(z64, scale)
    slack = np.zeros(rows)
    for r in range(rows):
        if np.isnan(want[r]):
            continue
        lq = R.log_softmax(np.where(i64[r] >= 0, t64[r], -np.inf)[None], scale)[0]
        live = ~np.isneginf(lq) & ~np.isneginf(lp[r, np.maximum(i64[r], 0)])
        lq, cp = lq[live], i64[r][live]
        d = np.abs(lq) + 10
        slack[r] = (np.exp(lq) * (off[r, cp] + R.U * (6 * d + 280) * (1 + np.abs(lq) + np.abs(lp[r, cp])))).sum() if live.any() else 0.0
    for with_grad in (False, True):
        if with_grad:
            loss, dz = op.forward_backward(z, teacher, index, weight)
        else:
            loss = op.forward(z, teacher, index)
        torch.cuda.synchronize()
        R.assert_within(loss, want, slack + R.rounded(want, F32), f"{what} loss {with_grad}")
    p = np.exp(np.where(np.isnan(lp), -np.inf, lp))
    grad = R.distill_grad(z64, t64, i64, scale, w64)
    bound = scale * np.abs(w64)[:, None] * (2 * rel * p + R.U * 400 * np.nan_to_num(q) + 2.0 ** -120)
    R.assert_within(dz, grad, bound + R.rounded(grad, dz.dtype), what + " gradient")


@pytest.mark.parametrize("rows, cols", SIZES)
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_distillation_sizes_and_types(rows, cols, dtype):
    say("distill", rows, cols, dtype)
    _check_distill(_logits(rows, cols, dtype, 1), 5, 1.0, f"{rows}x{cols}")


@pytest.mark.parametrize("k", [1, 2, 63, 64, 65, 255, 256])
@pytest.mark.parametrize("rows, cols", [(3, 6000), (1100, 900)])
def test_numbers_of_entries(k, rows, cols):
    say("entries", rows, cols, k)
    _check_distill(_logits(rows, cols, F16, 1), k, 0.5, f"{k} entries", teacher_dtype=F16, index_dtype=torch.int32)
    _check_distill(_logits(rows, cols, F32, 1), k, 2.0, f"{k} entries", teacher_dtype=BF16)


@pytest.mark.parametrize("rows, cols", [(4, 5000), (1100, 600)])
def test_bad_entries(rows, cols):
    """An index beyond the vocabulary or a teacher's NaN makes its row NaN and no other; weight 0 keeps a bad row out of the gradient."""
    z, (teacher, index) = _logits(rows, cols, F16, 1), _entries(rows, cols, 8, 5)
    op = Distillation(rows, cols, 8, dlogits_dtype=F32)
    good = [t.clone() for t in op.forward_backward(z, teacher, index)]
    index, teacher = index.clone(), teacher.clone()
    index[0, 3], teacher[1, 4] = cols, float("nan")
    weight = torch.ones(rows, device="cuda")
    loss, dz = op.forward_backward(z, teacher, index, weight)
    assert torch.isnan(loss[:2]).all() and torch.isnan(dz[:2]).all()
    assert torch.equal(loss[2:], good[0][2:]) and torch.equal(dz[2:], good[1][2:])
    weight[:2] = 0
    loss, dz = op.forward_backward(z, teacher, index, weight)
    assert not dz[:2].any() and torch.isnan(loss[:2]).all() and torch.equal(dz[2:], good[1][2:])


@pytest.mark.parametrize("rows, cols", [(3, 9001), (1100, 1000), (1, 70000)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_gradients_in_place(rows, cols, dtype):
    """Over the logits: the same bits as apart."""
    say("in place", rows, cols, dtype)
    z, tokens = _logits(rows, cols, dtype, 1).contiguous(), _tokens(rows, cols, 2)
    g, h = _randn(rows, 3), _randn(rows, 4)
    op = TokenLogProbs(rows, cols, dlogits_dtype=dtype)
    op.forward(z, tokens)
    want, a = op.backward(g, h), z.clone()
    op.forward(a, tokens)
    assert torch.equal(op.backward(g, h, out=a), want) and a.data_ptr() != want.data_ptr()
    teacher, index = _entries(rows, cols, 8, 5)
    dist, b = Distillation(rows, cols, 8, dlogits_dtype=dtype), z.clone()
    loss, dz = (t.clone() for t in dist.forward_backward(z, teacher, index, g))
    loss_b, dz_b = dist.forward_backward(b, teacher, index, g, out=b)
    assert torch.equal(loss, loss_b) and torch.equal(dz, dz_b)


def test_results_repeat_and_streams():
    z, tokens = _logits(5, 60000, BF16, 1), _tokens(5, 60000, 2)
    teacher, index = _entries(5, 60000, 8, 5)
    op, dist = TokenLogProbs(5, 60000, top_k=10, dlogits_dtype=BF16), Distillation(5, 60000, 8, dlogits_dtype=BF16)
    g = _randn(5, 3)
    run = lambda s: [t.clone() for t in (*op.forward(z, tokens, stream=s), op.backward(g, g, stream=s), *dist.forward_backward(z, teacher, index, stream=s))]
    first = run(None)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = run(side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(first, again))


def test_offsets_beyond_32_bits():
    rows, cols = 16500, 131072                             # 2.2e9 elements
    say("logits large", rows, cols)
    z = torch.zeros(rows, cols, dtype=BF16, device="cuda")
    z[-2:] = _logits(2, cols, BF16, 1)
    last, tokens = z[-2:].clone(), torch.zeros(rows, dtype=torch.int64, device="cuda")
    tokens[-1] = cols - 1
    op = TokenLogProbs(rows, cols, top_k=4)
    logp, entropy, top_logp, top_index = op.forward(z, tokens)
    w_logp, w_h, w_tl, w_ti = R.token_logprobs(R.f64(last), tokens[-2:].cpu().numpy(), 1.0, 4)
    rel, off = R.logits_bound(R.f64(last), 1.0)
    R.assert_within(logp[-2:], w_logp, off.max(1) + R.rounded(w_logp, F32), "logp")
    assert np.array_equal(top_index[-2:].cpu().numpy(), w_ti)
    g = torch.zeros(rows, device="cuda")
    g[-2:] = 1.0
    dz = op.backward(g, None, out=z)                       # in place
    want = R.token_logprobs_grad(R.f64(last), tokens[-2:].cpu().numpy(), 1.0, np.ones(2), np.zeros(2))
    R.assert_within(dz[-2:], want, 4 * rel.max() * (np.abs(want) + 2.0 ** -120) + 4 * rel.max(1, keepdims=True) * (want > 0) + R.rounded(want, BF16), "gradient")
    assert not dz[:-2].any()
    z[-2:] = last
    teacher, index = _entries(rows, cols, 3, 5)
    loss, dz = Distillation(rows, cols, 3).forward_backward(z, teacher, index, g, out=z)
    w_loss, _ = R.distill(R.f64(last), R.f64(teacher[-2:]), index[-2:].cpu().numpy(), 1.0)
    assert np.allclose(R.f64(loss[-2:]), w_loss, rtol=1e-4)
    assert not dz[:-2].any() and torch.isfinite(dz[-2:]).all() and dz[-1].any()


def test_in_a_graph():
    """Captured passes of a few rows (pieces joined by a second launch), replayed on new values."""
    z, tokens = _logits(3, 20001, F16, 1).clone(), _tokens(3, 20001, 2)
    teacher, index = _entries(3, 20001, 8, 5)
    g = _randn(3, 3)
    make = lambda: (TokenLogProbs(3, 20001, top_k=10, dlogits_dtype=F16), Distillation(3, 20001, 8, dlogits_dtype=F16))

    def passes(op, dist):
        return [*op.forward(z, tokens), op.backward(g, g), *dist.forward_backward(z, teacher, index, g)]
    mine, eager = make(), make()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        passes(*mine)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = passes(*mine)
    for seed in range(3):
        z.copy_(_logits(3, 20001, F16, 30 + seed))
        graph.replay()
        want = passes(*eager)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(captured, want))


def test_gradients_against_differences():
    """The operators' own forward passes, moved by a step along a direction: see the same test of the layer norm.  Log probabilities and
    losses near 10 have an absolute error of the bound each; the third derivative of a softmax along a direction of size 1 is at most 1."""
    rows, cols, step = 5, 400, 2.0 ** -7
    z, tokens = _logits(rows, cols, F32, 1), _tokens(rows, cols, 2)
    g, h = _randn(rows, 3), _randn(rows, 4)
    v = _randn(rows * cols, 9).view(rows, cols) * 0.5
    hi, lo = z + step * v, z - step * v
    moved = (R.f64(hi) - R.f64(lo)) / (2 * step)
    rel, off = R.logits_bound(R.f64(z), 1.0)
    op = TokenLogProbs(rows, cols, dlogits_dtype=F32)
    op.forward(z, tokens)
    dz = R.f64(op.backward(g, h))

    def f(a):
        logp, entropy, _, _ = op.forward(a, tokens)
        return (R.f64(g) * R.f64(logp) + R.f64(h) * R.f64(entropy)).sum()
    noise = ((np.abs(R.f64(g)) + 2 * np.abs(R.f64(h))) * off.max(1) * 8).sum() / step
    third = step ** 2 / 6 * ((np.abs(R.f64(g)) + 8 * np.abs(R.f64(h))) * np.abs(moved).max(1) ** 3).sum()
    assert abs((f(hi) - f(lo)) / (2 * step) - (dz * moved).sum()) <= noise + third
    teacher, index = _entries(rows, cols, 6, 5)
    dist = Distillation(rows, cols, 6, dlogits_dtype=F32)
    _, dz = dist.forward_backward(z, teacher, index, g)
    dz = R.f64(dz)
    f = lambda a: (R.f64(g) * R.f64(dist.forward(a, teacher, index))).sum()
    noise = (np.abs(R.f64(g)) * off.max(1) * 16).sum() / step
    assert abs((f(hi) - f(lo)) / (2 * step) - (dz * moved).sum()) <= noise + third


def test_what_the_classes_refuse():
    """Shapes, types, devices and orders of calls that the kernels must not see."""
    z, tokens = _logits(4, 100, F16, 1), _tokens(4, 100, 2)
    op = TokenLogProbs(4, 100, entropy=False)
    for bad in (lambda: op.forward(z.t(), tokens), lambda: op.forward(z[:, :99], tokens), lambda: op.forward(z.double(), tokens),
                lambda: op.forward(z[:1].expand(4, 100), tokens), lambda: op.forward(z, tokens[:3]), lambda: op.forward(z, tokens.float()),
                lambda: op.forward(z.cpu(), tokens), lambda: op.forward(torch.cat([z, z]), torch.cat([tokens, tokens]))):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(RuntimeError):
        op.backward(torch.ones(4, device="cuda"))
    op.forward(z)
    one = torch.ones(4, device="cuda")
    for bad in (lambda: op.backward(), lambda: op.backward(one), lambda: op.backward(None, one)):
        with pytest.raises(ValueError):
            bad()
    op.forward(z, tokens)
    for bad in (lambda: op.backward(one), lambda: op.backward(one[:3], out=z), lambda: op.backward(one, out=z[:, ::2]), lambda: op.backward(one.double(), out=z)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(Q.QsyncError) as e:                 # over the logits, in another type
        op.backward(one, out=z.view(BF16))
    assert e.value.status == Q.ERR_UNSUPPORTED
    dist = Distillation(4, 100, 3)
    teacher, index = _entries(4, 100, 3, 1)
    for bad in (lambda: dist.forward(z, teacher[:, :2], index), lambda: dist.forward(z, teacher, index.float()), lambda: dist.forward(z, teacher.cpu(), index),
                lambda: dist.forward_backward(z, teacher, index), lambda: dist.forward(z, teacher.t().contiguous().t(), index)):
        with pytest.raises(ValueError):
            bad()


@pytest.mark.parametrize("value", [-1e9, 7e8])
@pytest.mark.parametrize("first", range(8))
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_entropy_of_rows_of_one_value(dtype, first, value):
    """... wherever the row starts: ln cols.  The elements in front of and behind whole lines of memory count like the others."""
    for cols in (5, 27, 700, 70001):
        z = torch.full((1, cols + 8), value, dtype=dtype, device="cuda")[:, first:first + cols]
        _, entropy, _, _ = TokenLogProbs(1, cols).forward(z)
        # ... by what logits_bound counts, and the quotient of the two sums, up to 64 here, by the roundings of a lane's and the lanes' additions in each
        bound = (R.logits_bound(R.f64(z), 1.0)[0].max() + 64 * R.U * (cols // 256 + 40)) * 2 + R.rounded(np.log(cols), F32)
        R.assert_within(entropy, np.array([np.log(cols)]), bound, f"entropy {cols}")


class _Repeated:
    """An operator for `copies` times a batch's rows, called with them one after the other, `pad` elements between rows: so many rows are each
    kept whole, where a few would be cut into pieces.  All copies' results have the same bits -- of a multiple of eight rows, which all start
    at the same alignments in every copy --; the first's are returned."""

    def __init__(self, op, copies, pad=0):
        self.op, self.copies, self.pad = op, copies, pad

    def _given(self, t):
        if t is None or t.dim() == 1:
            return None if t is None else t.repeat(self.copies)
        return torch.nn.functional.pad(t.repeat(self.copies, 1), (0, self.pad))[:, :t.shape[1]] if self.pad and t.shape[1] == self.op.cols else t.repeat(self.copies, 1)

    def _first(self, t):
        if t is None:
            return None
        parts = t.view(self.copies, -1, *t.shape[1:])
        assert torch.equal(parts, parts[:1].expand_as(parts))
        return parts[0]

    def _call(self, f, *a):
        out = f(*[self._given(t) for t in a])
        return self._first(out) if isinstance(out, torch.Tensor) else tuple(self._first(t) for t in out)

    def forward(self, *a):
        return self._call(self.op.forward, *a)

    def backward(self, *a):
        return self._call(self.op.backward, *a)

    def forward_backward(self, *a):
        return self._call(self.op.forward_backward, *a)


# both sides of where a product with the scale leaves the reach of the fast form, far beyond it, and maxima as far up
FAR = [(dtype, value, scale) for dtype in (F32, BF16) for value, scale in
       ((-1e9, 1.0), (-1.38e9, 1.0), (-1.5e9, 1.0), (-1e10, 1.0), (-1e10, 2.5), (-1e15, 1.0), (-1e20, 0.7), (-1e29, 1.0), (1e9, 1.0), (1e10, 1.0), (1e20, 1.0))]
FAR += [(F16, -60000.0, 1e5), (F16, 30000.0, 1e6), (F16, 30000.0, 1e4)]


@pytest.mark.parametrize("copies, cols", [(1, 700), (1, 70001), (20, 70001)])
@pytest.mark.parametrize("dtype, value, scale", FAR)
def test_finite_values_far_from_zero(dtype, value, scale, copies, cols):
    """Rows of one such value, of nothing else but an ordinary one, with a few ordinary ones, in their second half, and in one place: rows of a
    workgroup, in pieces, and longer than a workgroup's registers."""
    say("far", dtype, value, scale, copies, cols)
    z = _masked(8, cols, dtype, value)
    z[4, cols // 2] = value
    tokens, k = _tokens(8, cols, 2), 7
    op = _Repeated(TokenLogProbs(8 * copies, cols, top_k=6, scale=scale, dlogits_dtype=dtype), copies)
    dist = _Repeated(Distillation(8 * copies, cols, k, scale=scale, dlogits_dtype=dtype), copies)
    _check_logprobs(z, tokens, scale, 6, "far", op)
    _check_distill(z, k, scale, "far", dist)
    # what lies so far below a row's maximum that its probability is 0 is as good as absent
    apart = torch.where(z.float() < z.float().amax(1, keepdim=True) - 1e4, -INF, z.float()).to(dtype)
    g, h, (teacher, index) = _randn(8, 3), _randn(8, 4), _entries(8, cols, k, 5)

    def results(a):
        _, entropy, _, _ = op.forward(a, tokens)
        return [entropy.clone(), op.backward(g, h).clone(), dist.forward_backward(a, teacher, index, g)[1].clone()]
    assert all(torch.equal(a, b) for a, b in zip(results(z), results(apart)))


@pytest.mark.parametrize("copies, cols", [(1, 700), (1, 70001), (20, 70001)])
def test_the_largest_and_smallest_scales(copies, cols):
    """A scale whose product with log2(e) no fp32 number holds: all weight is on the largest logits.  The smallest one: the uniform distribution."""
    say("scales", copies, cols)
    z, tokens = _logits(8, cols, BF16, 1).clone(), _tokens(8, cols, 2)
    z[0], z[1, 3] = 0.0, 50.0
    tokens[:2] = 3
    teacher, index = torch.zeros(8, 1, device="cuda"), torch.from_numpy(R.f64(z).argmax(1)).cuda()[:, None]      # (the first of equal ones)
    ties = (z == z.amax(1, keepdim=True)).sum(1).double().cpu().numpy()
    for scale, alive in ((3.2e38, ties), (1e-42, np.full(8, float(cols)))):
        op = _Repeated(TokenLogProbs(8 * copies, cols, top_k=1, scale=scale), copies)
        dist = _Repeated(Distillation(8 * copies, cols, 1, scale=scale), copies)
        logp, entropy, top_logp, top_index = op.forward(z, tokens)
        want = np.log(alive)
        bound = R.U * (cols // 256 + 120) + R.rounded(want, F32)
        R.assert_within(logp[:2], -want[:2], bound[:2], "logp")
        R.assert_within(top_logp[:, 0], -want, bound, "top_logp")
        R.assert_within(entropy, want, 2 * bound, "entropy")
        assert torch.equal(top_index.long(), index)
        R.assert_within(dist.forward(z, teacher, index), want, bound, "loss")


@pytest.mark.parametrize("copies", [1, 304])
def test_gradient_of_a_token_on_a_masked_column(copies):
    """Its log probability is -inf, whose gradient is the formula's: scale dlogp in its own column, and -scale dlogp p in the others, none
    of them masked; a row of nothing but masks has none."""
    z, tokens = _logits(3, 5000, F32, 1).clone(), torch.tensor([7, 4999, 3], device="cuda")
    z[0, 5:10], z[1, 2500:], z[2] = -INF, -INF, -INF
    op = _Repeated(TokenLogProbs(3 * copies, 5000, scale=0.5, dlogits_dtype=F32), copies)
    assert torch.isneginf(op.forward(z, tokens)[0]).all()
    g = torch.tensor([2.0, -3.0, 1.0], device="cuda")
    dz = op.backward(g)
    assert dz[0, 7] == 1.0 and dz[1, 4999] == -1.5 and not dz[2].any()
    masked = torch.isneginf(z)
    masked[[0, 1], tokens[:2]] = False
    assert not dz[masked].any()
    want = R.token_logprobs_grad(R.f64(z), tokens.cpu().numpy(), 0.5, R.f64(g), np.zeros(3))
    rel, _ = R.logits_bound(R.f64(z), 0.5)
    R.assert_within(dz, want, 4 * rel * np.abs(want) + 2.0 ** -120 + R.rounded(want, F32), "gradient")


# (20 copies of eight rows: enough that a row of any of these lengths is kept whole)
@pytest.mark.parametrize("pad", [0, 3])
@pytest.mark.parametrize("cols, dtype", [(20000, F32), (50021, F32), (40003, F16), (40003, BF16), (70001, F16), (70001, BF16), (131072, BF16)])
def test_long_rows_kept_whole(cols, dtype, pad):
    """Distillation steps over rows that fill the registers of a workgroup, and over longer ones, whose rest is read again."""
    say("whole", cols, dtype, pad)
    for z in (_logits(8, cols, dtype, 1), _masked(8, cols, dtype, -INF), _masked(8, cols, dtype, torch.finfo(dtype).min)):
        for grad_dtype in {dtype, F32}:
            _check_distill(z, 7, 0.7, f"{cols} {grad_dtype}", _Repeated(Distillation(160, cols, 7, scale=0.7, dlogits_dtype=grad_dtype), 20, pad))


@pytest.mark.parametrize("cols, dtype", [(50021, F32), (70001, BF16)])
def test_long_rows_kept_whole_in_place(cols, dtype):
    say("whole in place", cols, dtype)
    z, (teacher, index) = _logits(150, cols, dtype, 1).contiguous(), _entries(150, cols, 8, 5)
    g, op = _randn(150, 3), Distillation(150, cols, 8, dlogits_dtype=dtype)
    loss, dz = (t.clone() for t in op.forward_backward(z, teacher, index, g))
    again = op.forward_backward(z, teacher, index, g, out=z)
    assert torch.equal(again[0], loss) and torch.equal(z, dz)


@pytest.mark.parametrize("cols, top_k", [(98304, 9), (98305, 9), (200003, 64)])
def test_many_long_rows_with_alternatives(cols, top_k):
    """fp32 rows on both sides of what a search keeps of a row: one piece, and two or more of it, of more rows than the device has room for."""
    say("many long rows", cols, top_k)
    z = _logits(8, cols, F32, 1)
    z[3, cols // 2 - 40:cols // 2 + 40] = 30.0            # (equal ones on both sides of a limit)
    _check_logprobs(z, _tokens(8, cols, 2), 1.0, top_k, f"{cols}", _Repeated(TokenLogProbs(1104, cols, top_k=top_k, dlogits_dtype=F32), 138))
