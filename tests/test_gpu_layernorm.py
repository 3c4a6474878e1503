"""Layer norm and its gradients on the GPU against the 64-bit form, within bounds that count roundings (head_ref)."""
import numpy as np
import pytest
import torch

from paper_2407_02327_amd import qsync as Q
from paper_2407_02327_amd.head import LayerNorm
from tests import head_ref as R
from tests.gpu_util import say

pytestmark = pytest.mark.gpu
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
EPS = 1e-5
# (rows, cols): every way of dividing a row among lanes, both sides of each limit, odd and long ones, more rows than workgroups
SIZES = [(1, 1), (3, 7), (40, 128), (17, 129), (9, 512), (4, 515), (33, 1001), (5, 1024), (3, 1025), (2, 2048), (2, 2049), (3, 4096),
         (2, 5003), (2, 8192), (2, 8200), (1, 16384), (2, 20001), (2100, 72), (1500, 520), (2500, 1030)]


def _filled(rows, cols, dtype, seed, offset=0.0, pad=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = (torch.randn(rows, cols + pad, generator=g, device="cuda") * 1.5 + offset).to(dtype)
    return t[:, pad // 2:pad // 2 + cols]


def _params(cols, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(cols, generator=g, device="cuda") * 0.3 + 1.0, torch.randn(cols, generator=g, device="cuda") * 0.2


def _check(x, gamma, beta, dy, op, what):
    y = op.forward(x, gamma, beta)
    dx, dgamma, dbeta = op.backward(dy)
    torch.cuda.synchronize()
    g64 = R.f64(gamma) if gamma is not None else np.ones(x.shape[1])
    b64 = R.f64(beta) if beta is not None else np.zeros(x.shape[1])
    want, mean, rstd = R.layernorm(R.f64(x), g64, b64, op.eps)
    R.assert_within(y, want, R.layernorm_bound(R.f64(x), g64, b64, op.eps) + R.rounded(want, y.dtype), what + " y")
    for got, w, b in zip((dx, dgamma, dbeta), R.layernorm_grad(R.f64(dy), R.f64(x), g64, op.eps), R.layernorm_grad_bound(R.f64(dy), R.f64(x), g64, op.eps)):
        R.assert_within(got, w, b + R.rounded(w, got.dtype), what + " gradient")


@pytest.mark.parametrize("rows, cols", SIZES)
@pytest.mark.parametrize("x_dtype, dy_dtype", [(F32, F32), (F16, F16), (BF16, BF16), (F16, F32), (F32, BF16)])
def test_sizes_and_types(rows, cols, x_dtype, dy_dtype):
    say("layernorm", rows, cols, x_dtype, dy_dtype)
    gamma, beta = _params(cols, 3)
    op = LayerNorm(rows, cols, x_dtype=x_dtype, y_dtype=dy_dtype, dx_dtype=x_dtype, eps=EPS)
    _check(_filled(rows, cols, x_dtype, 1, 0.3), gamma, beta, _filled(rows, cols, dy_dtype, 2), op, f"{rows}x{cols}")


@pytest.mark.parametrize("dtypes", [(a, b, c) for a in (F32, F16, BF16) for b in (F32, F16, BF16) for c in (F32, F16, BF16)
                                    if len({a, b, c}) == 3 or (a, b, c) in ((BF16, F16, F16), (F16, BF16, BF16))])
def test_mixed_types(dtypes):
    """x, dy and the outputs each of a type of its own."""
    say("layernorm types", dtypes)
    gamma, beta = _params(260, 5)
    op = LayerNorm(6, 260, x_dtype=dtypes[0], y_dtype=dtypes[2], dx_dtype=dtypes[2], eps=EPS)
    _check(_filled(6, 260, dtypes[0], 1), gamma, beta, _filled(6, 260, dtypes[1], 2), op, str(dtypes))


@pytest.mark.parametrize("cols, pad", [(64, 2), (1001, 5), (1024, 8), (3001, 3), (9001, 1)])
@pytest.mark.parametrize("dtype", [F16, F32])
def test_rows_at_a_stride(cols, pad, dtype):
    """Rows inside a wider matrix, at any alignment; gamma and beta absent, and views at odd addresses."""
    say("layernorm stride", cols, pad, dtype)
    op = LayerNorm(7, cols, x_dtype=dtype, eps=EPS)
    _check(_filled(7, cols, dtype, 1, 0.5, pad), None, None, _filled(7, cols, dtype, 2, 0.0, pad), op, "strided")
    gamma, beta = _params(cols + 1, 3)
    _check(_filled(7, cols, dtype, 4, 0.5, pad), gamma[1:], beta[1:], _filled(7, cols, dtype, 5, 0.0, pad), op, "strided, parameters")
    _check(_filled(5, cols, dtype, 4, 0.5, pad), gamma[1:], None, _filled(5, cols, dtype, 5, 0.0, pad), op, "fewer rows")


@pytest.mark.parametrize("cols", [100, 700, 4096, 9000, 17000])
def test_values_far_from_zero(cols):
    """A mean a thousand deviations away, rows of one value, and rows of very large and very small values."""
    x = _filled(6, cols, F32, 1, 0.0)
    x[0] += 2000.0
    x[1] = 3.25
    x[2] *= 1e15
    x[3] *= 1e-15
    x[4] = 0.0
    gamma, beta = _params(cols, 3)
    _check(x, gamma, beta, _filled(6, cols, F32, 2), LayerNorm(6, cols, x_dtype=F32, eps=EPS), "far")


@pytest.mark.parametrize("cols", [24, 1000, 3000, 9000, 17000])
def test_a_bad_row_spoils_no_other(cols):
    x, dy = _filled(5, cols, F16, 1), _filled(5, cols, F16, 2)
    x[1, cols // 2] = float("nan")
    x[3, 0] = float("inf")
    gamma, beta = _params(cols, 3)
    op = LayerNorm(5, cols, x_dtype=F16, eps=EPS)
    y = R.f64(op.forward(x, gamma, beta))
    assert np.isnan(y[1]).all() and np.isnan(y[3]).all()
    keep = [0, 2, 4]
    want, _, _ = R.layernorm(R.f64(x)[keep], R.f64(gamma), R.f64(beta), EPS)
    R.assert_within(op.y[keep], want, R.layernorm_bound(R.f64(x)[keep], R.f64(gamma), R.f64(beta), EPS) + R.rounded(want, F16), "others")
    dx = op.backward(dy)[0]
    assert np.isnan(R.f64(dx)[1]).all() and not np.isnan(R.f64(dx)[keep]).any()


@pytest.mark.parametrize("cols", [40, 1000, 8192, 17000])
def test_in_place(cols):
    """y over x, dx over dy, dx over x: the same bits as apart."""
    gamma, beta = _params(cols, 3)
    x, dy = _filled(9, cols, BF16, 1, 0.2), _filled(9, cols, BF16, 2)
    op = LayerNorm(9, cols, x_dtype=BF16, eps=EPS)
    y = op.forward(x, gamma, beta).clone()
    dx, dgamma, dbeta = (t.clone() for t in op.backward(dy))
    ws = torch.empty(max(Q.qsync_layernorm_bwd_workspace_bytes(9, cols), 16), dtype=torch.uint8, device="cuda")
    z = x.clone()
    Q.qsync_layernorm_fwd(z, 9, cols, cols, gamma, beta, EPS, z, None, None)
    assert torch.equal(z, y)
    for over_x in (False, True):
        a, b = x.clone(), dy.clone()
        out, dg, db = (a if over_x else b), torch.empty_like(dgamma), torch.empty_like(dbeta)
        Q.qsync_layernorm_bwd(b, cols, a, 9, cols, cols, gamma, op.mean, op.rstd, out, dg, db, ws)
        assert torch.equal(out, dx) and torch.equal(dg, dgamma) and torch.equal(db, dbeta)


def test_single_outputs_and_empty_batches():
    x, dy, (gamma, beta) = _filled(50, 300, F16, 1), _filled(50, 300, F16, 2), _params(300, 3)
    op = LayerNorm(50, 300, x_dtype=F16, eps=EPS)
    op.forward(x, gamma, beta)
    dx, dgamma, dbeta = (t.clone() for t in op.backward(dy))
    for which in range(3):
        outs = [torch.full_like(t, 7.0) if i == which else None for i, t in enumerate((dx, dgamma, dbeta))]
        Q.qsync_layernorm_bwd(dy, 300, x, 50, 300, 300, gamma, op.mean, op.rstd, *outs, None if which == 0 else op.ws)
        assert torch.equal(outs[which], (dx, dgamma, dbeta)[which])
    assert op.forward(x[:0], gamma, beta).shape == (0, 300)
    dx, dgamma, dbeta = op.backward(dy[:0])
    assert dx.shape == (0, 300) and not dgamma.any() and not dbeta.any()
    op.dgamma.fill_(5.0)                                   # the C entry point clears them too
    Q.qsync_layernorm_bwd(dy, 300, x, 0, 300, 300, gamma, op.mean, op.rstd, None, op.dgamma, None, None)
    assert not op.dgamma.any()


@pytest.mark.parametrize("rows, cols", [(1, 33), (300, 1000), (5, 9000), (3, 17001)])
@pytest.mark.parametrize("y_dtype", [F16, BF16, F32])
def test_largest_output(rows, cols, y_dtype):
    """`y_amax` is max |y| as stored, over what it held before."""
    gamma, beta = _params(cols, 3)
    op = LayerNorm(rows, cols, x_dtype=F16, y_dtype=y_dtype, collect_y_amax=True)
    y = op.forward(_filled(rows, cols, F16, 1), gamma, beta)
    assert op.y_amax.item() == y.float().abs().max().item()
    op.y_amax.fill_(1000.0)
    op.forward(_filled(rows, cols, F16, 2), gamma, beta)
    assert op.y_amax.item() == 1000.0


def test_results_repeat_and_streams():
    """Two runs give the same bits, also on a stream of the caller's."""
    x, dy, (gamma, beta) = _filled(3000, 1024, F16, 1), _filled(3000, 1024, F16, 2), _params(1024, 3)
    op = LayerNorm(3000, 1024, x_dtype=F16)
    first = [t.clone() for t in (op.forward(x, gamma, beta), *op.backward(dy))]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    again = [op.forward(x, gamma, beta, stream=side), *op.backward(dy, stream=side)]
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(first, again))


def test_offsets_beyond_32_bits():
    rows, cols = 530000, 4096                              # 2.2e9 elements
    say("layernorm large", rows, cols)
    x = torch.zeros(rows, cols, dtype=BF16, device="cuda")
    x[-3:] = _filled(3, cols, BF16, 1, 0.4)
    gamma, beta = _params(cols, 3)
    op = LayerNorm(rows, cols, x_dtype=BF16, eps=EPS)
    y = op.forward(x, gamma, beta)
    want, _, _ = R.layernorm(R.f64(x[-3:]), R.f64(gamma), R.f64(beta), EPS)
    R.assert_within(y[-3:], want, R.layernorm_bound(R.f64(x[-3:]), R.f64(gamma), R.f64(beta), EPS) + R.rounded(want, BF16), "last rows")
    dy = torch.zeros_like(x)
    dy[-3:] = _filled(3, cols, BF16, 2)
    dx, _, dbeta = op.backward(dy)
    wants, bounds = R.layernorm_grad(R.f64(dy[-3:]), R.f64(x[-3:]), R.f64(gamma), EPS), R.layernorm_grad_bound(R.f64(dy[-3:]), R.f64(x[-3:]), R.f64(gamma), EPS)
    R.assert_within(dx[-3:], wants[0], bounds[0] + R.rounded(wants[0], BF16), "last gradients")
    R.assert_within(dbeta, wants[2], bounds[2] + R.rounded(wants[2], F32), "dbeta")


def test_in_a_graph():
    """Captured forward and backward passes, replayed on new values."""
    x, dy, (gamma, beta) = _filled(100, 1001, F16, 1), _filled(100, 1001, F16, 2), _params(1001, 3)
    op, eager = LayerNorm(100, 1001, x_dtype=F16), LayerNorm(100, 1001, x_dtype=F16)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        op.forward(x, gamma, beta)
        op.backward(dy)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        op.forward(x, gamma, beta)
        op.backward(dy)
    for seed in range(3):
        x.copy_(_filled(100, 1001, F16, 10 + seed))
        dy.copy_(_filled(100, 1001, F16, 20 + seed))
        graph.replay()
        want = [eager.forward(x, gamma, beta), *eager.backward(dy)]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((op.y, op.dx, op.dgamma, op.dbeta), want))


def test_gradient_against_differences():
    """The operator's own forward pass, moved by a step along a direction.  fp32 values of size 1 with a step of 2^-8: a central
    difference is off by the third derivative, 2^-16 / 6 of it (all derivatives here are of the size of the first at most 2^6), and by
    the forward's bound over the step."""
    rows, cols = 6, 200
    x, dy, (gamma, beta) = _filled(rows, cols, F32, 1), _filled(rows, cols, F32, 2), _params(cols, 3)
    op = LayerNorm(rows, cols, x_dtype=F32)
    op.forward(x, gamma, beta)
    dx = R.f64(op.backward(dy)[0])
    v, step = _filled(rows, cols, F32, 9), 2.0 ** -8
    f = lambda a: (R.f64(op.forward(a, gamma, beta)) * R.f64(dy)).sum()
    hi, lo = x + step * v, x - step * v
    moved = (R.f64(hi) - R.f64(lo)) / (2 * step)
    noise = (R.layernorm_bound(R.f64(x), R.f64(gamma), R.f64(beta), 1e-5) * np.abs(R.f64(dy))).sum() / step
    assert abs((f(hi) - f(lo)) / (2 * step) - (dx * moved).sum()) <= noise + 2.0 ** -10 * np.abs(dx * moved).sum()


@pytest.mark.parametrize("made_for, rows, cols", [(513, 512, 1030), (513, 512, 2443), (2049, 2048, 1001), (5200, 5120, 2051)])
@pytest.mark.parametrize("x_dtype, dy_dtype", [(F32, F32), (BF16, BF16), (F16, F32)])
def test_batches_shorter_than_the_operator(made_for, rows, cols, x_dtype, dy_dtype):
    """Fewer rows that are divided among more workgroups than the rows which the operator was made for."""
    say("layernorm fewer rows", made_for, rows, cols, x_dtype, dy_dtype)
    gamma, beta = _params(cols, 3)
    op = LayerNorm(made_for, cols, x_dtype=x_dtype, y_dtype=dy_dtype, dx_dtype=x_dtype, eps=EPS)
    for n in (rows, made_for):
        _check(_filled(n, cols, x_dtype, 1, 0.3), gamma, beta, _filled(n, cols, dy_dtype, 2), op, f"{n} of {made_for} x {cols}")


@pytest.mark.parametrize("rows", [0, 40])
def test_empty_batch_on_a_stream(rows):
    """The cleared gradients come in the order of the caller's stream, not of torch's current one."""
    op = LayerNorm(rows, 300, x_dtype=F16, eps=EPS)
    x, a = torch.empty(0, 300, dtype=F16, device="cuda"), torch.zeros(8192, 8192, dtype=F16, device="cuda")
    b, side = torch.empty_like(a), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(20):                                # some milliseconds, behind which an earlier batch's gradients arrive
            torch.mm(a, a, out=b)
        op.dgamma.fill_(5.0)
        op.dbeta.fill_(6.0)
    op.forward(x, stream=side)
    dx, dgamma, dbeta = op.backward(x, stream=side)
    with torch.cuda.stream(side):
        seen = dgamma.clone(), dbeta.clone()
    torch.cuda.synchronize()
    assert dx.shape == (0, 300) and not any(t.any() for t in (*seen, dgamma, dbeta))


def test_more_rows_than_a_launch_has_workgroups_for():
    rows = 1 << 30
    say("layernorm rows", rows)
    x = torch.zeros(rows, 2, dtype=F16, device="cuda")
    x[:, 1] = 1.0
    x[-3:] = torch.tensor([[3.0, -1.0], [-2.0, 2.0], [5.0, 5.0]], dtype=F16, device="cuda")
    gamma, beta = torch.tensor([0.5, 2.0], device="cuda"), torch.tensor([0.25, -1.0], device="cuda")
    op = LayerNorm(rows, 2, x_dtype=F16, eps=EPS, training=False)
    y = op.forward(x, gamma, beta)
    want, _, _ = R.layernorm(R.f64(x[-4:]), R.f64(gamma), R.f64(beta), EPS)
    R.assert_within(y[-4:], want, R.layernorm_bound(R.f64(x[-4:]), R.f64(gamma), R.f64(beta), EPS) + R.rounded(want, F16), "last rows")
    assert bool((y[:-3] == y[0]).all()) and torch.equal(y[0], y[-4])


def test_more_columns_than_a_launch_has_workgroups_for():
    cols = (1 << 27) + 8
    say("layernorm columns", cols)
    x, dy = torch.zeros(1, cols, dtype=BF16, device="cuda"), torch.ones(1, cols, dtype=BF16, device="cuda")
    dy[0, 0], dy[0, -1], dy[0, -9] = 3.0, -2.0, 4.0
    dgamma, dbeta = torch.full((cols,), 7.0, device="cuda"), torch.full((cols,), 7.0, device="cuda")
    mean, rstd = torch.full((1,), -0.5, device="cuda"), torch.full((1,), 2.0, device="cuda")      # xh is 1
    ws = torch.empty(Q.qsync_layernorm_bwd_workspace_bytes(1, cols), dtype=torch.uint8, device="cuda")
    Q.qsync_layernorm_bwd(dy, cols, x, 1, cols, cols, None, mean, rstd, None, dgamma, dbeta, ws)
    assert torch.equal(dgamma, dy[0].float()) and torch.equal(dbeta, dy[0].float())


@pytest.mark.parametrize("rows, cols", [(1100, 4500), (1100, 5003), (1100, 8192), (1100, 16384), (1100, 17001)])
@pytest.mark.parametrize("dtype", [F16, F32])
def test_many_wide_rows(rows, cols, dtype):
    """More rows than workgroups where a row takes a whole one: several turns of each, whose sums meet."""
    say("layernorm wide", rows, cols, dtype)
    gamma, beta = _params(cols, 3)
    _check(_filled(rows, cols, dtype, 1, 0.3), gamma, beta, _filled(rows, cols, dtype, 2), LayerNorm(rows, cols, x_dtype=dtype, eps=EPS), f"{rows}x{cols}")
