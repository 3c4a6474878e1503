"""Routing to experts and their linear operators on the GPU: places bit for bit, sums within bounds that count roundings (token_ref)."""
import numpy as np
import pytest
import torch

from paper_2407_02327_amd import qsync as Q
from paper_2407_02327_amd.experts import ExpertLinear, ExpertRoute
from tests import token_ref as R
from tests.gpu_util import say
from tests.head_ref import U, f64, rounded
from tests.token_ref import assert_within
from tests.test_gpu_token_linear import BF16, F16, F32, SEED, equal, expected, values

pytestmark = pytest.mark.gpu


def ids_of(tokens, k, experts, seed, dtype=torch.int64, outside=0.0):
    """Some experts preferred, some without tokens, a share of the entries outside."""
    g = torch.Generator().manual_seed(seed)
    ids = (torch.rand(tokens, k, generator=g) ** 2 * experts).long()
    ids[ids % 5 == 3] //= 2
    drop = torch.rand(tokens, k, generator=g) < outside
    ids = torch.where(drop, torch.where(torch.rand(tokens, k, generator=g) < 0.5, -1, experts + 3), ids)
    return ids.to(dtype).cuda()


@pytest.mark.parametrize("tokens, k", [(1, 1), (1, 8), (63, 1), (64, 1), (65, 1), (13, 5), (512, 2), (1025, 1), (700, 8), (8192, 8), (50000, 3), (2048, 1), (683, 3), (270000, 1)])
@pytest.mark.parametrize("experts", [1, 2, 7, 64, 512])
@pytest.mark.parametrize("dtype, outside", [(torch.int64, 0.0), (torch.int32, 0.2)])
def test_sort(tokens, k, experts, dtype, outside):
    say("expert sort", tokens, k, experts, dtype)
    route = ExpertRoute(tokens + 2, k, experts)
    for seed in (1, 2):                                   # (the second through what the first left)
        ids = ids_of(tokens, k, experts, seed, dtype, outside)
        route.source.fill_(-77)
        offsets = route.sort(ids)
        want, source, slot = R.sort(ids.cpu().numpy(), experts)
        equal(offsets, want, "offsets")
        equal(route.source[:len(source)], source, "source")
        equal(route.slot[:tokens], slot, "slot")
        assert (route.source[len(source):] == -77).all()


def test_sort_of_ids_no_expert_has():
    """Nothing but entries outside, the largest and smallest numbers among them; and no entries."""
    route = ExpertRoute(300, 2, 9)
    big = torch.full((300, 2), 9, dtype=torch.int64, device="cuda")
    big[::3, 0], big[1::3, 1], big[2::3, 0] = -1, 2 ** 63 - 1, -2 ** 63
    big[5, 1] = 2 ** 32                                   # (0 in its low half)
    assert not route.sort(big).any() and (route.slot == -1).all()
    assert not route.sort(big[:0]).any() and route.rows == 0
    one = torch.zeros(300, 2, dtype=torch.int32, device="cuda")
    offsets = route.sort(one)
    assert offsets[0] == 0 and (offsets[1:] == 600).all()
    equal(route.source, np.arange(600), "one expert's")


@pytest.mark.parametrize("tokens, k, experts, cols", [(1, 1, 1, 1), (5, 3, 4, 7), (70, 2, 8, 512), (33, 8, 16, 1001), (3, 5, 64, 8200), (2000, 2, 8, 264), (300, 1, 3, 4096),
                                                      (40, 13, 20, 130)])
@pytest.mark.parametrize("dtype, other", [(F16, F16), (BF16, F32), (F32, F32), (F32, BF16)])
@pytest.mark.parametrize("outside", [0.0, 0.25])
def test_rows_there_and_back(tokens, k, experts, cols, dtype, other, outside):
    say("expert rows", tokens, k, experts, cols, dtype, outside)
    route = ExpertRoute(tokens + 1, k, experts, cols, dtype=dtype)
    ids = ids_of(tokens, k, experts, 3, outside=outside)
    route.sort(ids)
    _, source, slot = R.sort(ids.cpu().numpy(), experts)
    n, rows = len(source), tokens * k
    x, z = values(tokens, cols, dtype, 4, pad=3), values(rows, cols, other, 5, pad=5)
    weight = torch.rand(tokens, k, device="cuda")
    for t in (route.rows_out, route.dz):
        t.fill_(7.0)
    z[n:] = float("nan")                                  # rows of no expert: whatever they hold
    got = route.gather(x)
    equal(got[:n].float(), f64(x)[source // k], "gathered")
    assert got.shape == (rows, cols) and (got[n:] == 7.0).all()
    Z, W = f64(z), f64(weight)
    take = lambda m: np.where((slot >= 0)[:, :, None], m[np.maximum(slot, 0)], 0.0)      # [tokens, k, cols]
    for w, w64 in ((weight, W), (None, np.ones((tokens, k)))):
        terms = w64[:, :, None] * take(Z)
        y = route.combine(z, w)
        assert_within(y, terms.sum(1), k * U * np.abs(terms).sum(1) + rounded(terms.sum(1), dtype) + 2.0 ** -149, "combined")
        dy = values(tokens, cols, other, 6, pad=1)
        dz, dweight = route.combine_backward(dy)
        G = f64(dy)
        want = np.full((rows, cols), 7.0)
        want[:n] = w64.reshape(-1)[source][:, None] * G[source // k]
        assert_within(dz, want, U * np.abs(want) + rounded(want, dtype) + 2.0 ** -149, "rows' gradient")
        dots = take(Z) * G[:, None, :]
        assert_within(dweight, dots.sum(2), (cols + 1) * U * np.abs(dots).sum(2) + 2.0 ** -149, "weights' gradient")
    drows = values(rows, cols, other, 7, pad=2)
    drows[n:] = float("inf")
    dx = route.gather_backward(drows)
    terms = take(f64(drows))
    assert_within(dx, terms.sum(1), k * U * np.abs(terms).sum(1) + rounded(terms.sum(1), dtype) + 2.0 ** -149, "tokens' gradient")


@pytest.mark.parametrize("cols", [*range(1, 19), 31, 33, 63, 65, 255, 257, 2047, 2049, 2055])
@pytest.mark.parametrize("dtype, other", [(F16, F32), (BF16, BF16), (F32, F16)])
def test_rows_of_any_width(cols, dtype, other):
    """A row's last vector overlaps the one before it: nothing is counted twice, nothing beside the row is written."""
    test_rows_there_and_back(9, 3, 4, cols, dtype, other, 0.25)


def test_route_gradients_against_differences():
    tokens, k, experts, cols = 6, 2, 3, 5
    route = ExpertRoute(tokens, k, experts, cols, dtype=F32)
    ids = ids_of(tokens, k, experts, 8, outside=0.2)
    route.sort(ids)
    _, source, slot = R.sort(ids.cpu().numpy(), experts)
    n = len(source)
    z, weight, dy, drows = values(tokens * k, cols, F32, 9), torch.rand(tokens, k, device="cuda"), values(tokens, cols, F32, 10), values(tokens * k, cols, F32, 11)
    route.combine(z, weight)
    dz, dweight = route.combine_backward(dy)
    dx = route.gather_backward(drows)
    Z, W, G, H, X = f64(z), f64(weight), f64(dy), f64(drows)[:n], np.zeros((tokens, cols))

    def combined(z_, w_):
        y = np.zeros((tokens, cols))
        for t, j in np.ndindex(tokens, k):
            if slot[t, j] >= 0:
                y[t] += w_[t, j] * z_[slot[t, j]]
        return (y * G).sum()

    def differences(at, f):                               # (linear: any step)
        out = np.empty(at.shape)
        for i in np.ndindex(at.shape):
            d = np.zeros(at.shape)
            d[i] = 1.0
            out[i] = (f(at + d) - f(at - d)) / 2
        return out

    size = lambda m: 8 * U * np.abs(m).max() * np.abs(G).max()
    assert_within(dz[:n], differences(Z, lambda v: combined(v, W))[:n], size(W) + 1e-12, "dz")
    assert_within(dweight, differences(W, lambda v: combined(Z, v)), cols * size(Z) + 1e-12, "dweight")
    assert_within(dx, differences(X, lambda v: (v[source // k] * H).sum()), 8 * U * np.abs(H).max() + 1e-12, "dx")


def check_expert_step(op, route, ids, x, w, dy, u, what):
    """x [tokens or rows]; one step against a TokenLinear's definition on each expert's rows."""
    y = op.forward(x, route, w=w).clone()
    dx, dw, db = op.backward(dy)
    torch.cuda.synchronize()
    offsets, source, _ = R.sort(ids.cpu().numpy(), op.sets)
    X, W, G = f64(x), f64(w), f64(dy)
    rows = X[source // ids.shape[1]] if op.gather else X[:len(source)]
    for e, (a, b) in enumerate(zip(offsets[:-1], offsets[1:])):
        if a == b:
            assert not dw[e].any() and (db is None or not db[e].any()), f"{what}: expert {e} without rows"
            continue
        want = expected(rows[a:b], W[e], G[a:b], None if op.bias is None else f64(op.bias)[e], None if u is None else u[a:b])
        for name, got in (("y", y[a:b]), ("dx", dx[a:b]), ("dw", dw[e]), ("db", None if db is None else db[e])):
            if got is not None:
                assert_within(got, want[name][0], want[name][1] + rounded(want[name][0], got.dtype), f"{what}, expert {e}: {name}")


@pytest.mark.parametrize("tokens, k, experts, N, K", [(1, 1, 1, 8, 8), (1, 2, 4, 130, 70), (40, 2, 16, 264, 136), (300, 3, 5, 70, 300), (900, 2, 3, 260, 520), (64, 8, 130, 24, 40)])
@pytest.mark.parametrize("dtype, bias, gather", [(F16, True, True), (BF16, False, False), (F32, True, False), (F32, False, True)])
def test_expert_steps(tokens, k, experts, N, K, dtype, bias, gather):
    say("expert step", tokens, k, experts, N, K, dtype, gather)
    route = ExpertRoute(tokens + 1, k, experts)
    op = ExpertLinear((tokens + 1) * k, N, K, experts, x_dtype=dtype, bias=bias, gather=gather, philox_seed=SEED)
    if bias:
        op.bias.copy_(torch.randn(experts, N, device="cuda"))
    for step, outside in enumerate((0.0, 0.3)):
        ids = ids_of(tokens, k, experts, 12 + step, outside=outside)
        route.sort(ids)
        x = values(tokens if gather else tokens * k, K, dtype, 13 + step, pad=1)
        w, dy = values(experts * N, K, F32, 14 + step).view(experts, N, K), values(tokens * k, N, dtype, 15 + step, pad=3)
        u = R.draws(tokens * k, N, SEED, op.offset)
        check_expert_step(op, route, ids, x, w, dy, u, f"step {step}")


def test_rows_without_an_expert_stay_as_they_were():
    route = ExpertRoute(50, 2, 4)
    op = ExpertLinear(100, 72, 40, 4, training=False, gather=False)
    ids = ids_of(50, 2, 4, 20, outside=0.4)
    n = int(route.sort(ids)[-1])
    x = values(100, 40, F16, 21)
    x[n:] = float("nan")
    op.y.fill_(7.0), op.sx.fill_(7.0), op.xq.fill_(7)
    op.convert_w(values(4 * 72, 40, F32, 22).view(4, 72, 40))
    y = op.forward(x, route)
    assert 0 < n < 100 and (y[n:] == 7.0).all() and (op.sx[n:] == 7.0).all() and (op.xq[n:] == 7).all()
    assert not torch.isnan(y[:n]).any()


def test_an_empty_batch_of_experts():
    route = ExpertRoute(4, 2, 3, 40)
    op = ExpertLinear(8, 24, 40, 3, bias=True)
    route.sort(torch.empty(0, 2, dtype=torch.int64, device="cuda"))
    none = torch.empty(0, 40, dtype=F16, device="cuda")
    y = op.forward(none, route, w=values(72, 40, F32, 23).view(3, 24, 40))
    dx, dw, db = op.backward(torch.empty(0, 24, dtype=F16, device="cuda"))
    assert y.shape == (0, 24) and dx.shape == (0, 40) and not dw.any() and not db.any()
    assert route.gather(none).shape == (0, 40) and route.combine(none).shape == (0, 40) and route.gather_backward(none).shape == (0, 40)
    dz, dweight = route.combine_backward(none)
    assert dz.shape == (0, 40) and dweight.shape == (0, 2)
    # ... and one whose entries all lie outside
    ids = torch.full((4, 2), -1, device="cuda")
    route.sort(ids)
    x = values(4, 40, F16, 24)
    op.forward(x, route)
    _, dw, db = op.backward(values(8, 24, F16, 25))
    assert not dw.any() and not db.any() and not route.combine(route.gather(x)).any() and not route.combine_backward(x)[1].any()


class Block:
    """Two experts' linears with a squared ReLU between them, in and out through a route."""

    def __init__(self, tokens, k, experts, C, F, dtype):
        self.route = ExpertRoute(tokens, k, experts, C, dtype=dtype)
        self.up = ExpertLinear(tokens * k, F, C, experts, x_dtype=dtype, philox_seed=SEED)
        self.down = ExpertLinear(tokens * k, C, F, experts, x_dtype=dtype, gather=False, philox_seed=SEED + 1)

    def step(self, ids, weight, x, w_up, w_down, dy):
        self.up.offset = self.down.offset = 0
        self.route.sort(ids)
        h = self.up.forward(x, self.route, w=w_up).relu()
        y = self.route.combine(self.down.forward(h * h, self.route, w=w_down), weight)
        dz, dweight = self.route.combine_backward(dy)
        da, dw_down, _ = self.down.backward(dz)
        drows, dw_up, _ = self.up.backward(2 * h * da)
        return y, dweight, dw_down, dw_up, self.route.gather_backward(drows)


def test_a_block_of_experts():
    """A whole step against 64 bits: each operator on what the ones before it returned."""
    tokens, k, experts, C, F = 200, 2, 6, 136, 264
    block = Block(tokens, k, experts, C, F, F32)
    ids, weight = ids_of(tokens, k, experts, 30, outside=0.1), torch.rand(tokens, k, device="cuda")
    x, dy = values(tokens, C, F32, 31), values(tokens, C, F32, 32)
    w_up, w_down = values(experts * F, C, F32, 33).view(experts, F, C), values(experts * C, F, F32, 34).view(experts, C, F)
    block.up.y.zero_(), block.down.dx.zero_()
    y, dweight, dw_down, dw_up, dx = block.step(ids, weight, x, w_up, w_down, dy)
    offsets, source, slot = R.sort(ids.cpu().numpy(), experts)
    n = len(source)
    X, W1, W2, G, P = f64(x), f64(w_up), f64(w_down), f64(dy), f64(weight)
    # operator by operator, each from the GPU's own result before it
    h64 = np.maximum(f64(block.up.y)[:n], 0.0)
    a32 = (block.up.y.relu() ** 2).double().cpu().numpy()[:n]
    dz = P.reshape(-1)[source][:, None] * G[source // k]
    dz32 = f64(block.route.dz)[:n]
    assert_within(block.route.dz[:n], dz, 2 * U * np.abs(dz) + 2.0 ** -149, "dz")
    da = f64(block.down.dx)[:n]
    dh = (2 * block.up.y.relu() * block.down.dx).double().cpu().numpy()[:n]
    u2, u1 = R.draws(tokens * k, C, SEED + 1, 0), R.draws(tokens * k, F, SEED, 0)
    out = np.zeros((tokens, C))
    for e, (a, b) in enumerate(zip(offsets[:-1], offsets[1:])):
        if a == b:
            continue
        for op, rows, w, g, u in ((block.up, X[source[a:b] // k], W1[e], dh[a:b], u1[a:b]), (block.down, a32[a:b], W2[e], dz32[a:b], u2[a:b])):
            want = expected(rows, w, g, None, u)
            for name, got in (("y", op.y[a:b]), ("dx", op.dx[a:b]), ("dw", op.dw[e])):
                assert_within(got, want[name][0], want[name][1] + rounded(want[name][0], F32), f"expert {e}: {name}")
    take = lambda m: np.where((slot >= 0)[:, :, None], m[np.maximum(slot, 0)], 0.0)
    terms = P[:, :, None] * take(f64(block.down.y))
    assert_within(y, terms.sum(1), 3 * U * np.abs(terms).sum(1) + 2.0 ** -149, "y")
    assert_within(dx, take(f64(block.up.dx)).sum(1), 3 * U * np.abs(take(f64(block.up.dx))).sum(1) + 2.0 ** -149, "dx")
    dots = take(f64(block.down.y)) * G[:, None, :]
    assert_within(dweight, dots.sum(2), (C + 1) * U * np.abs(dots).sum(2) + 2.0 ** -149, "dweight")


def bits(t):
    """(sums of this size pass the range of binary16, and a NaN equals none)"""
    return t.view({2: torch.int16, 4: torch.int32}[t.element_size()])


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
def test_graph_replays_equal_eager(dtype):
    """A block's step captured, and replayed over batches whose experts have other numbers of rows."""
    tokens, k, experts, C, F = 150, 2, 5, 136, 264
    ids, weight = ids_of(tokens, k, experts, 40), torch.rand(tokens, k, device="cuda")
    x, dy = values(tokens, C, dtype, 41), values(tokens, C, dtype, 42)
    w_up, w_down = values(experts * F, C, F32, 43).view(experts, F, C), values(experts * C, F, F32, 44).view(experts, C, F)
    args = (ids, weight, x, w_up, w_down, dy)
    block, eager = Block(tokens, k, experts, C, F, dtype), Block(tokens, k, experts, C, F, dtype)
    for b in (block, eager):
        for t in (b.up.y, b.up.dx, b.down.y, b.down.dx, b.route.dz):
            t.zero_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        block.step(*args)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = block.step(*args)
    for replay in range(4):
        say("experts graph", replay)
        ids.copy_(ids_of(tokens, k, experts, 50 + replay, outside=0.2 * replay))
        x.copy_(values(tokens, C, dtype, 60 + replay))
        want = [t.clone() for t in eager.step(*args)]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for i, (a, b) in enumerate(zip(out, want)):
            assert torch.equal(bits(a), bits(b)), (replay, i)


def test_rows_that_pass_32_bits():
    """More than 2^31 elements of gathered rows: the last ones of each pass."""
    tokens, k, experts, cols = 600_000, 2, 3, 1800
    say("expert rows, large")
    route = ExpertRoute(tokens, k, experts, cols, dtype=F16)
    ids = torch.randint(0, experts, (tokens, k), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    route.sort(ids)
    x = torch.empty(tokens, cols, dtype=F16, device="cuda")
    x.copy_((torch.arange(tokens, device="cuda") % 1999)[:, None].to(F16))
    x += (torch.arange(cols, device="cuda") % 8).to(F16)
    rows = route.gather(x)
    token = route.source.long() // k
    for part in (slice(0, 1000), slice(-1000, None)):
        assert torch.equal(rows[part], x[token[part]])
    y = route.combine(rows)
    assert torch.equal(y[-1000:], 2 * x[-1000:])
    dz, dweight = route.combine_backward(x)
    assert torch.equal(dz[-1000:], x[token[-1000:]])
    del dz, rows
    want = (x[-10:].double() ** 2).sum(1)
    assert ((dweight[-10:].double() - want[:, None]).abs() <= cols * U * want[:, None]).all()


def test_calls_out_of_their_order_are_refused():
    route, other = ExpertRoute(20, 2, 3, 16), ExpertRoute(20, 2, 4)
    op = ExpertLinear(40, 24, 16, 3, gather=False)
    ids, x = ids_of(20, 2, 3, 70), values(40, 16, F16, 71)
    for r in (route, other):
        r.sort(ids)
    with pytest.raises(RuntimeError, match="weights"):
        op.forward(x, route)
    with pytest.raises(ValueError, match="experts"):
        op.forward(x, other, w=torch.zeros(3, 24, 16, device="cuda"))
    w, dy = values(72, 16, F32, 72).view(3, 24, 16), values(40, 24, F16, 73)
    op.forward(x, route, w=w)
    for bad, error in ((dy[:39], ValueError), (dy.t(), ValueError), (dy.double(), ValueError), (dy.cpu(), ValueError)):
        with pytest.raises(error):
            op.backward(bad)
    with pytest.raises(ValueError, match="w:"):
        op.forward(x, route, w=w[:2])
    with pytest.raises(ValueError, match="x"):
        op.forward(x[:20], route)
    with pytest.raises(ValueError, match="cols"):
        other.gather(x[:20])
    with pytest.raises(ValueError, match="expected, not"):
        route.gather(values(20, 16, F32, 74))
    with pytest.raises(RuntimeError, match="combine"):
        route.combine_backward(x[:20])
    with pytest.raises(ValueError, match="weight"):
        route.combine(x, torch.ones(20, 2, device="cuda", dtype=torch.float64))
    with pytest.raises(RuntimeError, match="training"):
        ExpertRoute(20, 2, 3, 16, training=False).gather_backward(x)
    op.backward(dy)
    route.sort(ids)
    with pytest.raises(RuntimeError, match="another batch"):
        op.backward(dy)


def test_serving_in_graphs():
    """A few tokens to their experts and back, and through a token linear, captured and replayed over other tokens, ids and numbers of rows an
    expert; two graphs that share the operators' buffers."""
    from paper_2407_02327_amd.experts import TokenLinear
    T, k, E, C, F = 8, 2, 4, 256, 512
    route, up = ExpertRoute(T, k, E, C, training=False), ExpertLinear(T * k, F, C, E, training=False)
    down, last = ExpertLinear(T * k, C, F, E, gather=False, training=False), TokenLinear(T, 130, C, training=False)
    up.convert_w(values(E * F, C, F32, 80).view(E, F, C) / 64), down.convert_w(values(E * C, F, F32, 81).view(E, C, F) / 64), last.convert_w(values(130, C, F32, 82))
    x, ids, weight = values(T, C, F16, 83).clamp(-4, 4), ids_of(T, k, E, 84), torch.rand(T, k, device="cuda")
    for t in (up.y, down.y):
        t.zero_()

    def step(n):
        route.sort(ids[:n])
        y = route.combine(down.forward(up.forward(x[:n], route).relu(), route), weight[:n])
        return y, last.forward(y)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(T), step(1)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graphs = []
    for n in (T, 1):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            out = step(n)
        graphs.append((n, g, out))
    for replay in range(3):
        x.copy_(values(T, C, F16, 85 + replay).clamp(-4, 4))
        ids.copy_(ids_of(T, k, E, 90 + replay, outside=0.2 * replay))
        for n, g, out in graphs:
            say("serving graph", replay, n)
            want = [t.clone() for t in step(n)]
            for t in out:
                t.zero_()
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            for a, b in zip(out, want):
                assert torch.equal(bits(a), bits(b)), (replay, n)
