"""INT8 products with a scale for each token and channel on the GPU: codes and scales bit for bit, products within bounds that count
roundings (token_ref)."""
import numpy as np
import pytest
import torch

from paper_2407_02327_amd import qsync as Q
from paper_2407_02327_amd.experts import TokenLinear
from tests import token_ref as R
from tests.gpu_util import say
from tests.head_ref import U, f64, rounded
from tests.token_ref import assert_within

pytestmark = pytest.mark.gpu
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
SEED, OFFSET = 0x0123456789ABCDEF, (1 << 32) - 5          # (counters that pass 32 bits)
# (rows, cols): every way of dividing a row among lanes, both sides of each limit, odd and long ones
SIZES = [(1, 1), (3, 7), (5, 128), (9, 129), (6, 512), (130, 520), (33, 1001), (4, 1024), (3, 1025), (2, 2048), (2, 2056), (3, 4097), (2, 8192), (1, 8200),
         (2, 20001), (300, 64)]


def values(rows, cols, dtype, seed, pad=0):
    """Rows of different size, some zero; `pad`: elements between them."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = torch.randn(rows, cols + pad, generator=g, device="cuda") * torch.exp(2.0 * torch.randn(rows, 1, generator=g, device="cuda"))
    if rows > 4:
        t[3] = 0.0
    return t.to(dtype)[:, pad // 2:pad // 2 + cols]


def equal(got, want, what):
    got = got.detach().cpu().numpy()
    same = (got == want) | (np.isnan(got) & np.isnan(want)) if got.dtype.kind == "f" else got == want
    i = np.argwhere(~same)
    assert i.size == 0, f"{what}: {len(i)} of {got.size} differ, first at {tuple(i[0])}: got {got[tuple(i[0])]}, want {want[tuple(i[0])]}"


def quantize(x, rnd, source=None, group=1, rows=None, count=None):
    rows = x.shape[0] if rows is None else rows
    cols = x.shape[1]
    q = torch.full((rows, R.pad(cols)), 77, dtype=torch.int8, device="cuda")
    s = torch.full((rows,), -7.0, device="cuda")
    Q.qsync_token_quantize(x, x.shape[0], cols, max(x.stride(0), cols), source, group, rows, count, rnd, SEED, OFFSET, s, q)
    torch.cuda.synchronize()
    return q, s


def quantize_both(x, sets, offsets, rnd, sums=True, source=None, group=1, rows=None):
    rows = x.shape[0] if rows is None else rows
    cols = x.shape[1]
    given = offsets is not None
    q = torch.full((rows, R.pad(cols)), 77, dtype=torch.int8, device="cuda")
    s = torch.full((rows,), -7.0, device="cuda")
    qT = torch.full((Q.qsync_token_code_rows(rows, sets, given) * cols,), 77, dtype=torch.int8, device="cuda")
    sc, total = torch.full((sets, cols), -7.0, device="cuda"), torch.full((sets, cols), -7.0, device="cuda")
    ws = torch.empty(max(16, Q.qsync_token_quantize_both_workspace_bytes(rows, cols, sets, given)), dtype=torch.uint8, device="cuda").random_()
    Q.qsync_token_quantize_both(x, x.shape[0], cols, max(x.stride(0), cols), source, group, rows, sets, offsets, rnd, SEED, OFFSET, s, q, sc, qT,
                                total if sums else None, ws)
    torch.cuda.synchronize()
    return q, s, qT, sc, total


def check_rows(q, s, x, u, what):
    n, cols = x.shape
    wq, ws = R.codes(x, 1, u)
    equal(s[:n], ws, what + " scales")
    equal(q[:n, :cols], wq, what + " codes")
    assert not q[:n, cols:].any(), what + ": padding"
    assert (q[n:] == 77).all() and (s[n:] == -7.0).all(), what + ": rows behind the last"


@pytest.mark.parametrize("rows, cols", SIZES)
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("rnd", [Q.ROUND_NEAREST, Q.ROUND_STOCHASTIC])
def test_quantize_rows(rows, cols, dtype, rnd):
    say("token quantize", rows, cols, dtype, rnd)
    x = values(rows, cols, dtype, 1, pad=3)                  # (rows that start at any element)
    u = R.draws(rows, cols, SEED, OFFSET) if rnd else None
    check_rows(*quantize(x, rnd), f64(x), u, f"{rows}x{cols}")


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_that_are_not_ordinary(dtype):
    """Nothing but zeros, values whose inverse would overflow, the smallest and largest ones, infinities and NaN: none touches another row."""
    rows, cols = 12, 300
    x = values(rows, cols, F32, 2)
    x[1], x[2] = 0.0, 2.0 ** -101
    x[3] *= 2.0 ** -100 / x[3].abs().max().clamp(min=1e-30)
    x[4] = 1e-45
    x[5] *= torch.finfo(dtype).max / x[5].abs().max()
    x[6, 7], x[7, 0], x[8, 299] = float("inf"), float("-inf"), float("nan")
    x[9] = float("-inf")
    x = x.to(dtype)
    for rnd in (Q.ROUND_NEAREST, Q.ROUND_STOCHASTIC):
        u = R.draws(rows, cols, SEED, OFFSET) if rnd else None
        q, s = quantize(x, rnd)
        check_rows(q, s, f64(x), u, "rows")
        qb, sb, qT, sc, total = quantize_both(x, 1, None, rnd)
        check_rows(qb, sb, f64(x), u, "both")
        wq, ws = R.codes(f64(x), 0, u)
        equal(sc[0], ws, "columns' scales")
        assert np.isnan(ws).sum() == 300                      # (row 9 reaches every column)


@pytest.mark.parametrize("rnd", [Q.ROUND_NEAREST, Q.ROUND_STOCHASTIC])
def test_rows_taken_through_a_source(rnd):
    """Rows of tokens in any order, places outside of them, and rows behind the last, which stay as they were."""
    x = values(20, 150, F16, 3)
    source = torch.tensor([5, 0, 59, 59, 31, 2, 60, -1, 2 ** 31 - 1, 8, 1, 4], dtype=torch.int32, device="cuda")
    count = torch.tensor([10], dtype=torch.int32, device="cuda")
    q, s = quantize(x, rnd, source, 3, 12, count)
    rows = np.array([1, 0, 19, 19, 10, 0, -1, -1, -1, 2])
    want = f64(x)[np.maximum(rows, 0)]
    want[rows < 0] = np.nan
    check_rows(q, s, want, R.draws(12, 150, SEED, OFFSET)[:10] if rnd else None, "source")


def layouts():
    """(rows, sets, offsets or None)"""
    return [(1, 1, None), (127, 1, None), (300, 1, None), (12, 3, None), (390, 3, None), (5, 1, [0, 5]), (300, 4, [0, 0, 129, 129, 290]),
            (260, 3, [0, 128, 256, 260]), (64, 5, [0, 1, 2, 40, 40, 40]), (9, 2, [0, 0, 0]), (600, 512, list(range(0, 513)))]


@pytest.mark.parametrize("rows, sets, offsets", layouts())
@pytest.mark.parametrize("dtype, cols, rnd", [(F32, 77, Q.ROUND_STOCHASTIC), (F16, 128, Q.ROUND_NEAREST), (BF16, 1030, Q.ROUND_STOCHASTIC), (F16, 520, Q.ROUND_STOCHASTIC)])
def test_quantize_both(rows, sets, offsets, dtype, cols, rnd):
    say("token quantize both", rows, sets, offsets and offsets[:6], dtype, cols, rnd)
    x = values(rows, cols, dtype, 4, pad=5)
    given = None if offsets is None else torch.tensor(offsets, dtype=torch.int32, device="cuda")
    bounds = offsets if offsets is not None else [rows // sets * e for e in range(sets + 1)]
    q, s, qT, sc, total = quantize_both(x, sets, given, rnd)
    x64, u, n = f64(x), R.draws(rows, cols, SEED, OFFSET) if rnd else None, bounds[-1]
    check_rows(q, s, x64[:n], None if u is None else u[:n], "rows")
    flat = qT.cpu().numpy()
    wq, ws, wt = np.zeros((n, cols), np.int64), np.ones((sets, cols), np.float32), np.zeros((sets, cols))
    bound = np.zeros((sets, cols))
    for e, (a, b) in enumerate(zip(bounds[:-1], bounds[1:])):
        if b > a:
            wq[a:b], ws[e] = R.codes(x64[a:b], 0, None if u is None else u[a:b])
            wt[e], bound[e] = x64[a:b].sum(0), (b - a) * U * np.abs(x64[a:b]).sum(0)
    equal(sc, ws, "columns' scales")
    assert_within(total, wt, bound + 2.0 ** -149, "columns' sums")
    for e, (start, m) in R.transposed_layout(wq, bounds, offsets is not None).items():
        assert np.array_equal(flat[start:start + m.size].reshape(m.shape), m), f"codes along the rows of set {e}"


def test_quantize_both_through_a_source():
    x = values(40, 200, BF16, 5)
    ids = torch.randint(0, 4, (40, 2), generator=torch.Generator().manual_seed(1)).numpy()
    offsets, source, _ = R.sort(ids, 4)
    q, s, qT, sc, _ = quantize_both(x, 4, torch.from_numpy(offsets).cuda(), Q.ROUND_NEAREST, source=torch.from_numpy(source).cuda(), group=2, rows=80)
    rows = f64(x)[source // 2]
    check_rows(q, s, rows, None, "rows")
    for e in range(4):
        a, b = offsets[e], offsets[e + 1]
        equal(sc[e], R.codes(rows[a:b], 0)[1], "columns")
    for e, (start, m) in R.transposed_layout(np.concatenate([R.codes(rows[a:b], 0)[0] for a, b in zip(offsets[:-1], offsets[1:])]), offsets, True).items():
        assert np.array_equal(qT.cpu().numpy()[start:start + m.size].reshape(m.shape), m), e


# ---- products -------------------------------------------------------------------------------------------------------------------

def random_codes(rows, cols, g):
    q = torch.zeros(rows, R.pad(cols), dtype=torch.int8, device="cuda")
    q[:, :cols] = torch.randint(-127, 128, (rows, cols), generator=g, device="cuda", dtype=torch.int8)
    return q


PRODUCTS = [(1, 1, 1), (1, 1000, 130), (3, 17, 4096), (16, 64, 64), (17, 4096, 256), (64, 130, 8200), (65, 129, 1024), (100, 768, 6144), (128, 128, 128), (129, 257, 385),
            (200, 2000, 512), (1000, 24, 700), (300, 520, 2048), (1030, 1000, 260), (2, 20000, 64), (4100, 300, 128), (2050, 2056, 136)]


@pytest.mark.parametrize("M, N, K", PRODUCTS)
@pytest.mark.parametrize("dtype, bias", [(F32, True), (F16, False), (BF16, True)])
def test_products(M, N, K, dtype, bias):
    say("token product", M, N, K, dtype, bias)
    g = torch.Generator(device="cuda").manual_seed(6)
    a, b = random_codes(M, K, g), random_codes(N, K, g)
    sa, sb = torch.rand(M, generator=g, device="cuda") * 1e-3 + 1e-5, torch.rand(N, generator=g, device="cuda") * 1e-2
    bs = torch.randn(N, generator=g, device="cuda") if bias else None
    y = torch.full((M, N), 7.0, dtype=dtype, device="cuda")
    ws = torch.empty(Q.qsync_token_linear_workspace_bytes(M, N, K, 1) + 16, dtype=torch.uint8, device="cuda").random_()
    Q.qsync_token_linear_fwd(M, N, K, 1, None, a, sa, b, sb, bs, y, ws)
    torch.cuda.synchronize()
    want, bound = R.product(f64(a), sa.cpu().numpy(), f64(b), sb.cpu().numpy(), None if bs is None else f64(bs))
    assert_within(y, want, bound + rounded(want, dtype), f"{M}x{N}x{K}")


@pytest.mark.parametrize("M, N, K", [(100, 120, 16384), (300, 257, 9000), (64, 64, 100000), (1000, 130, 4096)])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_room_does_not_change_results(M, N, K, dtype):
    """A long contraction in as many pieces as the workspace holds: forward and weight gradient, bit for bit."""
    say("token product room", M, N, K, dtype)
    g = torch.Generator(device="cuda").manual_seed(16)
    a, b = random_codes(M, K, g), random_codes(N, K, g)
    sa, sb, bias = torch.rand(M, device="cuda") * 1e-3, torch.rand(N, device="cuda") * 1e-2, torch.randn(N, device="cuda")
    whole = Q.qsync_token_linear_workspace_bytes(M, N, K, 1)
    assert whole >= 2 * M * N * 4 and Q.qsync_token_wgrad_workspace_bytes(K, M, N, 1) >= 2 * M * N * 4
    out = []
    for room in (0, 3 * M * N * 4 // 2, 2 * M * N * 4 + 16, whole):
        ws = torch.empty(max(room, 16), dtype=torch.uint8, device="cuda").random_()[:room] if room else None
        y, dw = torch.full((M, N), 7.0, dtype=dtype, device="cuda"), torch.full((M, N), 7.0, dtype=dtype, device="cuda")
        Q.qsync_token_linear_fwd(M, N, K, 1, None, a, sa, b, sb, bias, y, ws)
        Q.qsync_token_linear_wgrad(K, M, N, 1, None, a, sa, b, sb, dw, ws)
        torch.cuda.synchronize()
        out.append((y, dw))
    want, bound = R.product(f64(a), sa.cpu().numpy(), f64(b), sb.cpu().numpy(), f64(bias))
    assert_within(out[0][0], want, bound + rounded(want, dtype), "y")
    want, bound = R.product(f64(a), sa.cpu().numpy(), f64(b), sb.cpu().numpy())
    assert_within(out[0][1], want, bound + rounded(want, dtype), "dw")
    for y, dw in out[1:]:
        assert torch.equal(y, out[0][0]) and torch.equal(dw, out[0][1])


@pytest.mark.parametrize("rows, N, K, offsets, dtype", [(4200, 4096, 100, None, F32), (8200, 4096, 256, None, BF16), (4200, 4096, 300, [0, 1500, 1500, 4133], F32),
                                                        (8200, 4096, 128, [0, 257, 5000, 8190], F16)])
def test_many_outputs_of_short_contractions(rows, N, K, offsets, dtype):
    """Forward and weight gradient (K rows a set), on each tile and the one of the rule: the same bits, and some of the rows against the formula."""
    say("token product, short contraction", rows, N, K, offsets, dtype)
    g = torch.Generator(device="cuda").manual_seed(26)
    sets = len(offsets) - 1 if offsets else 1
    at = [0, rows] if offsets is None else offsets
    a, b = random_codes(rows, K, g), random_codes(sets * N, K, g)
    sa, sb = torch.rand(rows, generator=g, device="cuda") * 1e-3, torch.rand(sets, N, generator=g, device="cuda") * 1e-2
    off = None if offsets is None else torch.tensor(offsets, dtype=torch.int32, device="cuda")
    M = rows // sets
    woff = None if offsets is None else torch.tensor([K * i for i in range(sets + 1)], dtype=torch.int32, device="cuda")
    positions = Q.qsync_token_code_rows(K * sets, sets, offsets is not None)
    c, d = torch.zeros(positions * M, dtype=torch.int8, device="cuda"), torch.zeros(positions * N, dtype=torch.int8, device="cuda")
    for e in range(sets):      # set e: a packed matrix [.., pad(K)] from position pad(K e) + 128 e on
        start = (R.pad(K * e) + 128 * e) if offsets else 0
        c[start * M:(start + R.pad(K)) * M] = random_codes(M, K, g).flatten()
        d[start * N:(start + R.pad(K)) * N] = random_codes(N, K, g).flatten()
    sc, sd = torch.rand(sets, M, generator=g, device="cuda") * 1e-3, torch.rand(sets, N, generator=g, device="cuda") * 1e-2
    out = []
    try:
        for tile in (-1, 0, 1, 2):
            Q.qsync_debug_set_gemm_tile(tile)
            y, dw = torch.full((rows, N), 7.0, dtype=dtype, device="cuda"), torch.full((sets, M, N), 7.0, dtype=dtype, device="cuda")
            Q.qsync_token_linear_fwd(rows, N, K, sets, off, a, sa, b, sb, None, y, None)
            Q.qsync_token_linear_wgrad(K * sets, M, N, sets, woff, c, sc, d, sd, dw, None)
            torch.cuda.synchronize()
            out.append((y, dw))
    finally:
        Q.qsync_debug_set_gemm_tile(-1)
    for y, dw in out[1:]:
        assert torch.equal(y, out[0][0]) and torch.equal(dw, out[0][1])
    y, dw = out[0]
    assert (y[at[-1]:] == 7.0).all()
    for e, (i, j) in enumerate(zip(at[:-1], at[1:])):
        some = sorted({i, (i + j) // 2, j - 1}) if j > i else []
        if some:
            want, bound = R.product(f64(a)[some], sa.cpu().numpy()[some], f64(b[e * N:(e + 1) * N]), sb.cpu().numpy()[e])
            assert_within(y[some], want, bound + rounded(want, dtype), f"y of set {e}")
        some, start = [0, 255, 256, M // 2, M - 1], (R.pad(K * e) + 128 * e) if offsets else 0
        rows_of = lambda t, n: f64(t[start * n:(start + R.pad(K)) * n]).reshape(n, R.pad(K))
        want, bound = R.product(rows_of(c, M)[some], sc.cpu().numpy()[e][some], rows_of(d, N), sd.cpu().numpy()[e])
        assert_within(dw[e][some], want, bound + rounded(want, dtype), f"dw of set {e}")


SETS = [(40, 5, [0, 3, 3, 20, 40, 40]), (700, 3, [0, 1, 650, 690]), (2000, 16, [0] + [125 * i - 60 for i in range(1, 16)] + [1990]), (6, 64, [0] * 30 + [2] * 20 + [6] * 15),
        (900, 1, [0, 900]), (513, 2, [0, 256, 513]), (5, 2, [0, 0, 0]), (4000, 7, [0, 600, 600, 1300, 2500, 2501, 3100, 4000])]


@pytest.mark.parametrize("rows, sets, offsets", SETS)
@pytest.mark.parametrize("N, K, dtype", [(33, 70, F32), (264, 1024, BF16), (1024, 300, F16), (100, 4100, F16), (96, 9000, F32)])
def test_products_of_sets(rows, sets, offsets, N, K, dtype):
    """Each set with weights of its own; rows that belong to none stay as they were."""
    say("token product of sets", rows, sets, N, K, dtype)
    g = torch.Generator(device="cuda").manual_seed(7)
    a, b = random_codes(rows, K, g), random_codes(sets * N, K, g)
    sa, sb = torch.rand(rows, generator=g, device="cuda") * 1e-3, torch.rand(sets, N, generator=g, device="cuda") * 1e-2
    bs = torch.randn(sets, N, generator=g, device="cuda")
    y = torch.full((rows, N), 7.0, dtype=dtype, device="cuda")
    ws = torch.empty(Q.qsync_token_linear_workspace_bytes(rows, N, K, sets) + 16, dtype=torch.uint8, device="cuda").random_()
    Q.qsync_token_linear_fwd(rows, N, K, sets, torch.tensor(offsets, dtype=torch.int32, device="cuda"), a, sa, b, sb, bs, y, ws)
    torch.cuda.synchronize()
    a64, b64 = f64(a), f64(b).reshape(sets, N, -1)
    want, bound = np.full((rows, N), 7.0), np.zeros((rows, N))
    for e, (i, j) in enumerate(zip(offsets[:-1], offsets[1:])):
        want[i:j], bound[i:j] = R.product(a64[i:j], sa.cpu().numpy()[i:j], b64[e], sb.cpu().numpy()[e], f64(bs)[e])
    n = offsets[-1]
    assert (y[n:] == 7.0).all()
    assert_within(y[:n], want[:n], bound[:n] + rounded(want[:n], dtype), "sets")


@pytest.mark.parametrize("rows, sets, offsets", SETS + [(1, 1, None), (384, 1, None), (5000, 1, None)])
@pytest.mark.parametrize("N, K, dtype", [(33, 70, F32), (264, 520, F16), (300, 64, BF16)])
def test_weight_gradients(rows, sets, offsets, N, K, dtype):
    say("token weight gradient", rows, sets, N, K, dtype)
    g = torch.Generator(device="cuda").manual_seed(8)
    given = offsets is not None
    bounds = offsets if given else [0, rows]
    n = bounds[-1]
    q = {}
    sides = []
    for side, cols in (("dy", N), ("x", K)):
        q[side] = torch.randint(-127, 128, (n, cols), generator=g, device="cuda").cpu().numpy()
        flat = np.full(Q.qsync_token_code_rows(rows, sets, given) * cols, 99, np.int8)
        for start, m in R.transposed_layout(q[side], bounds, given).values():
            flat[start:start + m.size] = m.reshape(-1)
        sides.append((torch.from_numpy(flat).cuda(), torch.rand(sets, cols, generator=g, device="cuda") * 1e-2))
    dw = torch.full((sets, N, K), 7.0, dtype=dtype, device="cuda")
    ws = torch.empty(Q.qsync_token_wgrad_workspace_bytes(rows, N, K, sets) + 16, dtype=torch.uint8, device="cuda").random_()
    Q.qsync_token_linear_wgrad(rows, N, K, sets, torch.tensor(offsets, dtype=torch.int32, device="cuda") if given else None, *sides[0], *sides[1], dw, ws)
    torch.cuda.synchronize()
    for e, (i, j) in enumerate(zip(bounds[:-1], bounds[1:])):
        want, bound = R.product(q["dy"][i:j].T, sides[0][1][e].cpu().numpy(), q["x"][i:j].T, sides[1][1][e].cpu().numpy())
        assert_within(dw[e], want, bound + rounded(want, dtype), f"set {e}")


@pytest.mark.parametrize("rows, N, K, sets, offsets", [(300, 200, 130, 1, None), (2187, 1001, 777, 1, None), (5, 40, 30, 1, None), (700, 90, 300, 4, [0, 100, 100, 690, 695]),
                                                       (3000, 520, 264, 30, [100 * i - (i % 3) * 7 for i in range(31)]), (9, 16, 16, 3, [0, 0, 0, 0]), (9000, 1100, 1500, 1, None)])
@pytest.mark.parametrize("x_dtype, w_dtype", [(F16, F32), (F32, BF16), (BF16, F16)])
def test_calls_that_join_two(rows, N, K, sets, offsets, x_dtype, w_dtype):
    """Conversion of both operands, and both gradients, in one call each: the bits of the separate calls, whatever the buffers held."""
    say("token linear, joined calls", rows, N, K, sets, x_dtype)
    given = None if offsets is None else torch.tensor(offsets, dtype=torch.int32, device="cuda")
    n, routed = rows if offsets is None else offsets[-1], offsets is not None
    x, w, dy = values(rows, K, x_dtype, 17, pad=3), values(sets * N, K, w_dtype, 18).contiguous(), values(rows, N, x_dtype, 19)
    xq, sx, xqT, sxc, _ = quantize_both(x, sets, given, Q.ROUND_NEAREST, sums=False)
    wq, sw, wqT, swc, _ = quantize_both(w, sets, None, Q.ROUND_NEAREST, sums=False)
    dq, sd, dqT, sdc, _ = quantize_both(dy, sets, given, Q.ROUND_STOCHASTIC)
    like = [torch.full_like(t, 77 if t.dtype == torch.int8 else -7) for t in (sx, xq, sxc, xqT, sw, wq, swc, wqT)]
    ws = [torch.empty(Q.qsync_token_quantize_both_workspace_bytes(*a), dtype=torch.uint8, device="cuda").random_() for a in ((rows, K, sets, routed), (sets * N, K, sets, False))]
    Q.qsync_token_convert(x, rows, K, x.stride(0), None, 1, rows, sets, given, *like[:4], w, N, *like[4:], *ws)
    torch.cuda.synchronize()
    for a, b in zip(like, (sx, xq, sxc, xqT, sw, wq, swc, wqT)):
        assert torch.equal(a, b)
    room = torch.empty(Q.qsync_token_linear_bwd_workspace_bytes(rows, N, K, sets) + 16, dtype=torch.uint8, device="cuda").random_()
    out = []
    for joined in (False, True):
        dx, dw = torch.full((rows, K), 7.0, dtype=x_dtype, device="cuda"), torch.full((sets, N, K), 7.0, device="cuda")
        if joined:
            Q.qsync_token_linear_bwd(rows, N, K, sets, given, dq, sd, wqT, swc, dqT, sdc, xqT, sxc, dx, dw, room)
        else:
            Q.qsync_token_linear_fwd(rows, K, N, sets, given, dq, sd, wqT, swc, None, dx, room)
            Q.qsync_token_linear_wgrad(rows, N, K, sets, given, dqT, sdc, xqT, sxc, dw, room)
        torch.cuda.synchronize()
        out.append((dx, dw))
    assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1]) and (out[1][0][n:] == 7.0).all()


def test_an_empty_contraction():
    """No features to sum over: the bias, and zeros."""
    one, codes = torch.ones(4, device="cuda"), torch.zeros(256, dtype=torch.int8, device="cuda")
    y, dx, dw = (torch.full((4, 3), 7.0, device="cuda") for _ in range(3))
    Q.qsync_token_linear_fwd(4, 3, 0, 1, None, codes, one, codes, one, one, y, None)
    Q.qsync_token_linear_wgrad(0, 4, 3, 1, None, codes, one, codes, one, dw, None)
    Q.qsync_token_linear_bwd(4, 0, 3, 1, None, codes, one, codes, one, codes, one, codes, one, dx, dw, None)
    torch.cuda.synchronize()
    assert (y == 1.0).all() and not dx.any() and not dw.any()


def test_accumulators_at_their_largest():
    """All codes 127 over a contraction whose sums need 25 bits and more: exact until the conversion to 32 bits."""
    M, N, K = 70, 90, 130000
    a = torch.zeros(M, R.pad(K), dtype=torch.int8, device="cuda")
    a[:, :K] = 127
    b = torch.zeros(N, R.pad(K), dtype=torch.int8, device="cuda")
    b[:, :K] = -127
    b[::2, :K] = 126
    one, y = torch.ones(M, device="cuda"), torch.empty(M, N, device="cuda")
    ws = torch.empty(Q.qsync_token_linear_workspace_bytes(M, N, K, 1) + 16, dtype=torch.uint8, device="cuda")
    Q.qsync_token_linear_fwd(M, N, K, 1, None, a, one, b, torch.ones(N, device="cuda"), None, y, ws)
    want = np.where(np.arange(N) % 2 == 0, 127.0 * 126 * K, -127.0 * 127 * K).astype(np.float32)
    equal(y, np.broadcast_to(want, (M, N)), "sums")


# ---- the operator ---------------------------------------------------------------------------------------------------------------

def expected(x, w, dy, bias, u):
    """{name: (value, bound)} of a training step, from 64-bit copies."""
    xq, sx = R.codes(x, 1)
    wq, sw = R.codes(w, 1)
    wc, swc = R.codes(w, 0)
    dq, sd = R.codes(dy, 1, u)
    dc, sdc = R.codes(dy, 0, u)
    xc, sxc = R.codes(x, 0)
    return {"y": R.product(xq, sx, wq, sw, bias), "dx": R.product(dq, sd, wc.T, swc), "dw": R.product(dc.T, sdc, xc.T, sxc),
            "db": (dy.sum(0), len(dy) * U * np.abs(dy).sum(0) + 2.0 ** -149)}


def check_step(op, x, w, dy, u, what, **kw):
    y = op.forward(x, w=w, **kw).clone()
    dx, dw, db = op.backward(dy, **kw)
    torch.cuda.synchronize()
    want = expected(f64(x), f64(w), f64(dy), None if op.bias is None else f64(op.bias), u)
    for name, got in (("y", y), ("dx", dx), ("dw", dw), ("db", db)):
        if got is not None:
            assert_within(got, want[name][0], want[name][1] + rounded(want[name][0], got.dtype), f"{what} {name}")


@pytest.mark.parametrize("n, N, K", [(1, 1, 1), (1, 300, 129), (130, 33, 70), (257, 264, 1000), (1000, 1030, 256)])
@pytest.mark.parametrize("x_dtype, dy_dtype, w_dtype", [(F16, F16, F32), (BF16, BF16, BF16), (F32, F32, F16), (F32, BF16, F32)])
def test_training_steps(n, N, K, x_dtype, dy_dtype, w_dtype):
    say("token linear step", n, N, K, x_dtype, dy_dtype)
    op = TokenLinear(n + 3, N, K, x_dtype=x_dtype, dx_dtype=dy_dtype, philox_seed=SEED)
    op.bias.copy_(torch.randn(N, device="cuda"))
    w = values(N, K, w_dtype, 9).contiguous()
    for step in range(2):                                     # (the second with other draws, through buffers that hold the first's)
        u = R.draws(n, N, SEED, op.offset)
        check_step(op, values(n, K, x_dtype, 10 + step, pad=2), w, values(n, N, dy_dtype, 20 + step, pad=4), u, f"step {step}")


def test_gradients_against_differences():
    """The product is linear in each argument, so differences of the unquantized loss are its gradients; the quantized ones differ by
    at most half a step (stochastic: a step) of each operand."""
    n, N, K = 40, 24, 56
    op = TokenLinear(n, N, K, x_dtype=F32)
    x, w, dy = values(n, K, F32, 30), values(N, K, F32, 31), values(n, N, F32, 32)
    op.forward(x, w=w)
    dx, dw, db = op.backward(dy)
    X, W, G = f64(x), f64(w), f64(dy)
    loss = lambda x_, w_, b_: (G * (x_ @ w_.T + b_)).sum()
    zero = np.zeros(N)

    def differences(at, f, h=0.5):
        out = np.empty(at.shape)
        for i in np.ndindex(at.shape):
            step = np.zeros(at.shape)
            step[i] = h
            out[i] = (f(at + step) - f(at - step)) / (2 * h)
        return out

    half = lambda t, axis: np.broadcast_to(np.abs(t).max(axis, keepdims=True) / 127 / 2, t.shape)

    def bound(a, ea, b, eb):                                  # of a @ b with operands off by ea, eb
        return np.abs(a) @ eb + ea @ np.abs(b) + ea @ eb

    checks = (("dx", dx, differences(X, lambda v: loss(v, W, zero)), bound(G, 2 * half(G, 1), W, half(W, 0))),
              ("dw", dw, differences(W, lambda v: loss(X, v, zero)), bound(G.T, 2 * half(G, 0).T, X, half(X, 0))),
              ("db", db, differences(zero, lambda v: loss(X, W, v)), n * U * np.abs(G).sum(0)))
    for name, got, want, b in checks:
        # (differences of a loss of this size lose some of 53 bits: 1e-9 of the largest gradient)
        assert_within(got, want, b * (1 + 1e-5) + 1e-9 * np.abs(want).max(), name)


def test_a_wide_token_costs_no_other_its_bits():
    """Rows next to one 10^4 times their size come out as they do without it."""
    op = TokenLinear(64, 48, 96, x_dtype=F16, training=False)
    x, w = values(64, 96, F16, 40), values(48, 96, F32, 41)
    op.convert_w(w)
    alone = op.forward(x).clone()
    x[5], x[6, 3] = 60000.0, float("nan")
    y = op.forward(x)
    keep = [i for i in range(64) if i not in (5, 6)]
    assert torch.equal(y[keep], alone[keep]) and torch.isnan(y[6]).all() and not torch.isnan(y[keep]).any()


def test_serving_equals_training():
    x, w = values(50, 200, BF16, 42), values(70, 200, BF16, 43)
    a, b = TokenLinear(50, 70, 200, x_dtype=BF16), TokenLinear(50, 70, 200, x_dtype=BF16, training=False)
    b.convert_w(w)
    assert torch.equal(a.forward(x, w=w), b.forward(x))
    assert torch.equal(a.forward(x[:7]), b.forward(x[:7])) and a.forward(x[:7]).shape == (7, 70)


@pytest.mark.parametrize("rows", [1, 2, 3, 4, 5, 8, 9, 16, 17, 64])
@pytest.mark.parametrize("N, K", [(16, 64), (1, 1), (33, 130), (1000, 4096), (130, 4100), (48, 8200), (40, 33000)])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_serving_in_one_call(rows, N, K, dtype):
    """The same outputs as of the two calls, bit for bit, for few rows (one launch) and more; a row that is not finite stays alone."""
    say("token linear, one call", rows, N, K, dtype)
    x, w = values(rows, K, dtype, 46, pad=3), values(N, K, F32, 47).contiguous()
    x[0, K // 2] = float("inf")
    bias = torch.randn(N, device="cuda")
    wq, sw = quantize(w, Q.ROUND_NEAREST)
    xq, sx = quantize(x, Q.ROUND_NEAREST)
    ws = torch.empty(Q.qsync_token_linear_workspace_bytes(rows, N, K, 1) + 16, dtype=torch.uint8, device="cuda").random_()
    a, b = torch.full((rows, N), 7.0, dtype=dtype, device="cuda"), torch.full((rows, N), 7.0, dtype=dtype, device="cuda")
    Q.qsync_token_linear_fwd(rows, N, K, 1, None, xq, sx, wq, sw, bias, a, ws)
    Q.qsync_token_linear(x, rows, K, x.stride(0), None, 1, rows, N, 1, None, wq, sw, bias, b, torch.empty_like(sx), torch.empty_like(xq), ws)
    torch.cuda.synchronize()
    assert torch.isnan(a[0]).all() and not torch.isnan(a[1:]).any()
    assert torch.equal(a[1:], b[1:]) and torch.isnan(b[0]).all()
    want, bound = R.product(*R.codes(f64(x)[1:], 1), *R.codes(f64(w), 1), f64(bias))
    assert_within(b[1:], want, bound + rounded(want, dtype), "y") if rows > 1 else None


def test_an_empty_batch():
    op = TokenLinear(4, 24, 40)
    y = op.forward(torch.empty(0, 40, dtype=F16, device="cuda"), w=values(24, 40, F32, 44))
    dx, dw, db = op.backward(torch.empty(0, 24, dtype=F16, device="cuda"))
    assert y.shape == (0, 24) and dx.shape == (0, 40) and not dw.any() and not db.any()


def test_another_stream_and_two_operators_at_once():
    g = [(values(300, 264, F16, 50 + i), values(520, 264, F32, 60 + i), values(300, 520, F16, 70 + i)) for i in range(2)]
    want = []
    for x, w, dy in g:
        op = TokenLinear(300, 520, 264)
        want.append([t.clone() for t in (op.forward(x, w=w), *op.backward(dy))])
    ops, streams = [TokenLinear(300, 520, 264) for _ in g], [torch.cuda.Stream() for _ in g]
    torch.cuda.synchronize()
    for _ in range(3):
        for op in ops:
            op.offset = 0
        ys = [op.forward(x, w=w, stream=s) for op, s, (x, w, _) in zip(ops, streams, g)]
        grads = [op.backward(dy, stream=s) for op, s, (_, _, dy) in zip(ops, streams, g)]
        torch.cuda.synchronize()
        for y, grad, ref in zip(ys, grads, want):
            for a, b in zip((y, *grad), ref):
                assert torch.equal(a, b)


def test_graph_replays_equal_eager():
    """Two graphs, of a training step and of a few rows' forward pass, on one operator's buffers, replayed in turn over changing inputs."""
    n, N, K = 300, 264, 392
    x, w, dy = values(n, K, F16, 80), values(N, K, F32, 81), values(n, N, F16, 82)
    op, eager = TokenLinear(n, N, K), TokenLinear(n, N, K)

    def step(o):
        o.offset = 0
        return (o.forward(x, w=w), *o.backward(dy))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(op), op.forward(x[:5])
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    train, few = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(train, stream=side):
        out = step(op)
    with torch.cuda.graph(few, stream=side):
        short = op.forward(x[:5])
    for replay in range(4):
        say("token linear graph", replay)
        x.copy_(values(n, K, F16, 90 + replay))
        w.copy_(values(N, K, F32, 95 + replay))
        want = [t.clone() for t in step(eager)]
        torch.cuda.synchronize()
        train.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, want):
            assert torch.equal(a, b), replay
        few.replay()
        torch.cuda.synchronize()
        assert torch.equal(short, want[0][:5])


def test_offsets_that_pass_32_bits():
    """More than 2^31 elements in the activation, its codes and the output: the last rows, and a few between."""
    rows, K, N = 1_100_000, 2050, 2000
    say("token linear, large")
    x = torch.empty(rows, K, dtype=F16, device="cuda")
    x.copy_(torch.arange(K, device="cuda") % 251 - 125)
    x *= ((torch.arange(rows, device="cuda") % 7) + 1).to(F16)[:, None]
    x[-1, 5], x[-2, 2049] = 2000.0, -3000.0
    w = values(N, K, F32, 45)
    op = TokenLinear(rows, N, K, training=False, bias=False)
    op.convert_w(w)
    y = op.forward(x)
    at = torch.tensor([0, 1, 524287, 1047552, 1047553, 1048576, rows - 2, rows - 1], device="cuda")
    xq, sx = R.codes(f64(x[at]), 1)
    want, bound = R.product(xq, sx, *R.codes(f64(w), 1))
    assert_within(y[at], want, bound + rounded(want, F16), "rows")


def test_fractions_that_32_bits_round():
    """Negative products above -1/2 whose distance to the floor below takes more than 24 bits, at the draws where that decides: the oracle's
    codes.  (A column of 127 is every row's largest, so that the products are the values themselves.)"""
    rows, cols = 64, 1032
    u = R.draws(rows, cols, SEED, OFFSET).astype(np.float64)
    x = np.full((rows, cols), 127.0, np.float32)
    x[:, 8:] = (-((65536 - u[:, 8:]) / 65536)).astype(np.float32)                       # the border itself, and one step of 2^-25 on either side
    x[1::3, 8:] = np.nextafter(x[1::3, 8:], np.float32(-2))
    x[2::3, 8:] = np.nextafter(x[2::3, 8:], np.float32(2))
    q, s, qT, sc, _ = quantize_both(torch.from_numpy(x).cuda(), 1, None, Q.ROUND_STOCHASTIC)
    down = np.floor(x)
    oracle = np.clip(down + (u < ((x - down).astype(np.float32) * np.float32(65536.0)).astype(np.uint32)), -127, 127)
    equal(q[:, :cols], oracle, "codes")
    check_rows(q, s, x, R.draws(rows, cols, SEED, OFFSET), "rows")


@pytest.mark.parametrize("N, K", [(1024, 8192), (520, 14336)])
def test_fewer_rows_than_an_operator_was_built_for(N, K):
    """What an operator of those rows returns, bit for bit, and no less room for it."""
    large = TokenLinear(8192, N, K, x_dtype=BF16, training=False)
    w = values(N, K, BF16, 149).contiguous()
    large.convert_w(w)
    for n in (1, 8, 64, 400, 1500):
        say("token linear, fewer rows", N, K, n)
        x = values(n, K, BF16, 150 + n)
        small = TokenLinear(n, N, K, x_dtype=BF16, training=False)
        small.convert_w(w)
        have, need = large.ws.numel(), small.ws.numel()
        assert have >= need
        a, b = small.forward(x), large.forward(x)
        assert torch.equal(a, b)
        some = [0, n // 2, n - 1]
        want, bound = R.product(*R.codes(f64(x)[some], 1), *R.codes(f64(w), 1))
        assert_within(b[some], want, bound + rounded(want, BF16), f"{n} rows")


def test_gradients_of_fewer_rows_than_an_operator_was_built_for():
    N, K = 3000, 520
    large, w = TokenLinear(20000, N, K, x_dtype=F16), values(3000, 520, F32, 151).contiguous()
    for n in (5, 200, 2100):
        say("token linear, fewer rows' gradients", n)
        x, dy = values(n, K, F16, 152 + n), values(n, N, F16, 153 + n)
        small, out = TokenLinear(n, N, K, x_dtype=F16), []
        have, need = large.ws_bwd.numel(), small.ws_bwd.numel()
        assert have >= need
        for op in (small, large):
            op.offset = 0
            out.append([t.clone() for t in (op.forward(x, w=w), *op.backward(dy))])
        for a, b in zip(*out):
            assert torch.equal(a, b)


SERVED = [(16, 64), (1, 1), (33, 130), (1000, 700), (4096, 640), (130, 1024), (50, 1500), (300, 2048), (1000, 4096), (48, 5400), (17, 8190), (130, 16384), (4097, 200)]


@pytest.mark.parametrize("rows", [1, 2, 3, 4, 5, 8, 9, 15, 16])
@pytest.mark.parametrize("N, K", SERVED)
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_every_row_of_a_serving_call(rows, N, K, dtype):
    """A handful of rows in one launch, one row among them, at every depth of its stages and at the ends of its rule (16384 codes, 4096 columns): each
    row against the formula, and the bits of the two calls; then with a last row that is not finite."""
    say("token linear, every row of one call", rows, N, K, dtype)
    x, w = values(rows, K, dtype, 146, pad=3), values(N, K, F32, 147).contiguous()
    bias = torch.randn(N, generator=torch.Generator(device="cuda").manual_seed(148), device="cuda")
    wq, sw = quantize(w, Q.ROUND_NEAREST)
    ws = torch.empty(Q.qsync_token_linear_workspace_bytes(rows, N, K, 1) + 16, dtype=torch.uint8, device="cuda").random_()
    wc = R.codes(f64(w), 1)
    for last in (None, float("nan")):
        if last is not None:
            x[rows - 1, K - 1] = last
        xq, sx = quantize(x, Q.ROUND_NEAREST)
        a, b = torch.full((rows, N), 7.0, dtype=dtype, device="cuda"), torch.full((rows, N), 7.0, dtype=dtype, device="cuda")
        Q.qsync_token_linear_fwd(rows, N, K, 1, None, xq, sx, wq, sw, bias, a, ws)
        Q.qsync_token_linear(x, rows, K, x.stride(0), None, 1, rows, N, 1, None, wq, sw, bias, b, torch.empty_like(sx), torch.empty_like(xq), ws)
        torch.cuda.synchronize()
        finite = rows if last is None else rows - 1
        assert torch.isnan(b[finite:]).all() and torch.isnan(a[finite:]).all()
        assert torch.equal(a[:finite], b[:finite])
        if finite:
            want, bound = R.product(*R.codes(f64(x)[:finite], 1), *wc, f64(bias))
            assert_within(b[:finite], want, bound + rounded(want, dtype), "y")


@pytest.mark.parametrize("M, N, K", [(300, 257, 9000), (130, 1030, 4200), (1000, 4098, 16384), (1024, 4096, 16384), (600, 520, 33000)])
@pytest.mark.parametrize("tile", [-1, 0, 1, 2])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_pieces_of_every_tile(M, N, K, tile, dtype):
    """Contractions in pieces on the tile of the rule (the 256 tile for 16384 deep) and on each of the others, outputs that are no whole tiles: forward and
    weight gradient, some rows against the formula, and all of them bit for bit as without pieces."""
    say("token product in pieces", M, N, K, tile, dtype)
    g = torch.Generator(device="cuda").manual_seed(116)
    a, b = random_codes(M, K, g), random_codes(N, K, g)
    sa, sb, bias = (torch.rand(M, generator=g, device="cuda") * 1e-3, torch.rand(N, generator=g, device="cuda") * 1e-2, torch.randn(N, generator=g, device="cuda"))
    out = []
    try:
        Q.qsync_debug_set_gemm_tile(tile)
        forward, wgrad = Q.qsync_token_linear_workspace_bytes(M, N, K, 1), Q.qsync_token_wgrad_workspace_bytes(K, M, N, 1)
        for pieces in (False, True):
            ws = torch.empty(max(forward, wgrad), dtype=torch.uint8, device="cuda").random_() if pieces else None
            y, dw = torch.full((M, N), 7.0, dtype=dtype, device="cuda"), torch.full((M, N), 7.0, dtype=dtype, device="cuda")
            Q.qsync_token_linear_fwd(M, N, K, 1, None, a, sa, b, sb, bias, y, ws)
            Q.qsync_token_linear_wgrad(K, M, N, 1, None, a, sa, b, sb, dw, ws)
            torch.cuda.synchronize()
            out.append((y, dw))
    finally:
        Q.qsync_debug_set_gemm_tile(-1)
    assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1])
    some = sorted({0, 1, 63, 64, 127, 128, M // 2, min(255, M - 1), min(256, M - 1), M - 2, M - 1})
    codes, scales, b64, sb64 = f64(a[some]), sa.cpu().numpy()[some], f64(b), sb.cpu().numpy()
    want, bound = R.product(codes, scales, b64, sb64, f64(bias))
    assert_within(out[1][0][some], want, bound + rounded(want, dtype), "y")
    want, bound = R.product(codes, scales, b64, sb64)
    assert_within(out[1][1][some], want, bound + rounded(want, dtype), "dw")


@pytest.mark.parametrize("rows, N, K, sets", [(700, 700, 600, 5), (2500, 1100, 1500, 4), (1500, 900, 1030, 23), (3000, 2100, 2000, 6), (3000, 1030, 1028, 24), (400, 2100, 2000, 8)])
@pytest.mark.parametrize("tile", [-1, 0, 1, 2])
def test_weight_gradients_of_few_large_sets(rows, N, K, sets, tile):
    """Sets of different and of no rows whose tiles are dealt out by eighths, and those next to them that are not; on each tile."""
    say("token weight gradient, sets of many tiles", rows, N, K, sets, tile)
    g = torch.Generator().manual_seed(160)
    cuts = sorted((torch.rand(sets - 1, generator=g) ** 2 * (rows - 9)).long().tolist())
    cuts[1 if sets > 4 else 0] = cuts[0]                       # (a set without rows)
    bounds = [0, *sorted(cuts), rows - 9]
    q = {c: torch.randint(-127, 128, (rows - 9, c), generator=g).numpy() for c in (N, K)}
    sides = []
    for cols in (N, K):
        flat = np.full(Q.qsync_token_code_rows(rows, sets, True) * cols, 99, np.int8)
        for start, m in R.transposed_layout(q[cols], bounds, True).values():
            flat[start:start + m.size] = m.reshape(-1)
        sides.append((torch.from_numpy(flat).cuda(), torch.rand(sets, cols, generator=g).cuda() * 1e-2))
    dw = torch.full((sets, N, K), 7.0, device="cuda")
    try:
        Q.qsync_debug_set_gemm_tile(tile)
        Q.qsync_token_linear_wgrad(rows, N, K, sets, torch.tensor(bounds, dtype=torch.int32, device="cuda"), *sides[0], *sides[1], dw, None)
        torch.cuda.synchronize()
    finally:
        Q.qsync_debug_set_gemm_tile(-1)
    for e, (i, j) in enumerate(zip(bounds[:-1], bounds[1:])):
        want, bound = R.product(q[N][i:j].T, sides[0][1][e].cpu().numpy(), q[K][i:j].T, sides[1][1][e].cpu().numpy())
        assert_within(dw[e], want, bound + rounded(want, F32), f"set {e}")


def test_tiles_of_many_wide_sets():
    """Gradients of 512 sets without rows, 2^20 columns wide: 2^23 tiles of 64 x 64, all of them zeros."""
    sets, K = 512, 1 << 20
    say("token weight gradient, 2^23 tiles")
    offsets, dw = torch.zeros(sets + 1, dtype=torch.int32, device="cuda"), torch.full((sets, 1, K), 7.0, dtype=BF16, device="cuda")
    some = torch.zeros(256, dtype=torch.int8, device="cuda")      # (no row's code or scale is read)
    Q.qsync_token_linear_wgrad(0, 1, K, sets, offsets, some, offsets.view(F32), some, offsets.view(F32), dw, None)
    torch.cuda.synchronize()
    assert not dw.any()


def test_two_operands_beyond_a_grid():
    """Columns of 128 sets whose scales, of one operand as many as the interface allows, would be more workgroups for both than a launch counts."""
    sets, K = 128, 1 << 20
    say("token convert, two operands of 2^27 columns")
    g = torch.Generator(device="cuda").manual_seed(154)
    x, w = (torch.randn(sets, K, generator=g, device="cuda", dtype=F16) for _ in range(2))
    offsets = torch.arange(sets + 1, dtype=torch.int32, device="cuda")
    out = []
    for joined in (True, False):
        dst = []
        for routed in (True, False):
            dst += [torch.empty(sets, device="cuda"), torch.empty(sets, K, dtype=torch.int8, device="cuda"), torch.empty(sets, K, device="cuda"),
                    torch.empty(Q.qsync_token_code_rows(sets, sets, routed) * K, dtype=torch.int8, device="cuda")]
        ws = [torch.empty(Q.qsync_token_quantize_both_workspace_bytes(sets, K, sets, routed), dtype=torch.uint8, device="cuda") for routed in (True, False)]
        if joined:
            Q.qsync_token_convert(x, sets, K, K, None, 1, sets, sets, offsets, *dst[:4], w, 1, *dst[4:], *ws)
        else:
            Q.qsync_token_quantize_both(x, sets, K, K, None, 1, sets, sets, offsets, Q.ROUND_NEAREST, 0, 0, *dst[:4], None, ws[0])
            Q.qsync_token_quantize_both(w, sets, K, K, None, 1, sets, sets, None, Q.ROUND_NEAREST, 0, 0, *dst[4:], None, ws[1])
        torch.cuda.synchronize()
        out.append(dst)
    for i, (a, b) in enumerate(zip(*out)):
        if i == 3:      # (a set has one row; the stretch behind each set's belongs to none)
            for e in range(sets):
                start = (R.pad(e) + 128 * e) * K
                assert torch.equal(a[start:start + 128 * K], b[start:start + 128 * K]), e
        else:
            assert torch.equal(a, b), i
    for t, scale in ((x, out[0][2]), (w, out[0][6])):      # (64-bit quotients of 11-bit values by 127 are near no border of 32 bits)
        assert torch.equal(scale, torch.where(t == 0, 1.0, t.double().abs() / 127).float())
    del out, dst, ws
    torch.cuda.empty_cache()
