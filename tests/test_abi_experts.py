"""Host-side checks of the operators with a scale for each token and of the experts': what the C ABI, the binding and the classes refuse, and
what is a no-op (CPU only)."""
import ctypes

import pytest
import torch

from paper_2407_02327_amd import qsync as Q
from paper_2407_02327_amd.experts import ExpertLinear, ExpertRoute, TokenLinear

lib = Q.lib
pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="argument validation on made-up device addresses: CPU-only boxes")
_at = lambda n, off=0: ctypes.c_void_p((n << 34) + off)       # made-up device addresses far apart
OK_OR_NO_GPU = (Q.OK, Q.ERR_HIP)
BIG = 1 << 30
NULL = ctypes.c_void_p(None)


class Call:
    def __init__(self, fn, names, values):
        self.fn, self.names, self.values = fn, names.split(), values
        assert len(self.names) == len(values)

    def but(self, **other):
        assert set(other) <= set(self.names), other
        return self.fn(*[other.get(n, v) for n, v in zip(self.names, self.values)])


ROWS = Call(lib.qsync_token_quantize, "x xdt x_rows cols ld source group rows count rnd seed offset scale q stream",
            [_at(1), Q.BF16, 4, 100, 101, _at(2), 2, 8, _at(3), 1, 1, 2, _at(4), _at(5), None])
BOTH = Call(lib.qsync_token_quantize_both, "x xdt x_rows cols ld source group rows sets offsets rnd seed offset scale q col_scale qT sums ws ws_bytes stream",
            [_at(1), Q.F16, 4, 100, 101, _at(2), 2, 8, 3, _at(3), 0, 1, 2, _at(4), _at(5), _at(6), _at(7), _at(8), _at(9), BIG, None])
FWD = Call(lib.qsync_token_linear_fwd, "rows N K sets offsets a sa b sb bias y ydt ws ws_bytes stream",
           [40, 30, 20, 3, _at(1), _at(2), _at(3), _at(4), _at(5), _at(6), _at(7), Q.BF16, _at(8), BIG, None])
CONVERT = Call(lib.qsync_token_convert, "x xdt x_rows cols ld source group rows sets offsets scale q col_scale qT w wdt N sw wq swc wqT ws ws_bytes ws_w ws_w_bytes stream",
               [_at(1), Q.BF16, 4, 100, 101, _at(2), 2, 8, 3, _at(3), _at(4), _at(5), _at(6), _at(7), _at(8), Q.F32, 30, _at(9), _at(10), _at(11), _at(12), _at(13), BIG, _at(14), BIG, None])
SERVE = Call(lib.qsync_token_linear, "x xdt x_rows cols ld source group rows N sets offsets b sb bias y ydt scale q ws ws_bytes stream",
             [_at(1), Q.BF16, 4, 100, 101, _at(2), 2, 8, 30, 3, _at(3), _at(4), _at(5), _at(6), _at(7), Q.F16, _at(8), _at(9), _at(10), BIG, None])
WGRAD = Call(lib.qsync_token_linear_wgrad, "rows N K sets offsets a sa b sb y ydt ws ws_bytes stream",
             [40, 30, 20, 3, _at(1), _at(2), _at(3), _at(4), _at(5), _at(7), Q.F32, _at(8), BIG, None])
GRADS = Call(lib.qsync_token_linear_bwd, "rows N K sets offsets a sa b sb dyT sdc xT sxc dx dxdt dw dwdt ws ws_bytes stream",
             [40, 30, 20, 3, _at(1), _at(2), _at(3), _at(4), _at(5), _at(6), _at(7), _at(8), _at(9), _at(10), Q.F16, _at(11), Q.F32, _at(12), BIG, None])
SORT = Call(lib.qsync_expert_sort, "ids idt tokens group experts offsets source slot ws ws_bytes stream",
            [_at(1), Q.I64, 40, 2, 8, _at(2), _at(3), _at(4), _at(5), BIG, None])
GATHER = Call(lib.qsync_expert_gather, "x xdt x_rows cols ld source group rows count y stream", [_at(1), Q.F16, 4, 100, 100, _at(2), 2, 8, _at(3), _at(4), None])
COMBINE = Call(lib.qsync_expert_combine, "x xdt rows cols ld slot tokens group weight y ydt stream", [_at(1), Q.F16, 8, 100, 100, _at(2), 4, 2, _at(3), _at(4), Q.F32, None])
BWD = Call(lib.qsync_expert_combine_bwd, "x xdt tokens cols ld z zdt rows ldz slot group weight dz dzdt dweight stream",
           [_at(1), Q.F16, 4, 100, 100, _at(2), Q.F32, 8, 100, _at(3), 2, _at(4), _at(5), Q.BF16, _at(6), None])


@pytest.mark.parametrize("call, required", [(ROWS, "x scale q"), (BOTH, "x scale q col_scale qT"), (CONVERT, "x scale q col_scale qT w sw wq swc wqT"), (SERVE, "x b sb y scale q"), (FWD, "a sa b sb y"), (WGRAD, "a sa b sb y"), (GRADS, "a sa b sb dyT sdc xT sxc dx dw"), (SORT, "ids offsets source slot"),
                                            (GATHER, "x source count y"), (COMBINE, "x slot y"), (BWD, "x slot z")], ids="rows both convert serve fwd wgrad bwd sort gather combine combine_bwd".split())
def test_what_is_required(call, required):
    assert call.but() in OK_OR_NO_GPU
    for name in required.split():
        assert call.but(**{name: NULL}) == Q.ERR_NULL, name
    for name in set(call.names) & {"xdt", "ydt", "idt", "zdt", "dzdt", "wdt", "dxdt", "dwdt"}:
        for bad in (Q.I8, 6, -1) + ((Q.F32, Q.F16, Q.BF16) if name == "idt" else (Q.I32, Q.I64)):
            assert call.but(**{name: bad}) == Q.ERR_BAD_ENUM, (name, bad)


@pytest.mark.parametrize("call", [ROWS, BOTH, CONVERT, SERVE, GATHER, COMBINE, BWD], ids="rows both convert serve gather combine bwd".split())
def test_matrices(call):
    for shape in (dict(rows=-1), dict(cols=-1), dict(ld=99), dict(group=0), dict(rows=1 << 50, cols=1 << 50, ld=1 << 50)):
        assert call.but(**shape) == Q.ERR_BAD_SHAPE, shape
    assert call.but(cols=(1 << 20) + 1, ld=1 << 21, **({"ldz": 1 << 21} if call is BWD else {})) == Q.ERR_UNSUPPORTED
    assert call.but(rows=(1 << 23) + 1) == Q.ERR_UNSUPPORTED
    assert call.but(x=_at(1, 1)) == Q.ERR_ALIGN
    assert call.but(x=_at(1, 2)) in OK_OR_NO_GPU                  # any element is a start
    if call is not BWD:
        assert call.but(cols=0) in OK_OR_NO_GPU
    for name in set(call.names) & {"source", "slot", "count", "weight", "dweight", "scale", "col_scale", "sums", "offsets"}:
        value = dict(zip(call.names, call.values))[name]
        assert call.but(**{name: ctypes.c_void_p(value.value + 2)}) == Q.ERR_ALIGN, name


@pytest.mark.parametrize("call, out, inputs", [(ROWS, "q", "x"), (BOTH, "q", "x"), (BOTH, "qT", "x"), (CONVERT, "q", "x"), (CONVERT, "q", "w"), (CONVERT, "wqT", "x"), (CONVERT, "wq", "w"), (CONVERT, "ws_w", "ws"),
                                               (SERVE, "q", "x"), (SERVE, "scale", "x"), (SERVE, "y", "x"), (SERVE, "y", "q"), (GATHER, "y", "x"), (COMBINE, "y", "x"), (BWD, "dz", "x"), (BWD, "dz", "z")])
def test_outputs_do_not_overlap_inputs(call, out, inputs):
    source = dict(zip(call.names, call.values))[inputs]
    assert call.but(**{out: source}) == Q.ERR_UNSUPPORTED
    assert call.but(**{out: ctypes.c_void_p(source.value + 160)}) == Q.ERR_UNSUPPORTED


def test_quantizers():
    for call in (ROWS, BOTH):
        assert call.but(rnd=Q.ROUND_FLOOR) == Q.ERR_UNSUPPORTED and call.but(rnd=3) == Q.ERR_BAD_ENUM
        assert call.but(source=NULL) == Q.ERR_BAD_SHAPE and call.but(source=NULL, x_rows=8) in OK_OR_NO_GPU      # rows that are x's own
        assert call.but(q=_at(5, 8)) == Q.ERR_ALIGN
    assert ROWS.but(rows=0) == Q.OK and ROWS.but(count=NULL) in OK_OR_NO_GPU
    assert BOTH.but(qT=_at(7, 8)) == Q.ERR_ALIGN and BOTH.but(sums=NULL) in OK_OR_NO_GPU
    assert BOTH.but(sets=0) == Q.ERR_UNSUPPORTED and BOTH.but(sets=513) == Q.ERR_UNSUPPORTED and BOTH.but(sets=-1) == Q.ERR_BAD_SHAPE
    assert BOTH.but(offsets=NULL) == Q.ERR_BAD_SHAPE and BOTH.but(offsets=NULL, sets=4) in OK_OR_NO_GPU          # equal shares
    need = Q.qsync_token_quantize_both_workspace_bytes(8, 100, 3, True)
    assert need > 0 and BOTH.but(ws_bytes=need - 1) == Q.ERR_WORKSPACE and BOTH.but(ws=NULL) == Q.ERR_WORKSPACE and BOTH.but(ws=_at(9, 8)) == Q.ERR_ALIGN
    assert BOTH.but(rows=0, sums=NULL) == Q.OK
    huge = dict(x_rows=1 << 23, rows=1 << 23, ws_bytes=1 << 62)                    # (more than a grid's threads count)
    assert BOTH.but(cols=1 << 14, ld=1 << 14, **huge) == Q.ERR_UNSUPPORTED and BOTH.but(cols=1 << 19, ld=1 << 19, sets=512) == Q.ERR_UNSUPPORTED


def test_convert():
    need_x, need_w = Q.qsync_token_quantize_both_workspace_bytes(8, 100, 3, True), Q.qsync_token_quantize_both_workspace_bytes(90, 100, 3, False)
    assert CONVERT.but(ws_bytes=need_x - 1) == Q.ERR_WORKSPACE and CONVERT.but(ws_w_bytes=need_w - 1) == Q.ERR_WORKSPACE
    assert CONVERT.but(ws_bytes=need_x, ws_w_bytes=need_w) in OK_OR_NO_GPU and CONVERT.but(ws_w=_at(14, 8)) == Q.ERR_ALIGN
    assert CONVERT.but(N=-1) == Q.ERR_BAD_SHAPE and CONVERT.but(sets=0) == Q.ERR_UNSUPPORTED and CONVERT.but(N=1 << 23) == Q.ERR_UNSUPPORTED
    assert CONVERT.but(wqT=_at(12, 8)) == Q.ERR_ALIGN and CONVERT.but(w=_at(8, 2)) == Q.ERR_ALIGN
    assert CONVERT.but(rows=0) in OK_OR_NO_GPU and CONVERT.but(N=0) in OK_OR_NO_GPU and CONVERT.but(rows=0, N=0) == Q.OK


def test_serving():
    assert SERVE.but(source=NULL) == Q.ERR_BAD_SHAPE and SERVE.but(source=NULL, x_rows=8) in OK_OR_NO_GPU
    assert SERVE.but(offsets=NULL) == Q.ERR_UNSUPPORTED and SERVE.but(offsets=NULL, sets=1) in OK_OR_NO_GPU
    assert SERVE.but(q=_at(9, 8)) == Q.ERR_ALIGN and SERVE.but(b=_at(4, 8)) == Q.ERR_ALIGN
    assert SERVE.but(rows=0) == Q.OK and SERVE.but(N=0) == Q.OK and SERVE.but(N=-1) == Q.ERR_BAD_SHAPE


def test_sizes_of_codes():
    assert [Q.qsync_token_code_cols(n) for n in (0, 1, 128, 129, -1, 1 << 21)] == [0, 128, 128, 256, 0, 0]
    assert Q.qsync_token_code_rows(300, 1, False) == 384 and Q.qsync_token_code_rows(300, 3, False) == 384
    assert Q.qsync_token_code_rows(300, 3, True) == 384 + 3 * 128 and Q.qsync_token_code_rows(300, 7, False) == 0
    assert Q.qsync_token_code_rows(300, 0, True) == 0 and Q.qsync_token_code_rows(-1, 1, True) == 0
    # whatever the offsets: the sets' stretches follow one another and end in the buffer
    import random
    rng = random.Random(1)
    pad = lambda n: (n + 127) // 128 * 128
    for _ in range(2000):
        rows, sets = rng.randint(0, 1500), rng.randint(1, 9)
        offsets = [0] + sorted(rng.randint(0, rows) for _ in range(sets))
        end = 0
        for e in range(sets):
            start = pad(offsets[e]) + 128 * e
            assert start >= end
            end = start + pad(offsets[e + 1] - offsets[e])
        assert end <= Q.qsync_token_code_rows(rows, sets, True)


@pytest.mark.parametrize("call", [FWD, WGRAD], ids=["fwd", "wgrad"])
def test_products(call):
    for name in ("rows", "N", "K"):
        assert call.but(**{name: -1}) == Q.ERR_BAD_SHAPE
        assert call.but(**{name: 1 << 24}) == Q.ERR_UNSUPPORTED
    assert call.but(sets=0) == Q.ERR_UNSUPPORTED and call.but(sets=513) == Q.ERR_UNSUPPORTED
    assert call.but(offsets=NULL) == Q.ERR_UNSUPPORTED and call.but(offsets=NULL, sets=1) in OK_OR_NO_GPU
    for name, off in (("a", 8), ("b", 8), ("sa", 2), ("sb", 2), ("y", 1), ("offsets", 2)):
        value = dict(zip(call.names, call.values))[name]
        assert call.but(**{name: ctypes.c_void_p(value.value + off)}) == Q.ERR_ALIGN, name
    assert call.but(N=0) == Q.OK
    if call is FWD:
        assert call.but(rows=0) == Q.OK and call.but(bias=_at(6, 2)) == Q.ERR_ALIGN and call.but(bias=NULL) in OK_OR_NO_GPU
        assert call.but(y=_at(2)) == Q.ERR_UNSUPPORTED
    else:
        assert call.but(K=0) == Q.OK
    # the products run with any room, and without
    assert call.but(ws=NULL, ws_bytes=0) in OK_OR_NO_GPU and call.but(ws_bytes=0) in OK_OR_NO_GPU and call.but(ws=_at(8, 8)) == Q.ERR_ALIGN
    assert Q.qsync_token_linear_workspace_bytes(200, 128, 16384, 1) > 0 and Q.qsync_token_wgrad_workspace_bytes(16384, 128, 200, 1) > 0


def test_both_gradients():
    for name in ("rows", "N", "K"):
        assert GRADS.but(**{name: -1}) == Q.ERR_BAD_SHAPE and GRADS.but(**{name: 1 << 24}) == Q.ERR_UNSUPPORTED
        assert GRADS.but(**{name: 0}) in OK_OR_NO_GPU
    assert GRADS.but(rows=0, N=0) == Q.OK and GRADS.but(sets=513) == Q.ERR_UNSUPPORTED and GRADS.but(offsets=NULL) == Q.ERR_UNSUPPORTED
    for name in ("a", "b", "dyT", "xT"):
        value = dict(zip(GRADS.names, GRADS.values))[name]
        assert GRADS.but(**{name: ctypes.c_void_p(value.value + 8)}) == Q.ERR_ALIGN, name
        assert GRADS.but(dx=value) == Q.ERR_UNSUPPORTED and GRADS.but(dw=value) == Q.ERR_UNSUPPORTED, name
    assert GRADS.but(dx=_at(11)) == Q.ERR_UNSUPPORTED and GRADS.but(ws=NULL, ws_bytes=0) in OK_OR_NO_GPU and GRADS.but(ws=_at(12, 8)) == Q.ERR_ALIGN


def test_sort():
    assert SORT.but(tokens=-1) == Q.ERR_BAD_SHAPE and SORT.but(group=0) == Q.ERR_BAD_SHAPE and SORT.but(experts=-1) == Q.ERR_BAD_SHAPE
    assert SORT.but(experts=0) == Q.ERR_UNSUPPORTED and SORT.but(experts=513) == Q.ERR_UNSUPPORTED and SORT.but(tokens=1 << 23) == Q.ERR_UNSUPPORTED
    assert SORT.but(ids=_at(1, 4)) == Q.ERR_ALIGN and SORT.but(ids=_at(1, 4), idt=Q.I32) in OK_OR_NO_GPU
    need = Q.qsync_expert_sort_workspace_bytes(80, 8)
    if need:
        assert SORT.but(ws_bytes=need - 1) == Q.ERR_WORKSPACE and SORT.but(ws=NULL) == Q.ERR_WORKSPACE


def test_workspaces_for_more_are_enough_for_fewer():
    sizes = [1, 2, 100, 1000, 2048, 2049, 5000, 100_000, 262_144, 262_145, 300_000, 524_289, 4_000_000, 1 << 23]
    for fewer, more in zip(sizes, sizes[1:]):
        assert Q.qsync_expert_sort_workspace_bytes(fewer, 64) <= Q.qsync_expert_sort_workspace_bytes(more, 64)
        for cols, sets, given in ((100, 1, False), (1000, 7, True)):
            assert Q.qsync_token_quantize_both_workspace_bytes(fewer, cols, sets, given) <= Q.qsync_token_quantize_both_workspace_bytes(more, cols, sets, given)


def test_combine_backward():
    assert BWD.but(dz=NULL, dweight=NULL) == Q.ERR_NULL
    assert BWD.but(dweight=NULL, z=NULL) in OK_OR_NO_GPU and BWD.but(dz=NULL) in OK_OR_NO_GPU
    assert BWD.but(ldz=99) == Q.ERR_BAD_SHAPE and BWD.but(tokens=0) == Q.OK


def test_classes_refuse_sizes_and_types():
    for bad in (dict(tokens=-1), dict(k=0), dict(experts=0), dict(experts=513), dict(cols=0), dict(dtype=torch.int8), dict(tokens=1 << 23, k=2)):
        with pytest.raises(ValueError):
            ExpertRoute(**{**dict(tokens=4, k=2, experts=3, cols=8, device="cpu"), **bad})
    for bad in (dict(rows=-1), dict(N=0), dict(K=0), dict(rows=(1 << 23) + 1), dict(K=(1 << 20) + 1), dict(x_dtype=torch.int8), dict(dw_dtype=torch.float64),
                dict(dy_round=Q.ROUND_FLOOR)):
        with pytest.raises(ValueError):
            TokenLinear(**{**dict(rows=4, N=8, K=8, device="cpu"), **bad})
    for bad in (dict(experts=0), dict(experts=513), dict(experts=512, N=1 << 15)):
        with pytest.raises(ValueError):
            ExpertLinear(**{**dict(rows=4, N=8, K=8, experts=2, device="cpu"), **bad})


def test_classes_refuse_calls():
    """Buffers on no GPU, and passes out of their order."""
    route, linear, experts = ExpertRoute(4, 2, 3, 8, device="cpu"), TokenLinear(4, 8, 8, device="cpu"), ExpertLinear(8, 8, 8, 3, device="cpu")
    x = torch.zeros(4, 8, dtype=torch.float16)
    with pytest.raises(ValueError, match="GPU"):
        route.sort(torch.zeros(4, 2, dtype=torch.int64))
    with pytest.raises(ValueError, match="ids"):
        route.sort(torch.zeros(5, 2, dtype=torch.int64))
    with pytest.raises(ValueError, match="ids"):
        route.sort(torch.zeros(4, dtype=torch.int64))
    for call in (lambda: route.gather(x), lambda: route.combine(x), lambda: route.combine_backward(x), lambda: experts.forward(x, route), lambda: route.rows):
        with pytest.raises(RuntimeError, match="sort"):
            call()
    with pytest.raises(ValueError, match="GPU"):
        linear.forward(x)
    with pytest.raises(ValueError, match="w:"):
        linear.convert_w(torch.zeros(8, 9))
    with pytest.raises(ValueError, match="GPU"):
        linear.convert_w(torch.zeros(8, 8))
    with pytest.raises(RuntimeError, match="forward"):
        linear.backward(x)
    with pytest.raises(RuntimeError, match="forward"):
        experts.backward(x)
    with pytest.raises(RuntimeError, match="forward"):
        TokenLinear(4, 8, 8, training=False, device="cpu").backward(x)


@pytest.mark.parametrize("N, K", [(1024, 8192), (4096, 14336), (14336, 4096), (128, 4096), (1, 200_000), (64, 2048), (1000, 3000), (2048, 16384), (300, 60_000)])
def test_room_for_many_rows_is_enough_for_fewer(N, K):
    """The products' K splits, too: an operator built for a prompt is called with a few rows."""
    sizes = [*range(1, 70), 100, 127, 128, 129, 200, 255, 400, 511, 512, 513, 700, 1000, 1024, 1100, 1500, 1600, 2000, 2047, 2048, 2049, 3000, 4095, 4096, 8192, 16384,
             20_000, 40_000, 100_000, 1 << 18]
    queries = [Q.qsync_token_wgrad_workspace_bytes, Q.qsync_token_linear_bwd_workspace_bytes] + ([Q.qsync_token_linear_workspace_bytes] if K <= 1 << 20 else [])
    for query in queries:
        need = [query(rows, N, K, 1) for rows in sizes]
        assert need == sorted(need), query.__name__
        assert need[-1] <= 64 << 20      # (what fills the units: one 256 x 256 sum each)


def test_room_of_a_large_operator():
    """Sizes whose calls of a few rows are planned in pieces, at the least two."""
    assert Q.qsync_token_linear_workspace_bytes(8192, 4096, 14336, 1) >= Q.qsync_token_linear_workspace_bytes(64, 4096, 14336, 1) >= 2 * 64 * 4096 * 4
    assert Q.qsync_token_linear_workspace_bytes(16384, 1024, 8192, 1) >= Q.qsync_token_linear_workspace_bytes(1600, 1024, 8192, 1) >= 2 * 1600 * 1024 * 4
    assert Q.qsync_token_linear_bwd_workspace_bytes(4096, 14336, 4096, 1) >= Q.qsync_token_linear_bwd_workspace_bytes(200, 14336, 4096, 1) >= 2 * 200 * 4096 * 4


def test_room_follows_a_pinned_tile():
    """1024 x 4096, 16384 deep: four pieces on the 256 tile, the rule's choice; the 128 tile fills the units with two."""
    piece = 1024 * 4096 * 4
    rooms = {}
    try:
        for tile in (-1, 0, 1):
            Q.qsync_debug_set_gemm_tile(tile)
            rooms[tile] = Q.qsync_token_wgrad_workspace_bytes(16384, 1024, 4096, 1), Q.qsync_token_linear_workspace_bytes(1024, 4096, 16384, 1)
    finally:
        Q.qsync_debug_set_gemm_tile(-1)
    assert all(r == 4 * piece for r in rooms[-1] + rooms[0]) and all(r <= 2 * piece for r in rooms[1])


def test_products_of_more_tiles_than_a_grid_counts():
    """Refused as such, before anything is launched; what fits on larger tiles is not."""
    wide = dict(rows=1 << 23, N=1 << 20)                                           # 2^27 tiles of 256 x 256
    assert FWD.but(**wide) == Q.ERR_UNSUPPORTED and FWD.but(offsets=NULL, sets=1, **wide) == Q.ERR_UNSUPPORTED
    assert FWD.but(rows=1 << 20, N=1 << 16) in OK_OR_NO_GPU                        # 2^20
    assert SERVE.but(x_rows=1 << 22, **wide) == Q.ERR_UNSUPPORTED
    assert WGRAD.but(sets=512, N=1, K=1 << 20) in OK_OR_NO_GPU and WGRAD.but(sets=512, N=70, K=1 << 20) in OK_OR_NO_GPU      # 2^21
    assert WGRAD.but(sets=512, N=1280, K=1 << 20) == Q.ERR_UNSUPPORTED             # 2^21 x 5
    assert GRADS.but(sets=512, N=1280, K=1 << 20, dw=_at(4000)) == Q.ERR_UNSUPPORTED
    assert GRADS.but(rows=1 << 23, N=1, K=1 << 20, dx=_at(40), dw=_at(4000)) == Q.ERR_UNSUPPORTED      # (the data gradient's)


def test_experts_keep_no_room_for_pieces():
    """One expert's rows lie where the route says, too, and such contractions are not split."""
    one, linear = (c(8192, 64, 4096, *extra, device="cpu") for c, extra in ((ExpertLinear, (1,)), (TokenLinear, ())))
    assert one.ws.numel() <= 256 and one.ws_bwd.numel() <= 256 < min(linear.ws.numel(), linear.ws_bwd.numel())
