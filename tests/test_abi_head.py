"""Host-side checks of layer norm, token log-probabilities and distillation: what the C ABI, the binding and the classes refuse, and
what is a no-op (CPU only)."""
import ctypes

import pytest
import torch

from paper_2407_02327_amd import qsync as Q
from paper_2407_02327_amd.head import Distillation, LayerNorm, TokenLogProbs

lib = Q.lib
pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="argument validation on made-up device addresses: CPU-only boxes")
_at = lambda n, off=0: ctypes.c_void_p((n << 30) + off)       # made-up device addresses a gigabyte apart
OK_OR_NO_GPU = (Q.OK, Q.ERR_HIP)
BIG = 1 << 28


class Call:
    """A well-formed argument list by name; `but` replaces some of it."""

    def __init__(self, fn, names, values):
        self.fn, self.names, self.values = fn, names.split(), values
        assert len(self.names) == len(values)

    def but(self, **other):
        assert set(other) <= set(self.names), other
        return self.fn(*[other.get(n, v) for n, v in zip(self.names, self.values)])


FWD = Call(lib.qsync_layernorm_fwd, "x xdt rows cols ld gamma beta eps y ydt mean rstd amax stream",
           [_at(1), Q.F16, 4, 100, 100, _at(2), _at(3), 1e-5, _at(4), Q.BF16, _at(5), _at(6), _at(7), None])
BWD = Call(lib.qsync_layernorm_bwd, "dy dydt lddy x xdt rows cols ldx gamma mean rstd dx dxdt dgamma dbeta ws ws_bytes stream",
           [_at(1), Q.F16, 100, _at(2), Q.F32, 4, 100, 100, _at(3), _at(4), _at(5), _at(6), Q.BF16, _at(7), _at(8), _at(9), BIG, None])
LOGP = Call(lib.qsync_token_logprobs, "z ldt rows cols ld scale tokens tdt logp entropy stats top_k top_logp top_index ws ws_bytes stream",
            [_at(1), Q.F16, 4, 100, 100, 1.0, _at(2), Q.I64, _at(3), _at(4), _at(5), 8, _at(6), _at(7), _at(8), BIG, None])
GRAD = Call(lib.qsync_token_logprobs_bwd, "z ldt rows cols ld scale tokens tdt stats entropy dlogp dentropy dz ddt stream",
            [_at(1), Q.F16, 4, 100, 100, 1.0, _at(2), Q.I32, _at(3), _at(4), _at(5), _at(6), _at(7), Q.F32, None])
DISTILL = Call(lib.qsync_distill_topk, "z ldt rows cols ld scale teacher teacher_dt index idt k weight loss dz ddt ws ws_bytes stream",
               [_at(1), Q.BF16, 4, 100, 100, 0.5, _at(2), Q.F32, _at(3), Q.I32, 16, _at(4), _at(5), _at(6), Q.F16, _at(7), BIG, None])
NULL = ctypes.c_void_p(None)


@pytest.mark.parametrize("call", [FWD, BWD, LOGP, GRAD, DISTILL], ids=["fwd", "bwd", "logprobs", "logprobs_bwd", "distill"])
def test_what_all_calls_share(call):
    assert call.but() in OK_OR_NO_GPU
    src, dt, ld = ("x", "xdt", "ldx" if call is BWD else "ld") if call in (FWD, BWD) else ("z", "ldt", "ld")
    assert call.but(**{src: NULL}) == Q.ERR_NULL
    for bad in (Q.I8, Q.I32, Q.I64, 6, -1):
        assert call.but(**{dt: bad}) == Q.ERR_BAD_ENUM
    for shape in (dict(rows=-1), dict(cols=-1), {ld: 99}, dict(rows=1 << 40, cols=1 << 40, **{ld: 1 << 40})):
        assert call.but(**shape) == Q.ERR_BAD_SHAPE
    assert call.but(**{src: _at(1, 1)}) == Q.ERR_ALIGN                                         # half an element
    assert call.but(**{src: _at(1, 4)}) in OK_OR_NO_GPU                                        # any element is a start
    assert call.but(cols=0) == Q.OK
    if call is not BWD:
        assert call.but(rows=0) == Q.OK
    if call not in (FWD, BWD):
        for scale in (0.0, -1.0, float("inf"), float("nan")):
            assert call.but(scale=scale) == Q.ERR_UNSUPPORTED
        assert call.but(rows=1, cols=(1 << 30) + 1, ld=(1 << 30) + 1, ws_bytes=1 << 62) == Q.ERR_UNSUPPORTED if "ws_bytes" in call.names \
            else call.but(rows=1, cols=(1 << 30) + 1, ld=(1 << 30) + 1) == Q.ERR_UNSUPPORTED


def test_layernorm_forward_refusals():
    assert FWD.but(gamma=NULL, beta=NULL, mean=NULL, rstd=NULL, amax=NULL) in OK_OR_NO_GPU
    assert FWD.but(y=NULL) == Q.ERR_NULL and FWD.but(ydt=Q.I8) == Q.ERR_BAD_ENUM
    for eps in (0.0, -1e-5, float("nan"), float("inf")):
        assert FWD.but(eps=eps) == Q.ERR_UNSUPPORTED
    for name in ("gamma", "beta", "mean", "rstd", "amax"):
        assert FWD.but(**{name: _at(2, 2)}) == Q.ERR_ALIGN
    assert FWD.but(y=_at(4, 1)) == Q.ERR_ALIGN
    assert FWD.but(y=_at(1), ydt=Q.F16) in OK_OR_NO_GPU                                        # in place
    assert FWD.but(y=_at(1), ydt=Q.BF16) == Q.ERR_UNSUPPORTED                                  # another type
    assert FWD.but(y=_at(1), ydt=Q.F16, ld=101) == Q.ERR_UNSUPPORTED                           # not packed
    assert FWD.but(y=_at(1), ydt=Q.F16, ld=101, rows=1) in OK_OR_NO_GPU
    assert FWD.but(y=_at(1, 2), ydt=Q.F16) == Q.ERR_UNSUPPORTED                                # displaced
    assert FWD.but(y=_at(1, 800), ydt=Q.F16) in OK_OR_NO_GPU                                   # behind it


def test_layernorm_backward_refusals():
    for name in ("dy", "mean", "rstd"):
        assert BWD.but(**{name: NULL}) == Q.ERR_NULL
    assert BWD.but(dx=NULL, dgamma=NULL, dbeta=NULL) == Q.ERR_NULL
    assert BWD.but(dydt=Q.I32) == Q.ERR_BAD_ENUM and BWD.but(dxdt=Q.I32) == Q.ERR_BAD_ENUM
    assert BWD.but(dx=NULL, dxdt=99) in OK_OR_NO_GPU                                           # (not looked at)
    assert BWD.but(lddy=99) == Q.ERR_BAD_SHAPE
    need = lib.qsync_layernorm_bwd_workspace_bytes(4, 100)
    assert need > 0 and lib.qsync_layernorm_bwd_workspace_bytes(-1, 100) == 0 and lib.qsync_layernorm_bwd_workspace_bytes(0, 100) == 0
    assert BWD.but(ws_bytes=need - 1) == Q.ERR_WORKSPACE and BWD.but(ws=NULL) == Q.ERR_WORKSPACE and BWD.but(ws=_at(9, 8)) == Q.ERR_ALIGN
    assert BWD.but(ws=NULL, ws_bytes=0, dgamma=NULL, dbeta=NULL) in OK_OR_NO_GPU
    assert BWD.but(rows=0, dgamma=NULL, dbeta=NULL) == Q.OK
    assert BWD.but(dx=_at(1), dxdt=Q.F16) in OK_OR_NO_GPU and BWD.but(dx=_at(2), dxdt=Q.F32) in OK_OR_NO_GPU
    for bad in (dict(dx=_at(1)), dict(dx=_at(2)), dict(dx=_at(1), dxdt=Q.F16, lddy=104), dict(dx=_at(2, 4), dxdt=Q.F32)):
        assert BWD.but(**bad) == Q.ERR_UNSUPPORTED


def test_logprobs_refusals():
    none = dict(logp=NULL, entropy=NULL, stats=NULL, top_k=0)
    assert LOGP.but(**none) == Q.ERR_NULL
    for keep in ("logp", "entropy", "stats"):
        assert LOGP.but(**{k: v for k, v in none.items() if k != keep}) in OK_OR_NO_GPU
    assert LOGP.but(tokens=NULL) == Q.ERR_NULL and LOGP.but(tokens=NULL, logp=NULL, tdt=77) in OK_OR_NO_GPU
    assert LOGP.but(tdt=Q.F32) == Q.ERR_BAD_ENUM
    assert LOGP.but(top_logp=NULL) == Q.ERR_NULL and LOGP.but(top_index=NULL) == Q.ERR_NULL
    assert LOGP.but(top_k=65) == Q.ERR_UNSUPPORTED and LOGP.but(top_k=-1) == Q.ERR_UNSUPPORTED
    assert LOGP.but(top_k=64) in OK_OR_NO_GPU and LOGP.but(cols=8) in OK_OR_NO_GPU and LOGP.but(cols=7) == Q.ERR_BAD_SHAPE
    for name, off in (("tokens", 4), ("logp", 2), ("entropy", 1), ("stats", 2), ("top_logp", 2), ("top_index", 2)):
        assert LOGP.but(**{name: _at(2, off)}) == Q.ERR_ALIGN
    need = lib.qsync_token_logprobs_workspace_bytes(Q.F16, 4, 100, 8)
    assert LOGP.but(ws_bytes=need - 1) == Q.ERR_WORKSPACE and LOGP.but(ws=NULL) == Q.ERR_WORKSPACE and LOGP.but(ws=_at(8, 8)) == Q.ERR_ALIGN


def test_a_workspace_serves_fewer_rows():
    for dt in (Q.F32, Q.F16, Q.BF16):
        for cols in (5, 3000, 200000):
            for top in (0, 5):
                sizes = [lib.qsync_token_logprobs_workspace_bytes(dt, rows, cols, top) for rows in (1, 2, 7, 100, 1023, 1024, 1025, 9000)]
                assert sizes == sorted(sizes) and sizes[0] > 0
                sizes = [lib.qsync_distill_topk_workspace_bytes(dt, rows, cols) for rows in (1, 2, 7, 100, 1023, 1024, 1025, 9000)]
                assert sizes == sorted(sizes) and sizes[0] > 0
    assert lib.qsync_token_logprobs_workspace_bytes(Q.I8, 4, 4, 0) == 0 and lib.qsync_token_logprobs_workspace_bytes(Q.F32, 4, 4, 65) == 0
    assert lib.qsync_distill_topk_workspace_bytes(Q.F32, -4, 4) == 0


def test_logprobs_gradient_refusals():
    for name in ("stats", "dz"):
        assert GRAD.but(**{name: NULL}) == Q.ERR_NULL
    assert GRAD.but(dlogp=NULL, dentropy=NULL) == Q.ERR_NULL and GRAD.but(tokens=NULL) == Q.ERR_NULL and GRAD.but(entropy=NULL) == Q.ERR_NULL
    assert GRAD.but(tokens=NULL, dlogp=NULL) in OK_OR_NO_GPU and GRAD.but(entropy=NULL, dentropy=NULL) in OK_OR_NO_GPU
    assert GRAD.but(ddt=Q.I32) == Q.ERR_BAD_ENUM and GRAD.but(tdt=Q.F16) == Q.ERR_BAD_ENUM
    assert GRAD.but(dz=_at(1), ddt=Q.F16) in OK_OR_NO_GPU
    for bad in (dict(dz=_at(1)), dict(dz=_at(1), ddt=Q.F16, ld=128), dict(dz=_at(1, 20), ddt=Q.F16)):
        assert GRAD.but(**bad) == Q.ERR_UNSUPPORTED


def test_distillation_refusals():
    for name in ("teacher", "index", "loss"):
        assert DISTILL.but(**{name: NULL}) == Q.ERR_NULL
    assert DISTILL.but(dz=NULL, ddt=55, weight=NULL) in OK_OR_NO_GPU
    assert DISTILL.but(teacher_dt=Q.I32) == Q.ERR_BAD_ENUM and DISTILL.but(idt=Q.F32) == Q.ERR_BAD_ENUM and DISTILL.but(ddt=Q.I8) == Q.ERR_BAD_ENUM
    assert DISTILL.but(k=0) == Q.ERR_BAD_SHAPE and DISTILL.but(k=257) == Q.ERR_UNSUPPORTED and DISTILL.but(k=256) in OK_OR_NO_GPU
    for name, off in (("teacher", 2), ("index", 2), ("weight", 2), ("loss", 1), ("dz", 1)):
        assert DISTILL.but(**{name: _at(2, off)}) == Q.ERR_ALIGN
    need = lib.qsync_distill_topk_workspace_bytes(Q.BF16, 4, 100)
    assert DISTILL.but(ws_bytes=need - 1) == Q.ERR_WORKSPACE and DISTILL.but(ws=NULL) == Q.ERR_WORKSPACE
    assert DISTILL.but(dz=_at(1), ddt=Q.BF16) in OK_OR_NO_GPU
    for bad in (dict(dz=_at(1)), dict(dz=_at(1), ddt=Q.BF16, ld=104), dict(dz=_at(1, 6), ddt=Q.BF16)):
        assert DISTILL.but(**bad) == Q.ERR_UNSUPPORTED


def test_other_calls_do_not_take_the_new_types():
    """bfloat16 and 64-bit integers are for the calls above: the others refuse them as they did."""
    x, s = torch.empty(8, dtype=torch.bfloat16), torch.empty(1)
    with pytest.raises(KeyError):
        Q.qsync_quantize(x, 1, 8, 8, Q.FP16, 0, 0, 0, 0, 0, None, s, None, 0)
    for dt in (Q.BF16, Q.I64):
        assert lib.qsync_quantize(_at(1), dt, 4, 8, 8, Q.FP16, 0, 0, 0, 0, 0, None, _at(2), None, None) == Q.ERR_BAD_ENUM
        assert lib.qsync_dequantize(_at(1), Q.I32, 4, 4, 4, None, None, 1.0, None, None, _at(2), dt, None) == Q.ERR_BAD_ENUM
    Q.qsync_layernorm_fwd(x, 0, 8, 8, None, None, 1e-5, x, None, None, None, 0)               # (no rows: nothing is launched)
    with pytest.raises(Q.QsyncError) as e:
        Q.qsync_token_logprobs(x, 1, 8, 8, 1.0, x, s, None, None, 0, None, None, None, 0)      # tokens of a floating type
    assert e.value.status == Q.ERR_BAD_ENUM


def test_classes_refuse_sizes_and_devices():
    for bad in (lambda: LayerNorm(-1, 4, device="cpu"), lambda: LayerNorm(4, 0, device="cpu"), lambda: LayerNorm(4, 4, x_dtype=torch.float64, device="cpu"),
                lambda: TokenLogProbs(4, 8, top_k=9, device="cpu"), lambda: TokenLogProbs(4, 100, top_k=65, device="cpu"),
                lambda: TokenLogProbs(4, 8, dlogits_dtype=torch.int32, device="cpu"), lambda: Distillation(4, 8, 0, device="cpu"),
                lambda: Distillation(4, 8, 257, device="cpu")):
        with pytest.raises(ValueError):
            bad()
    x = torch.zeros(4, 8, dtype=torch.float16)
    for op in (LayerNorm(4, 8, device="cpu"), TokenLogProbs(4, 8, device="cpu")):
        with pytest.raises(ValueError, match="GPU"):
            op.forward(x)
    with pytest.raises(RuntimeError):
        LayerNorm(4, 8, training=False, device="cpu").backward(x)


@pytest.mark.parametrize("cols", [64, 128, 700, 1024, 1025, 2048, 2443, 4096, 4097, 8192, 8193, 20000])
def test_layernorm_workspace_serves_fewer_rows(cols):
    """A workspace for some number of rows is enough for fewer: an operator's batches may be shorter than it was made for."""
    sizes = [Q.qsync_layernorm_bwd_workspace_bytes(rows, cols) for rows in range(1, 20000)]
    assert all(a <= b for a, b in zip(sizes, sizes[1:]))
