"""INT8 linear operators with a scale for each token, and the experts' layers that are made of them, as measurable cases.

Three operators, each through the package's public classes:

  linear    y = x w^T + b in 8-bit integers, a scale for each token of x and for each channel of w: `forward` alone on weights that
            were converted once (serving, evaluation), or a training step: weights converted, `forward`, `backward`
  route     tokens sorted by the experts that a router gave them, gathered, and the experts' rows combined with the router's weights:
            forward alone, or forward and both backward passes
  experts   the linear operator on routed tokens, a weight matrix for each expert: forward alone, or a training step

With `own` false the same results come from elementary torch operations in 32 bits, rounded once to the output's type.  Activations are
N(0, 1) with a few wide channels and tokens of different size, some of them zero (padding); gradients are small and differ from token to
token; the router prefers some experts.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

_TORCH = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
_ESZ = {"f16": 2, "bf16": 2, "f32": 4}
_SEED = 0x5EED0123456789AB      # of the gradients' stochastic rounding
_TINY = 2.0 ** -100             # a row below it counts as zero


def _linear(name, rows, n, k, dtype, train, bias=True):
    return {"name": name, "kind": "linear", "rows": rows, "n": n, "k": k, "dtype": dtype, "train": train, "bias": bias}


def _route(name, tokens, top, experts, cols, dtype, train):
    return {"name": name, "kind": "route", "tokens": tokens, "top": top, "experts": experts, "cols": cols, "dtype": dtype, "train": train}


def _experts(name, tokens, top, experts, n, k, dtype, train, gather=True):
    return {"name": name, "kind": "experts", "tokens": tokens, "top": top, "experts": experts, "n": n, "k": k, "dtype": dtype,
            "train": train, "gather": gather}


def listed():
    return [
        # the next token of one sequence through the narrow side of a feed-forward block: latency is all there is
        _linear("linear_one_token", 1, 1024, 4096, "f16", False),
        # the next tokens of a batch of sequences
        _linear("linear_some_tokens", 64, 4096, 4096, "bf16", False),
        # all tokens of a large batch through the wide side of a feed-forward block
        _linear("linear_forward", 16384, 4096, 1024, "bf16", False),
        # a training step on the narrow side
        _linear("linear_train", 16384, 1024, 4096, "f16", True),
        # a last, incomplete batch of sizes that fit no vector, full precision
        _linear("linear_train_odd", 2187, 1001, 777, "f32", True),
        # the next tokens of sixteen sequences to two of eight experts and back
        _route("route_some_tokens", 16, 2, 8, 4096, "bf16", False),
        # a training step's routing: many small experts, the largest
        _route("route_train", 8192, 8, 64, 1024, "bf16", True),
        # odd sizes, full precision
        _route("route_train_odd", 3333, 3, 13, 1001, "f32", True),
        # the next tokens of eight sequences: weights of most experts are read for a token or two each
        _experts("experts_some_tokens", 8, 2, 16, 4096, 1024, "bf16", False),
        # a prompt through the second half of a block of experts, rows sorted already
        _experts("experts_forward", 8192, 2, 8, 1024, 4096, "bf16", False, gather=False),
        # a training step on the first half
        _experts("experts_train", 8192, 2, 16, 4096, 1024, "bf16", True),
        # many experts of few rows, sizes that fit no vector, half precision
        _experts("experts_train_odd", 1111, 3, 37, 333, 520, "f16", True),
    ]


def _log(rng, lo, hi):
    """An integer between lo and hi, even over the logarithm: one half of those above 80 multiples of 80, the others odd."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if v > 80:
        v = v // 80 * 80 if rng.random() < 0.5 else v - 1 + v % 2
    return max(lo, min(hi, v))


def draw(rng):
    kind, dtype, train = rng.choice(["linear", "route", "experts"]), rng.choice(["f16", "bf16", "f32"]), rng.random() < 0.5
    largest = {c["name"]: work(c) for c in listed()}
    while True:
        if kind == "linear":
            c = {"kind": kind, "rows": _log(rng, 1, 16384), "n": _log(rng, 48, 8192), "k": _log(rng, 48, 8192), "dtype": dtype, "train": train,
                 "bias": rng.random() < 0.5}
            most = largest["linear_train" if train else "linear_forward"]
        else:
            experts = _log(rng, 2, 128)
            c = {"kind": kind, "tokens": _log(rng, 1, 8192), "top": rng.randint(1, min(8, experts)), "experts": experts, "dtype": dtype,
                 "train": train}
            if kind == "route":
                c["cols"] = _log(rng, 48, 8192)
                most = largest["route_train"]
            else:
                c.update(n=_log(rng, 48, 4096), k=_log(rng, 48, 4096), gather=rng.random() < 0.5)
                most = largest["experts_train" if train else "experts_forward"]
        w = work(c)
        if w["bytes"] <= most["bytes"] and (kind == "route" or w["flops"] <= most["flops"]):
            return c


def work(case):
    """Each input read once and each output written once; operations of the formulas."""
    e, train = _ESZ[case["dtype"]], case["train"]
    if case["kind"] == "route":
        t, c = case["tokens"], case["cols"]
        r = t * case["top"]
        forward = (t + r) * c * e + (r + t) * c * e + r * 16          # gathered; combined
        if not train:
            return {"bytes": forward, "flops": 2 * r * c}
        # dy and the experts' rows read again, their gradient written; the gathered rows' gradient read, the tokens' written
        return {"bytes": forward + (t + 2 * r) * c * e + (r + t) * c * e + r * 8, "flops": 7 * r * c}
    n, k = case["n"], case["k"]
    if case["kind"] == "linear":
        rows, x_rows, sets, used = case["rows"], case["rows"], 1, 1
    else:
        rows = case["tokens"] * case["top"]
        x_rows, sets = case["tokens"] if case["gather"] else rows, case["experts"]
        used = min(sets, rows)
    if not train:      # (weights: codes and scales)
        return {"bytes": x_rows * k * e + used * n * (k + 4) + rows * n * e, "flops": 2 * rows * n * k}
    return {"bytes": x_rows * k * e + rows * (2 * n + k) * e + 8 * sets * n * k, "flops": 6 * rows * n * k}


# ---- inputs ---------------------------------------------------------------------------------------------------------------

def _activations(rows, cols, dtype, gen):
    x = torch.randn(rows, cols, generator=gen, device="cuda")
    x[:, ::61] *= 8.0
    x *= torch.exp(torch.randn(rows, 1, generator=gen, device="cuda"))
    if rows > 100:
        x[7::50] = 0.0
    return x.to(_TORCH[dtype])


def _gradients(rows, cols, dtype, gen):
    g = torch.randn(rows, cols, generator=gen, device="cuda") * torch.exp(torch.randn(rows, 1, generator=gen, device="cuda"))
    return (g * 0.02).to(_TORCH[dtype])


def _router(tokens, top, experts, gen):
    """(ids [tokens, top] int64, all of a token's different; weights [tokens, top], of a softmax over them)."""
    z = torch.randn(tokens, experts, generator=gen, device="cuda") + 0.7 * torch.randn(experts, generator=gen, device="cuda")
    value, ids = z.topk(top, dim=1)
    return ids, torch.softmax(value, 1)


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype, train = case["dtype"], case["train"]
    if case["kind"] == "route":
        t, r, c = case["tokens"], case["tokens"] * case["top"], case["cols"]
        ids, weight = _router(t, case["top"], case["experts"], gen)
        given = {"ids": ids, "weight": weight, "x": _activations(t, c, dtype, gen), "z": _activations(r, c, dtype, gen)}
        if train:
            given.update(dy=_gradients(t, c, dtype, gen), drows=_gradients(r, c, dtype, gen))
        return given
    n, k = case["n"], case["k"]
    given = {}
    if case["kind"] == "linear":
        rows, x_rows, sets = case["rows"], case["rows"], ()
        if case["bias"]:
            given["bias"] = torch.randn(n, generator=gen, device="cuda")
    else:
        rows, sets = case["tokens"] * case["top"], (case["experts"],)
        x_rows = case["tokens"] if case["gather"] else rows
        given["ids"] = _router(case["tokens"], case["top"], case["experts"], gen)[0]
    given["x"] = _activations(x_rows, k, dtype, gen)
    given["w"] = torch.randn(*sets, n, k, generator=gen, device="cuda") * (torch.rand(n, 1, generator=gen, device="cuda") + 0.5) / k ** 0.5
    if train:
        given["dy"] = _gradients(rows, n, dtype, gen)
    return given


def prepare(case, seed):
    state = {"case": case, **_inputs(case, seed)}
    (_prepare_own if own else _prepare_plain)(state)
    return state


def _prepare_own(state):
    from paper_2407_02327_amd import experts
    case, train = state["case"], state["case"]["train"]
    dt = _TORCH[case["dtype"]]
    if case["kind"] == "route":
        state["op"] = experts.ExpertRoute(case["tokens"], case["top"], case["experts"], case["cols"], dtype=dt, training=train)
        return
    if case["kind"] == "linear":
        state["op"] = op = experts.TokenLinear(case["rows"], case["n"], case["k"], x_dtype=dt, philox_seed=_SEED, bias=case["bias"],
                                               training=train)
        if case["bias"]:
            op.bias.copy_(state["bias"])
    else:
        state["route"] = experts.ExpertRoute(case["tokens"], case["top"], case["experts"])
        state["route"].sort(state["ids"])
        state["op"] = op = experts.ExpertLinear(case["tokens"] * case["top"], case["n"], case["k"], case["experts"], x_dtype=dt,
                                                philox_seed=_SEED, gather=case["gather"], training=train)
    if not train:
        op.convert_w(state["w"])
        del state["w"]


def _prepare_plain(state):
    case = state["case"]
    if case["kind"] == "route":
        return
    if case["kind"] == "experts":      # (the program that made the ids knows how many rows each expert has)
        offsets, source, _ = _sort(state["ids"], case["experts"])
        state.update(source=source, bounds=offsets.tolist())
    if not case["train"]:
        state["wq"], state["sw"] = _codes(state["w"], -1)
        del state["w"]


# ---- one pass -------------------------------------------------------------------------------------------------------------

def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(state):
    case, op = state["case"], state["op"]
    if case["kind"] == "route":
        offsets = op.sort(state["ids"])
        out = {"offsets": offsets, "rows": op.gather(state["x"]), "y": op.combine(state["z"], state["weight"])}
        if case["train"]:
            out["dz"], out["dweight"] = op.combine_backward(state["dy"])
            out["dx"] = op.gather_backward(state["drows"])
        return out
    route = () if case["kind"] == "linear" else (state["route"],)
    if not case["train"]:
        return {"y": op.forward(state["x"], *route)}
    op.offset = 0      # (the same rounding in every pass)
    y = op.forward(state["x"], *route, w=state["w"])
    dx, dw, db = op.backward(state["dy"])
    out = {"y": y, "dx": dx, "dw": dw}
    if db is not None:
        out["db"] = db
    return out


def _sort(ids, experts):
    """(offsets [experts + 1], source: the sorted rows' places in ids, slot: where each of them went)."""
    flat = ids.reshape(-1)
    source = torch.sort(flat, stable=True).indices
    slot = torch.empty_like(source)
    slot[source] = torch.arange(flat.numel(), device=flat.device)
    counts = (flat[:, None] == torch.arange(experts, device=flat.device)).sum(0)
    offsets = torch.cat([counts.new_zeros(1), counts.cumsum(0)])
    return offsets.to(torch.int32), source, slot.view(ids.shape)


def _draws(rows, cols):
    """The 16-bit draws of a gradient's elements: Philox4x32-10, a block for eight elements of a row, counters row after row."""
    per_row = (cols + 7) // 8
    block = torch.arange(rows * per_row, device="cuda")
    c = [block & 0xFFFFFFFF, block >> 32, torch.zeros_like(block), torch.zeros_like(block)]
    k0, k1 = _SEED & 0xFFFFFFFF, _SEED >> 32
    for _ in range(10):
        p0, p1 = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57      # (modulo 2^64)
        c = [((p1 >> 32) & 0xFFFFFFFF) ^ c[1] ^ k0, p1 & 0xFFFFFFFF, ((p0 >> 32) & 0xFFFFFFFF) ^ c[3] ^ k1, p0 & 0xFFFFFFFF]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    words = torch.stack(c, 1).to(torch.float64)            # (exact)
    low = torch.remainder(words, 65536.0)
    u = torch.stack([low, (words - low) / 65536.0], 2).to(torch.float32)
    return u.view(rows, per_row * 8)[:, :cols]


def _codes(x, dim, u=None):
    """(codes, scales) with a scale for each slice along `dim`; `u`: the draws of stochastic rounding."""
    x = x.float()
    top = x.abs().amax(dim, keepdim=True)
    some = top >= _TINY
    # one correctly rounded division each (between tensors: torch multiplies by the inverse of a number)
    top, most = torch.where(some, top, 1.0).double(), torch.full((), 127.0, dtype=torch.float64, device=x.device)
    scale = torch.where(some, (top / most).float(), 1.0)
    inverse = torch.where(some, (most / top).float(), 0.0)
    v = x * inverse
    if u is None:
        q = torch.round(v)
    else:
        down = torch.floor(v)
        q = down + (u < torch.floor((v - down) * 65536.0))
    return q.clamp(-127.0, 127.0), scale


def _run_plain(state):
    case, train = state["case"], state["case"]["train"]
    dt = _TORCH[case["dtype"]]
    if case["kind"] == "route":
        offsets, source, slot = _sort(state["ids"], case["experts"])
        token = source // case["top"]
        weight = state["weight"]
        back = state["z"].float()[slot]                                  # [tokens, top, cols]
        out = {"offsets": offsets, "rows": state["x"][token], "y": (weight[:, :, None] * back).sum(1).to(dt)}
        if train:
            dy = state["dy"].float()
            out["dz"] = (weight.reshape(-1)[source][:, None] * dy[token]).to(dt)
            out["dweight"] = (back * dy[:, None, :]).sum(2)
            out["dx"] = state["drows"].float()[slot].sum(1).to(dt)
        return out
    if case["kind"] == "linear":
        parts = [(0, case["rows"])]
        x = state["x"].float()
        weights = lambda name: state[name][None]
    else:
        parts = list(zip(state["bounds"][:-1], state["bounds"][1:]))
        x = state["x"].float()
        if case["gather"]:
            x = x[state["source"] // case["top"]]
        weights = lambda name: state[name]
    xq, sx = _codes(x, 1)
    if train:
        wq, sw = _codes(weights("w"), 2)
        wc, swc = _codes(weights("w"), 1)
        dy = state["dy"].float()
        u = _draws(*dy.shape)
        dyq, sdy = _codes(dy, 1, u)
    else:
        wq, sw = weights("wq"), weights("sw")
    bias = state.get("bias")
    ys, dxs, dws = [], [], []
    for e, (a, b) in enumerate(parts):
        y = (xq[a:b] @ wq[e].t()) * (sx[a:b] * sw[e].t())
        ys.append((y if bias is None else y + bias).to(dt))
        if not train:
            continue
        dxs.append(((dyq[a:b] @ wc[e]) * (sdy[a:b] * swc[e])).to(dt))
        if a == b:
            dws.append(torch.zeros_like(wq[e]))
            continue
        dyc, sdyc = _codes(dy[a:b], 0, u[a:b])
        xc, sxc = _codes(x[a:b], 0)
        dws.append((dyc.t() @ xc) * (sdyc.t() * sxc))
    out = {"y": torch.cat(ys)}
    if train:
        out.update(dx=torch.cat(dxs), dw=dws[0] if case["kind"] == "linear" else torch.stack(dws))
        if bias is not None:
            out["db"] = dy.sum(0)
    return out


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------------------

def exact(case, seed):
    given = _inputs(case, seed)
    if case["kind"] == "route":
        return _exact_route(case, given)
    if case["kind"] == "linear":
        order, owner = np.arange(case["rows"]), np.zeros(case["rows"], np.int64)
    else:
        flat = given["ids"].cpu().numpy().reshape(-1)
        order = np.argsort(flat, kind="stable")
        owner = flat[order]
    x = given["x"].double()
    if case["kind"] == "experts" and case["gather"]:
        x = x[torch.from_numpy(order // case["top"]).cuda()]
    w = given["w"].double().reshape(-1, case["n"], case["k"])
    rows, bias = x.shape[0], given.get("bias")
    y = torch.zeros(rows, case["n"], dtype=torch.float64, device="cuda")
    if case["train"]:
        dy = given["dy"].double()
        draws = torch.from_numpy(_exact_draws(rows, case["n"])).cuda()
        dx, dw = torch.zeros(rows, case["k"], dtype=torch.float64, device="cuda"), torch.zeros_like(w)
    for e in range(w.shape[0]):
        mine = torch.from_numpy(np.flatnonzero(owner == e)).cuda()
        if mine.numel() == 0:
            continue
        y[mine] = _quantized(x[mine]) @ _quantized(w[e]).t()
        if case["train"]:
            g, u = dy[mine], draws[mine]
            dx[mine] = _quantized(g, u) @ _quantized(w[e].t()).t()
            dw[e] = _quantized(g.t(), u.t()) @ _quantized(x[mine].t()).t()
    out = {"y": y if bias is None else y + bias.double()}
    if case["train"]:
        out.update(dx=dx, dw=dw[0] if case["kind"] == "linear" else dw)
        if bias is not None:
            out["db"] = dy.sum(0)
    return out


def _single(v):
    """Rounded to 32 bits, as the definition has it there, and back."""
    return v.float().double()


def _quantized(x, u=None):
    """The values that the codes of the rows of x stand for."""
    top = x.abs().max(1, keepdim=True).values
    zero = top < _TINY
    top = torch.where(zero, torch.ones_like(top), top)
    most = torch.full_like(top, 127.0)
    v = _single(x * _single(most / top))
    if u is None:
        q = torch.round(v)
    else:
        part = torch.floor((v - torch.floor(v)) * 65536.0)
        q = torch.floor(v) + (u < part).double()
    return q.clamp(-127.0, 127.0) * _single(top / most) * (~zero)


def _exact_draws(rows, cols):
    per_row = -(-cols // 8)
    out = np.empty((rows, per_row, 8), np.int32)
    step = max(1, (1 << 21) // per_row)
    low32, half = np.uint64(0xFFFFFFFF), np.uint64(32)
    for r in range(0, rows, step):
        n = np.arange(r * per_row, min(rows, r + step) * per_row, dtype=np.uint64)
        a, b, c, d = n & low32, n >> half, np.zeros_like(n), np.zeros_like(n)
        key = [_SEED % 2 ** 32, _SEED // 2 ** 32]
        for _ in range(10):
            left, right = a * np.uint64(0xD2511F53), c * np.uint64(0xCD9E8D57)
            a, b, c, d = (right >> half) ^ b ^ np.uint64(key[0]), right & low32, (left >> half) ^ d ^ np.uint64(key[1]), left & low32
            key = [(key[0] + 0x9E3779B9) % 2 ** 32, (key[1] + 0xBB67AE85) % 2 ** 32]
        block = out[r:r + step].reshape(-1, 8)
        for i, word in enumerate((a, b, c, d)):
            block[:, 2 * i] = word & np.uint64(0xFFFF)
            block[:, 2 * i + 1] = word >> np.uint64(16)
    return out.reshape(rows, per_row * 8)[:, :cols]


def _exact_route(case, given):
    ids = given["ids"].cpu().numpy()
    tokens, top = ids.shape
    order = sorted(range(tokens * top), key=lambda i: (ids[i // top, i % top], i))
    counts = np.bincount(ids.reshape(-1), minlength=case["experts"])
    order = torch.tensor(order, device="cuda")
    token, choice = order // top, order % top
    weight = given["weight"].double()[token, choice]
    y = torch.zeros(tokens, case["cols"], dtype=torch.float64, device="cuda")
    y.index_add_(0, token, weight[:, None] * given["z"].double())
    out = {"offsets": torch.from_numpy(np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)).cuda(),
           "rows": given["x"].double()[token], "y": y}
    if case["train"]:
        dy = given["dy"].double()[token]
        dweight, dx = torch.zeros(tokens, top, dtype=torch.float64, device="cuda"), torch.zeros_like(y)
        dweight[token, choice] = (dy * given["z"].double()).sum(1)
        dx.index_add_(0, token, given["drows"].double())
        out.update(dz=weight[:, None] * dy, dweight=dweight, dx=dx)
    return out
