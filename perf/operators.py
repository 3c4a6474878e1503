"""What a language model's training and evaluation do around its quantized linear operators, as measurable cases.

Three operators, each through the package's public classes:

  norm      layer norm: `forward` alone (serving, evaluation), or `forward` + `backward` with both parameter gradients (training)
  logprobs  log probabilities of given tokens with the entropy and the top alternatives of every position: `forward` alone
            (evaluation, a teacher's pass, the next tokens of a few sequences), or `forward` + `backward` (policy training)
  distill   distillation from a teacher's top logits: the loss alone (evaluation), or the loss with its gradient (training)

With `own` false the same results come from elementary torch operations in 32 bits, rounded once to the output's type.
Activations are N(0.3, 1.5) with a few wide channels, logits N(0, 2) with some likely tokens in every row; a part of the
vocabulary is masked where a case says so, and some positions have no token (-100).
"""
from __future__ import annotations

import math

import torch

own = False

_TORCH = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
_ESZ = {"f16": 2, "bf16": 2, "f32": 4}
_EPS = 1e-5


def _norm(name, rows, cols, dtype, train):
    return {"name": name, "kind": "norm", "rows": rows, "cols": cols, "dtype": dtype, "train": train}


def _logprobs(name, rows, cols, dtype, top, train=False, temperature=1.0, masked=False):
    return {"name": name, "kind": "logprobs", "rows": rows, "cols": cols, "dtype": dtype, "top": top, "train": train,
            "temperature": temperature, "masked": masked}


def _distill(name, rows, cols, dtype, k, train, temperature=2.0):
    return {"name": name, "kind": "distill", "rows": rows, "cols": cols, "dtype": dtype, "k": k, "train": train,
            "temperature": temperature}


def listed():
    return [
        # one new token of one sequence: latency is all there is
        _norm("norm_one_token", 1, 4096, "f16", False),
        # the hidden layer of the large feed-forward block, all tokens of a batch, evaluated
        _norm("norm_wide_forward", 16384, 4096, "bf16", False),
        # a training step on the block's residual stream
        _norm("norm_train", 16384, 1024, "f16", True),
        # a last, incomplete batch of a width that fits no vector; full precision
        _norm("norm_train_odd", 2187, 1001, "f32", True),
        # the next token of four sequences over a large vocabulary, sampled at a temperature, with alternatives to show
        _logprobs("logprobs_next_token", 4, 131072, "bf16", 20, temperature=0.7),
        # perplexity and alternatives of an evaluation batch
        _logprobs("logprobs_evaluate", 2048, 32768, "f16", 8),
        # an odd vocabulary in full precision, the end of it padding that is masked
        _logprobs("logprobs_odd_masked", 333, 50021, "f32", 5, masked=True),
        # a teacher's pass: the alternatives that a student is distilled from
        _logprobs("logprobs_teacher", 1024, 131072, "bf16", 64),
        # policy training: log probabilities and entropy, then their gradient
        _logprobs("logprobs_train", 2048, 65536, "bf16", 0, train=True),
        # validation loss of a student on a few positions
        _distill("distill_evaluate", 16, 32768, "f16", 64, False),
        # a student's training step, the largest
        _distill("distill_train", 4096, 65536, "bf16", 64, True),
        # the same in full precision, nothing a multiple of anything
        _distill("distill_train_odd", 517, 50021, "f32", 33, True),
    ]


def _log(rng, lo, hi):
    """An integer between lo and hi, even over the logarithm: one half of those above 80 multiples of 80, the others odd."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if v > 80:
        v = v // 80 * 80 if rng.random() < 0.5 else v - 1 + v % 2
    return max(lo, min(hi, v))


def draw(rng):
    kind = rng.choice(["norm", "logprobs", "distill"])
    dtype = rng.choice(["f16", "bf16", "f32"])
    if kind == "norm":
        while True:
            c = {"kind": "norm", "rows": _log(rng, 1, 16384), "cols": _log(rng, 64, 8192), "dtype": dtype, "train": rng.random() < 0.5}
            if work(c)["bytes"] <= work(_norm("", 16384, 4096, "bf16", False))["bytes"]:
                return c
    while True:
        rows, cols, train = _log(rng, 1, 4096), _log(rng, 1000, 131072), rng.random() < 0.5
        if kind == "logprobs":
            c = {"kind": "logprobs", "rows": rows, "cols": cols, "dtype": dtype, "top": 0 if train else rng.choice([0, 1, 5, 20, rng.randint(2, 64)]),
                 "train": train, "temperature": rng.choice([1.0, 0.7]), "masked": rng.random() < 0.3}
        else:
            c = {"kind": "distill", "rows": rows, "cols": cols, "dtype": dtype, "k": _log(rng, 1, 256), "train": train,
                 "temperature": rng.choice([1.0, 2.0, 4.0])}
        if work(c)["bytes"] <= work(_distill("", 4096, 65536, "bf16", 64, True))["bytes"]:
            return c


def work(case):
    """Each input read once and each output written once; operations of the formulas."""
    n, e, rows = case["rows"] * case["cols"], _ESZ[case["dtype"]], case["rows"]
    if case["kind"] == "norm":
        if not case["train"]:
            return {"bytes": 2 * n * e + 8 * case["cols"], "flops": 8 * n}
        # x is read again by the backward pass, long after the forward pass has written y
        return {"bytes": 5 * n * e + 20 * case["cols"] + 16 * rows, "flops": 24 * n}
    if case["kind"] == "logprobs":
        if not case["train"]:
            return {"bytes": n * e + rows * (8 + 8 + 8 * case["top"]), "flops": 8 * n}
        # ... and the logits likewise
        return {"bytes": 3 * n * e + rows * (8 + 8 + 8 + 16), "flops": 16 * n}
    return {"bytes": (2 if case["train"] else 1) * n * e + rows * (8 * case["k"] + 8), "flops": (12 if case["train"] else 6) * n}


# ---- inputs ---------------------------------------------------------------------------------------------------------------

def _spread(rows, cols, k, gen):
    """k different columns for every row, ascending."""
    stride = cols // k
    return (torch.arange(k, device="cuda") * stride)[None, :] + torch.randint(0, stride, (rows, k), generator=gen, device="cuda")


def _logits(case, gen):
    rows, cols = case["rows"], case["cols"]
    z = torch.randn(rows, cols, generator=gen, device="cuda").mul_(2.0)
    likely = _spread(rows, cols, 24, gen)
    z.scatter_add_(1, likely, 6.0 + 2.0 * torch.randn(rows, 24, generator=gen, device="cuda"))
    if case.get("masked"):
        z[:, cols - cols // 16:] = -math.inf
    return z.to(_TORCH[case["dtype"]]), likely


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rows, cols, dt = case["rows"], case["cols"], _TORCH[case["dtype"]]
    if case["kind"] == "norm":
        x = torch.randn(rows, cols, generator=gen, device="cuda").mul_(1.5).add_(0.3)
        x[:, ::61] *= 8.0
        given = {"x": x.to(dt), "gamma": torch.randn(cols, generator=gen, device="cuda").mul_(0.1).add_(1.0),
                 "beta": torch.randn(cols, generator=gen, device="cuda").mul_(0.1)}
        if case["train"]:
            given["dy"] = torch.randn(rows, cols, generator=gen, device="cuda").mul_(0.05).to(dt)
        return given
    z, likely = _logits(case, gen)
    if case["kind"] == "logprobs":
        tokens = torch.where(torch.rand(rows, generator=gen, device="cuda") < 0.7, likely[:, 5],
                             torch.randint(0, cols, (rows,), generator=gen, device="cuda"))
        if case.get("masked"):
            tokens = tokens.clamp_(max=cols - cols // 16 - 1)
        given = {"logits": z, "tokens": tokens}
        if case["train"]:
            given["tokens"] = torch.where(torch.rand(rows, generator=gen, device="cuda") < 0.05, -100, tokens)
            given["dlogp"] = torch.randn(rows, generator=gen, device="cuda")
            given["dentropy"] = torch.randn(rows, generator=gen, device="cuda").mul_(0.1)
        return given
    # the teacher's alternatives: what the student finds likely, and others
    k = case["k"]
    index = _spread(rows, cols, k, gen)
    known = min(k, 24)
    index[:, :known] = torch.where((likely[:, :known] // (cols // k)) == torch.arange(known, device="cuda"), likely[:, :known], index[:, :known])
    teacher = torch.randn(rows, k, generator=gen, device="cuda").mul_(2.0) + 0.8 * z.gather(1, index).float()
    given = {"logits": z, "teacher": teacher, "index": index.to(torch.int32)}
    if case["train"]:
        given["weight"] = torch.rand(rows, generator=gen, device="cuda").add_(0.5) * 16.0
    return given


def prepare(case, seed):
    state = {"case": case, **_inputs(case, seed)}
    if not own:
        return state
    from paper_2407_02327_amd import head
    rows, cols, dt = case["rows"], case["cols"], _TORCH[case["dtype"]]
    if case["kind"] == "norm":
        state["op"] = head.LayerNorm(rows, cols, x_dtype=dt, eps=_EPS, training=case["train"])
    elif case["kind"] == "logprobs":
        state["op"] = head.TokenLogProbs(rows, cols, top_k=case["top"], scale=1.0 / case["temperature"],
                                         dlogits_dtype=dt if case["train"] else None)
    else:
        state["op"] = head.Distillation(rows, cols, case["k"], scale=1.0 / case["temperature"],
                                        dlogits_dtype=dt if case["train"] else None)
    return state


# ---- one pass -------------------------------------------------------------------------------------------------------------

def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(state):
    case, op = state["case"], state["op"]
    if case["kind"] == "norm":
        y = op.forward(state["x"], state["gamma"], state["beta"])
        if not case["train"]:
            return {"y": y}
        dx, dgamma, dbeta = op.backward(state["dy"])
        return {"y": y, "dx": dx, "dgamma": dgamma, "dbeta": dbeta}
    if case["kind"] == "logprobs":
        logp, entropy, top_logp, top_index = op.forward(state["logits"], state["tokens"])
        out = {"logp": logp, "entropy": entropy}
        if case["train"]:
            out["dlogits"] = op.backward(state["dlogp"], state["dentropy"])
        elif case["top"]:
            out.update(top_logp=top_logp, top_index=top_index)
        return out
    if not case["train"]:
        return {"loss": op.forward(state["logits"], state["teacher"], state["index"])}
    loss, dlogits = op.forward_backward(state["logits"], state["teacher"], state["index"], state["weight"])
    return {"loss": loss, "dlogits": dlogits}


def _rank_keys(z):
    """Whole numbers in the order (value, then lower index first) of a row's entries: all different."""
    bits = (z + 0.0).view(torch.int32)
    ordered = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).to(torch.int64)
    return ordered * (1 << 32) + ((1 << 31) - torch.arange(z.shape[1], device=z.device))


def _run_plain(state):
    case = state["case"]
    if case["kind"] == "norm":
        x, gamma, beta = state["x"].float(), state["gamma"], state["beta"]
        centred = x - x.mean(1, keepdim=True)
        rstd = torch.rsqrt((centred * centred).mean(1, keepdim=True) + _EPS)
        xhat = centred * rstd
        out = {"y": (xhat * gamma + beta).to(state["x"].dtype)}
        if case["train"]:
            dy = state["dy"].float()
            g = dy * gamma
            dx = rstd * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))
            out.update(dx=dx.to(state["x"].dtype), dgamma=(dy * xhat).sum(0), dbeta=dy.sum(0))
        return out
    scale = 1.0 / case["temperature"]
    z = state["logits"].float() * scale
    top = z.amax(1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(1, keepdim=True)
    logp_all = z - top - torch.log(total)
    p = e / total
    if case["kind"] == "logprobs":
        tokens = state["tokens"][:, None]
        here = tokens >= 0
        logp = torch.where(here, logp_all.gather(1, tokens.clamp(min=0)), 0.0)
        surprise = torch.where(p > 0, p * logp_all, 0.0)
        entropy = -surprise.sum(1, keepdim=True)
        out = {"logp": logp[:, 0], "entropy": entropy[:, 0]}
        if case["train"]:
            g, h = torch.where(here, state["dlogp"][:, None], 0.0), state["dentropy"][:, None]
            d = -(g * p) - h * (surprise + p * entropy)
            d.scatter_add_(1, tokens.clamp(min=0), g)
            out["dlogits"] = (d * scale).to(state["logits"].dtype)
        elif case["top"]:
            index = _rank_keys(state["logits"].float()).topk(case["top"], dim=1).indices
            out.update(top_logp=logp_all.gather(1, index), top_index=index.to(torch.int32))
        return out
    index = state["index"].long()
    t = state["teacher"] * scale
    t = t - t.amax(1, keepdim=True)
    q = torch.exp(t)
    q_total = q.sum(1, keepdim=True)
    q, log_q = q / q_total, t - torch.log(q_total)
    out = {"loss": (q * (log_q - logp_all.gather(1, index))).sum(1)}
    if case["train"]:
        d = p.scatter_add(1, index, -q)
        out["dlogits"] = (d * (state["weight"][:, None] * scale)).to(state["logits"].dtype)
    return out


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------------------

def exact(case, seed):
    given = _inputs(case, seed)
    parts = []
    step = max(1, (1 << 26) // case["cols"])      # rows at a time
    for r in range(0, case["rows"], step):
        part = {n: t[r:r + step] if n not in ("gamma", "beta") else t for n, t in given.items()}
        parts.append(_exact_rows(case, part))
    out = {}
    for name in parts[0]:
        column = [p[name] for p in parts]
        out[name] = torch.stack(column).sum(0) if name in ("dgamma", "dbeta") else torch.cat(column)
    return out


def _exact_rows(case, given):
    if case["kind"] == "norm":
        x, gamma, beta = given["x"].double(), given["gamma"].double(), given["beta"].double()
        n = x.shape[1]
        mean = x.sum(1) / n
        var = ((x - mean[:, None]) ** 2).sum(1) / n
        std = torch.sqrt(var + _EPS)[:, None]
        unit = (x - mean[:, None]) / std
        out = {"y": unit * gamma + beta}
        if case["train"]:
            dy = given["dy"].double()
            dunit = dy * gamma
            # d unit_j / d x_i = (delta_ij - 1/n - unit_i unit_j / n) / std
            dx = (dunit - dunit.sum(1, keepdim=True) / n - unit * ((dunit * unit).sum(1, keepdim=True) / n)) / std
            out.update(dx=dx, dgamma=(dy * unit).sum(0), dbeta=dy.sum(0))
        return out
    beta = 1.0 / case["temperature"]
    z = given["logits"].double() * beta
    log_p = z - torch.logsumexp(z, 1, keepdim=True)
    if case["kind"] == "logprobs":
        rows = torch.arange(z.shape[0], device=z.device)
        tokens = given["tokens"]
        present = tokens >= 0
        logp = log_p[rows, tokens.clamp(min=0)] * present
        plogp = torch.nan_to_num(torch.exp(log_p) * log_p, nan=0.0)
        entropy = -plogp.sum(1)
        out = {"logp": logp, "entropy": entropy}
        if case["train"]:
            g, h = given["dlogp"].double() * present, given["dentropy"].double()[:, None]
            p = torch.exp(log_p)
            d = -g[:, None] * p - h * (plogp + p * entropy[:, None])
            d[rows, tokens.clamp(min=0)] += g
            out["dlogits"] = beta * d
        elif case["top"]:
            order = torch.sort(given["logits"].double(), dim=1, descending=True, stable=True).indices[:, :case["top"]]
            out.update(top_logp=log_p.gather(1, order), top_index=order.to(torch.int32))
        return out
    index = given["index"].long()
    t = given["teacher"].double() * beta
    log_q = t - torch.logsumexp(t, 1, keepdim=True)
    q = torch.exp(log_q)
    out = {"loss": (q * (log_q - log_p.gather(1, index))).sum(1)}
    if case["train"]:
        d = torch.exp(log_p)
        d.scatter_add_(1, index, -q)
        out["dlogits"] = d * (beta * given["weight"].double()[:, None])
    return out
