"""Measured operators: the products and the routing of mixture-of-experts layers.

Three operators of the library, each in a plain form (elementary torch
operations in float32, or float64 for the routing, whose scores decide whole
numbers) and as the library's own call (``own``):

  linear     y = act(x w^T + bias) + residual
  moe_route  experts and weights of every row from the router's logits
  moe_ffn    the routed experts' SwiGLU feed-forward products, summed by weight

Sizes: the widths of ``workloads.configs`` (2048, 4096, 11008, 256, 688), rows
of a decoding step (1), of a verification block (K + 1 = 9, 33, 513) and of
prompts (thousands), and a generic expert bank (128 experts of 768 columns
over 2048, 8 per row).
"""

from __future__ import annotations

import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
LOWEST = -3.4028234663852886e38   # largest finite float32, negated


# ------------------------------------------------------------------- cases --

def _linear(name=None, *, rows, k, n, dtype="bf16", out="bf16", act="none", bias=False, residual=False):
    c = {"op": "linear", "rows": rows, "k": k, "n": n, "dtype": dtype, "out": out, "act": act, "bias": bias,
         "residual": residual}
    return {**c, "name": name} if name else c


def _route(name=None, *, rows, experts, top_k, dtype="f32", score="softmax", bias=False, renormalize=True, scale=1.0,
           n_groups=1, top_groups=1, group_top=1):
    c = {"op": "route", "rows": rows, "experts": experts, "top_k": top_k, "dtype": dtype, "score": score,
         "bias": bias, "renormalize": renormalize, "scale": scale, "n_groups": n_groups, "top_groups": top_groups,
         "group_top": group_top}
    return {**c, "name": name} if name else c


def _ffn(name=None, *, rows, d, f, experts, top_k, dtype="bf16", residual=False):
    c = {"op": "ffn", "rows": rows, "d": d, "f": f, "experts": experts, "top_k": top_k, "dtype": dtype,
         "residual": residual}
    return {**c, "name": name} if name else c


def listed():
    return [
        # router logits of one decoded token: the smallest product, latency alone
        _linear("router 1 row", rows=1, k=2048, n=128, out="f32"),
        # biased q/k/v projection of a Reuse block of 32 draft tokens: every weight for 33 rows
        _linear("qkv bias 33 rows", rows=33, k=4096, n=6144, bias=True),
        # output projection with the residual of the longest verification block
        _linear("out residual 513 rows", rows=513, k=4096, n=4096, residual=True),
        # an activated up projection over the rows of a batch of prompts: bound by the matrix cores
        _linear("up silu 8192 rows", rows=8192, k=4096, n=11008, bias=True, act="silu"),
        # the small fp32 model's feed-forward width, K = 8
        _linear("fp32 gelu 9 rows", rows=9, k=256, n=688, dtype="f32", out="f32", act="gelu", bias=True, residual=True),
        # routing of one decoded token
        _route("route 1 row", rows=1, experts=128, top_k=8),
        # a verification block on bf16 logits, whose ties are frequent
        _route("route bf16 513 rows", rows=513, experts=64, top_k=6, dtype="bf16", renormalize=False, scale=1.5),
        # prompts through a balanced router: sigmoid scores, bias, 4 of 8 groups
        _route("route groups 16384 rows", rows=16384, experts=256, top_k=8, score="sigmoid", bias=True, scale=2.5,
               n_groups=8, top_groups=4, group_top=2),
        # one decoded token through 8 of 128 experts: their weights stream once
        _ffn("experts 1 row", rows=1, d=2048, f=768, experts=128, top_k=8),
        # a Reuse block: almost every expert is hit by a few rows
        _ffn("experts 33 rows", rows=33, d=2048, f=768, experts=128, top_k=8, residual=True),
        # a batch of prompts: some 512 rows for every expert
        _ffn("experts 8192 rows", rows=8192, d=2048, f=768, experts=128, top_k=8),
        # the small fp32 model with a bank of 8 experts, K = 8
        _ffn("experts fp32 9 rows", rows=9, d=256, f=352, experts=8, top_k=2, dtype="f32", residual=True),
    ]


def draw(rng):
    def spread(lo, hi, step=1):
        v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / step)) * step
        return max(lo, min(hi, v))

    op = rng.choice(("linear", "route", "ffn"))
    if op == "linear":
        dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
        while True:
            rows, k, n = spread(1, 8192), spread(64, 8192, 32), spread(1, 32256)
            if rows * k * n <= 8192 * 4096 * 11008 // (1 if dtype == "bf16" else 16):
                break
        return _linear(rows=rows, k=k, n=n, dtype=dtype, out="f32" if dtype == "f32" else rng.choice(("bf16", "f32")),
                       act=rng.choice(("none", "silu", "gelu", "gelu_tanh", "relu")), bias=rng.random() < 0.5,
                       residual=rng.random() < 0.5)
    if op == "route":
        groups = rng.choice((1, 1, 2, 4, 8))
        experts = groups * spread(2, 512 // groups)
        top_groups = rng.randint(1, groups)
        top_k = min(rng.randint(1, 16), experts // groups * top_groups)
        return _route(rows=spread(1, 16384), experts=experts, top_k=top_k, dtype=rng.choice(("f32", "bf16")),
                      score=rng.choice(("softmax", "sigmoid")), bias=rng.random() < 0.5,
                      renormalize=rng.random() < 0.7, scale=rng.choice((1.0, 2.5)), n_groups=groups,
                      top_groups=top_groups, group_top=rng.choice((1, 2)))
    dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
    most = 1 if dtype == "bf16" else 16
    while True:
        rows, d, f = spread(1, 8192), spread(256, 7168, 32), spread(64, 4096, 32)
        experts = spread(2, 256)
        top_k = rng.randint(1, min(10, experts))
        if experts * d * f * most <= 128 * 2048 * 768 and rows * top_k * d * f * most <= 8192 * 8 * 2048 * 768:
            break
    return _ffn(rows=rows, d=d, f=f, experts=experts, top_k=top_k, dtype=dtype, residual=rng.random() < 0.5)


# ------------------------------------------------------------------ inputs --

def _normal(gen, *shape, std=1.0, dtype=torch.float32):
    return (torch.randn(*shape, generator=gen, device="cuda") * std).to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    c, T = case, case["rows"]
    if c["op"] == "linear":
        dt, out = DTYPES[c["dtype"]], DTYPES[c["out"]]
        return {"case": c, "x": _normal(gen, T, c["k"], dtype=dt),
                "w": _normal(gen, c["n"], c["k"], std=c["k"] ** -0.5, dtype=dt),
                "bias": _normal(gen, c["n"], std=0.5) if c["bias"] else None,
                "residual": _normal(gen, T, c["n"], dtype=out) if c["residual"] else None}
    if c["op"] == "route":
        # some experts are popular, as a router leaves them
        logits = _normal(gen, T, c["experts"], std=2.0) + _normal(gen, c["experts"])
        return {"case": c, "logits": logits.to(DTYPES[c["dtype"]]),
                "bias": _normal(gen, c["experts"], std=0.1) if c["bias"] else None}
    dt, E, d, f = DTYPES[c["dtype"]], c["experts"], c["d"], c["f"]
    popular = _normal(gen, T, E, std=2.0) + _normal(gen, E)
    top = torch.sort(popular, dim=-1, descending=True, stable=True)
    share = torch.exp(top[0][:, :c["top_k"]])
    return {"case": c, "x": _normal(gen, T, d, dtype=dt),
            "w_gate_up": _normal(gen, E, 2 * f, d, std=d ** -0.5, dtype=dt),
            "w_down": _normal(gen, E, d, f, std=f ** -0.5, dtype=dt),
            "ids": top[1][:, :c["top_k"]].to(torch.int32).contiguous(),
            "weights": (share / share.sum(-1, keepdim=True)).contiguous(),
            "residual": _normal(gen, T, d, dtype=dt) if c["residual"] else None}


# ------------------------------------------------------------- plain forms --

def _act(v, act):
    if act == "silu":
        return v / (1 + torch.exp(-v))
    if act == "gelu":
        return 0.5 * v * (1 + torch.erf(v * 0.7071067811865476))
    if act == "gelu_tanh":
        return v / (1 + torch.exp(-1.5957691216057308 * (v + 0.044715 * v * v * v)))
    return torch.where(v < 0, torch.zeros_like(v), v) if act == "relu" else v


def _plain_linear(s):
    y = s["x"].float() @ s["w"].float().t()
    if s["bias"] is not None:
        y = y + s["bias"]
    y = _act(y, s["case"]["act"])
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return y.to(DTYPES[s["case"]["out"]])


def _plain_route(s):
    c, l = s["case"], s["logits"].double()
    none = torch.full_like(l, -math.inf)
    dead = torch.isnan(l) | (l == -math.inf)
    l = torch.clamp(l, max=-LOWEST)
    if c["score"] == "softmax":
        e = torch.where(dead, torch.zeros_like(l), torch.exp(l - torch.where(dead, none, l).amax(-1, keepdim=True)))
        score = e / e.sum(-1, keepdim=True)
    else:
        score = 1 / (1 + torch.exp(-l))
    score = torch.where(dead, torch.zeros_like(l), score)
    key = score if s["bias"] is None else score + s["bias"].double()
    key = torch.where(dead, none, key)
    if c["n_groups"] > 1:
        g = key.reshape(len(key), c["n_groups"], -1)
        best = torch.sort(g, dim=-1, descending=True)[0][..., :c["group_top"]]
        value = torch.where(best == -math.inf, torch.zeros_like(best), best).sum(-1)
        value = torch.where(best[..., 0] == -math.inf, best[..., 0], value)
        order = torch.sort(value, dim=-1, descending=True, stable=True)[1][:, :c["top_groups"]]
        keep = torch.zeros_like(value, dtype=torch.bool).scatter(1, order, True)
        key = torch.where(keep[..., None], g, torch.full_like(g, -math.inf)).reshape(key.shape)
    top, ids = torch.sort(key, dim=-1, descending=True, stable=True)
    top, ids = top[:, :c["top_k"]], ids[:, :c["top_k"]]
    w = torch.where(top == -math.inf, torch.zeros_like(top), torch.gather(score, 1, ids))
    if c["renormalize"]:
        total = w.sum(-1, keepdim=True)
        w = torch.where(total > 0, w / total, torch.zeros_like(w))
    ids = torch.where(top == -math.inf, torch.full_like(ids, -1), ids)
    return ids.to(torch.int32), (w * c["scale"]).float()


def _plain_ffn(s):
    c, x, f = s["case"], s["x"].float(), s["case"]["f"]
    T, k, E = c["rows"], c["top_k"], c["experts"]
    ids = s["ids"].long().reshape(-1)
    if T * k <= E:   # fewer pairs of row and expert than experts: each pair gathers its expert's weights
        xp = x.repeat_interleave(k, 0)[:, None, :]
        gu, down = s["w_gate_up"][ids].float(), s["w_down"][ids].float()
    else:            # the pairs sorted by expert, padded to the fullest expert's rows
        count = torch.bincount(ids, minlength=E)
        first = torch.cumsum(count, 0) - count
        order = torch.argsort(ids, stable=True)
        place = torch.empty_like(ids)
        place[order] = torch.arange(T * k, device=ids.device) - first[ids[order]]
        xp = torch.zeros(E, int(count.max()), x.shape[1], device=x.device)
        xp[ids, place] = x.repeat_interleave(k, 0)
        gu, down = s["w_gate_up"].float(), s["w_down"].float()
    h = torch.bmm(xp, gu.transpose(1, 2))
    z = h[..., :f] / (1 + torch.exp(-h[..., :f])) * h[..., f:]
    y = torch.bmm(z, down.transpose(1, 2))
    y = y[:, 0] if T * k <= E else y[ids, place]
    out = (y.reshape(T, k, -1) * s["weights"][..., None]).sum(1)
    if s["residual"] is not None:
        out = out + s["residual"].float()
    return out.to(s["x"].dtype)


def run(state):
    c = state["case"]
    if own:
        import paper_2506_02780_amd as ee
        if c["op"] == "linear":
            return ee.linear(state["x"], state["w"], bias=state["bias"], act=c["act"], residual=state["residual"],
                             out_dtype=DTYPES[c["out"]])
        if c["op"] == "route":
            return ee.moe_route(state["logits"], c["top_k"], score=c["score"], bias=state["bias"],
                                renormalize=c["renormalize"], scale=c["scale"], n_groups=c["n_groups"],
                                top_groups=c["top_groups"], group_top=c["group_top"])
        return ee.moe_ffn(state["x"], state["w_gate_up"], state["w_down"], state["ids"], state["weights"],
                          residual=state["residual"])
    return {"linear": _plain_linear, "route": _plain_route, "ffn": _plain_ffn}[c["op"]](state)


# ------------------------------------------------------------ work and exact --

def work(case):
    c, T = case, case["rows"]
    size = 2 if c["dtype"] == "bf16" else 4
    if c["op"] == "linear":
        out = 2 if c["out"] == "bf16" else 4
        nbytes = size * (T * c["k"] + c["n"] * c["k"]) + out * T * c["n"] * (2 if c["residual"] else 1)
        return {"bytes": nbytes + (4 * c["n"] if c["bias"] else 0), "flops": 2 * T * c["n"] * c["k"]}
    if c["op"] == "route":
        return {"bytes": T * (c["experts"] * size + 8 * c["top_k"]) + (4 * c["experts"] if c["bias"] else 0),
                "flops": 8 * T * c["experts"]}
    # experts that some row is routed to, as if all were equally popular
    E, k, d, f = c["experts"], c["top_k"], c["d"], c["f"]
    hit = E * (1 - (1 - k / E) ** T)
    return {"bytes": size * (3 * d * f * hit + T * d * (3 if c["residual"] else 2)) + 8 * T * k,
            "flops": 6 * T * k * d * f}


def _exact_route(s):
    c = s["case"]
    l = s["logits"].double().cpu().numpy()
    T, E = l.shape
    alive = ~np.isnan(l) & (l != -np.inf)
    l = np.minimum(np.where(alive, l, 0.0), -LOWEST)
    if c["score"] == "softmax":
        e = np.where(alive, np.exp(l - np.where(alive, l, -np.inf).max(1, keepdims=True)), 0.0)
        score = e / e.sum(1, keepdims=True)
    else:
        score = np.where(alive, 1.0 / (1.0 + np.exp(-l)), 0.0)
    key = np.where(alive, score if s["bias"] is None else score + s["bias"].double().cpu().numpy(), -np.inf)
    if c["n_groups"] > 1:
        g = key.reshape(T, c["n_groups"], -1)
        left, value = g.copy(), np.zeros(g.shape[:2])
        for _ in range(min(c["group_top"], g.shape[2])):
            at = left.argmax(2)[..., None]
            best = np.take_along_axis(left, at, 2)[..., 0]
            value += np.where(best == -np.inf, 0.0, best)
            np.put_along_axis(left, at, -np.inf, 2)
        value = np.where(g.max(2) == -np.inf, -np.inf, value)
        keep = np.zeros(value.shape, bool)
        for _ in range(c["top_groups"]):
            at = np.where(keep, -np.inf, value).argmax(1)
            keep[np.arange(T), at] = True
        key = np.where(keep[..., None], g, -np.inf).reshape(T, E)
    ids, w = np.full((T, c["top_k"]), -1, np.int32), np.zeros((T, c["top_k"]))
    for j in range(c["top_k"]):
        at = key.argmax(1)   # the first of equal ones
        some = key[np.arange(T), at] > -np.inf
        ids[:, j] = np.where(some, at, -1)
        w[:, j] = np.where(some, score[np.arange(T), at], 0.0)
        key[np.arange(T), at] = -np.inf
    if c["renormalize"]:
        total = w.sum(1, keepdims=True)
        w = np.divide(w, total, out=np.zeros_like(w), where=total > 0)
    return ids, w * c["scale"]


def exact(case, seed):
    s, c = prepare(case, seed), case
    if c["op"] == "route":
        return _exact_route(s)
    if c["op"] == "linear":
        y = torch.mm(s["x"].double(), s["w"].double().T.contiguous())
        if c["bias"]:
            y += s["bias"].double()
        if c["act"] == "silu":
            y *= torch.sigmoid(y)
        elif c["act"] == "gelu":
            y *= torch.special.ndtr(y)
        elif c["act"] == "gelu_tanh":
            y *= 0.5 * (1 + torch.tanh(math.sqrt(2 / math.pi) * (y + 0.044715 * y ** 3)))
        elif c["act"] == "relu":
            y.clamp_(min=0)
        return y + s["residual"].double() if c["residual"] else y
    out = s["residual"].double() if c["residual"] else torch.zeros(c["rows"], c["d"], dtype=torch.float64, device="cuda")
    for e in range(c["experts"]):
        row, slot = torch.nonzero(s["ids"] == e, as_tuple=True)
        if not len(row):
            continue
        h = s["x"][row].double() @ s["w_gate_up"][e].double().T.contiguous()
        gate, up = h.split(c["f"], dim=1)
        y = (gate * torch.sigmoid(gate) * up) @ s["w_down"][e].double().T.contiguous()
        out.index_add_(0, row, y * s["weights"][row, slot].double()[:, None])
    return out
