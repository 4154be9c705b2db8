"""Layers with experts in place of the dense MLP, as cases that can be timed and checked.

Four operators that stand between the norm before the MLP and the residual stream behind it:

act     a projection with bias, activation and residual in its epilogue, into bf16 or fp32: the router's logits, a dense MLP
        without a gate (model.bctm_linear_act)
route   each token's experts and their weights from the router's logits, and the tokens in the order of their experts
        (model.bctm_route)
gated   the gated product of each token with its experts, ragged rows by expert (model.bctm_expert_swiglu)
down    the experts' down projections, weighted and added up token by token (model.bctm_expert_linear)

The plain forms are elementary torch operations in 32 bits, rounded once; a router's scores with a selection bias are in 64
bits, as the border between two experts needs it.  A pair is a token and one of its experts: number token * k + slot.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
#: a drawn case stays below these, those of the largest listed ones
MAX_ACT_FLOPS = 3.6e11
MAX_SCORES = 16384 * 256
MAX_EXPERT_FLOPS = 7.3e11
MAX_EXPERT_VALUES = 64 * 2 * 1376 * 4096


def _act(name, rows, K, N, act="none", bias=True, residual=False, out="bf16", tiled=False):
    return {"name": name, "kind": "act", "rows": rows, "K": K, "N": N, "act": act, "bias": bias, "residual": residual, "out": out,
            "tiled": tiled}


def _route(name, rows, E, k, dtype="f32", sigmoid=False, bias=False, normalise=True, scale=1.0, pad=0, masked=0.0):
    """pad: columns of the logits behind the experts; masked: the share of experts that a row may not use, and of rows that are
    padding and may use none."""
    return {"name": name, "kind": "route", "rows": rows, "E": E, "k": k, "dtype": dtype, "sigmoid": sigmoid, "bias": bias,
            "normalise": normalise, "scale": scale, "pad": pad, "masked": masked}


def _gated(name, rows, K, N, E, k, skew=0.3, none=0.0):
    """skew: how much more likely some experts are than others; none: the share of tokens that are padding."""
    return {"name": name, "kind": "gated", "rows": rows, "K": K, "N": N, "E": E, "k": k, "skew": skew, "none": none}


def _down(name, rows, K, N, E, k, skew=0.3, none=0.0, residual=True):
    return {"name": name, "kind": "down", "rows": rows, "K": K, "N": N, "E": E, "k": k, "skew": skew, "none": none,
            "residual": residual}


def listed():
    return [
        # a few sequences through a small projection with everything in its epilogue: latency
        _act("act_small", 5, 1024, 1024, act="silu", residual=True),
        # the router of a layer 4096 wide over a prompt chunk of 8 sequences x 512 tokens: 64 experts, fp32 logits
        _act("act_router", 4096, 4096, 64, bias=False, out="f32"),
        # the first product of a dense MLP without a gate, 7B-shaped, over the same chunk
        _act("act_mlp_prompt", 4096, 4096, 11008, act="gelu_tanh", tiled=True),
        # one token of one sequence
        _route("route_one", 1, 64, 8),
        # a decode batch of bf16 logits in padded rows, an odd number of experts, some of them closed to a row
        _route("route_decode", 77, 60, 4, dtype="bf16", pad=4, masked=0.1),
        # a prompt chunk of 32 sequences x 512 tokens, scores that do not compete, a bias that evens out the experts' load
        _route("route_prompt", 16384, 256, 8, sigmoid=True, bias=True, scale=2.5),
        # one token through two of a few small experts: latency
        _gated("gated_one", 1, 1024, 512, 16, 2),
        # the serving batch of the 7B-shaped layer, its MLP cut into experts of an eighth of its width, eight of 64 a token
        _gated("gated_decode", 32, 4096, 1376, 64, 8),
        # the same over a prompt chunk of 8 sequences x 512 tokens
        _gated("gated_prompt", 4096, 4096, 1376, 64, 8),
        # the way back of the serving batch
        _down("down_decode", 32, 1376, 4096, 64, 8),
        # ragged prompts with padding, few experts of which some are much more liked than others
        _down("down_ragged", 777, 2080, 2048, 12, 2, skew=1.0, none=0.2),
        # the way back of the prompt chunk
        _down("down_prompt", 4096, 1376, 4096, 64, 8),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["act", "route", "gated", "gated", "down", "down"])
    if kind == "act":
        decode = rng.random() < 0.5
        rows, K = _log(rng, 1, 127) if decode else _log(rng, 128, 4096), 32 * _log(rng, 8, 344)
        N = 16 * _log(rng, 2, 688)
        while 2.0 * rows * K * N > MAX_ACT_FLOPS:
            rows = rows // 2
        return {k: v for k, v in _act("", rows, K, N, rng.choice(["none", "relu", "silu", "gelu", "gelu_tanh", "sigmoid"]),
                                      rng.random() < 0.8, rng.random() < 0.4, rng.choice(["bf16", "bf16", "f32"]),
                                      rng.random() < 0.5).items() if k != "name"}
    if kind == "route":
        E = _log(rng, 4, 512)
        rows = max(1, min(_log(rng, 1, 20000), MAX_SCORES // E))
        return {k: v for k, v in _route("", rows, E, min(E, rng.choice([1, 2, 4, 6, 8, 16])), rng.choice(["f32", "f32", "bf16"]),
                                        rng.random() < 0.5, rng.random() < 0.4, rng.random() < 0.7, rng.choice([1.0, 1.0, 2.5]),
                                        rng.choice([0, 0, 3]), rng.choice([0.0, 0.0, 0.2])).items() if k != "name"}
    E = _log(rng, 4, 128)
    k = min(E, rng.choice([1, 2, 4, 6, 8]))
    decode = rng.random() < 0.5
    rows = _log(rng, 1, 127) if decode else _log(rng, 128, 4096)
    wide, narrow = 32 * _log(rng, 16, 128), 32 * _log(rng, 8, 64)
    mats = 2 if kind == "gated" else 1
    while mats * E * wide * narrow > MAX_EXPERT_VALUES:
        narrow = 32 * max(1, narrow // 64)
    while 2.0 * mats * rows * k * wide * narrow > MAX_EXPERT_FLOPS:
        rows = rows // 2
    skew, none = rng.choice([0.0, 0.3, 1.0]), rng.choice([0.0, 0.0, 0.2])
    c = _gated("", rows, wide, narrow, E, k, skew, none) if kind == "gated" else \
        _down("", rows, narrow, wide, E, k, skew, none, rng.random() < 0.7)
    return {k: v for k, v in c.items() if k != "name"}


# ------------------------------------------------------------------ inputs


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _normal(g, shape, dtype=torch.bfloat16, std=1.0):
    return (torch.randn(shape, generator=g, device=DEV) * std).to(dtype)


def _act_inputs(c, seed):
    g = _gen(seed)
    rows, K, N = c["rows"], c["K"], c["N"]
    return {"x": _normal(g, (rows, K)), "w": _normal(g, (N, K), std=K ** -0.5), "bias": _normal(g, (N,), std=0.5) if c["bias"] else None,
            "residual": _normal(g, (rows, N)) if c["residual"] else None}


def _route_inputs(c, seed):
    g = _gen(seed)
    rows, E = c["rows"], c["E"]
    x = torch.randn((rows, E + c["pad"]), generator=g, device=DEV) * 1.5
    if c["masked"]:
        closed = torch.rand((rows, E + c["pad"]), generator=g, device=DEV) < c["masked"]
        padding = torch.rand((rows, 1), generator=g, device=DEV) < c["masked"] / 2
        x.masked_fill_(closed | padding, float("-inf"))
    return {"logits": x.to(DTYPES[c["dtype"]])[:, :E],
            "bias": torch.randn(E, generator=g, device=DEV) * 0.05 if c["bias"] else None}


def _chosen(c, g):
    """Each token's experts, int32 [rows][k], none of them (-1) for padding, and their weights."""
    rows, E, k = c["rows"], c["E"], c["k"]
    score = torch.randn((rows, E), generator=g, device=DEV) + c["skew"] * torch.randn(E, generator=g, device=DEV)
    top, ids = torch.sort(score, dim=-1, descending=True, stable=True)
    padding = torch.rand((rows, 1), generator=g, device=DEV) < c["none"]
    weights = torch.softmax(top[:, :k], -1)
    return torch.where(padding, -1, ids[:, :k]).int().contiguous(), torch.where(padding, 0.0, weights).contiguous()


def _gated_inputs(c, seed):
    g = _gen(seed)
    K, N, E = c["K"], c["N"], c["E"]
    ids, weights = _chosen(c, g)
    return {"x": _normal(g, (c["rows"], K)), "w": [_normal(g, (E, N, K), std=K ** -0.5) for _ in range(2)], "ids": ids}


def _down_inputs(c, seed):
    g = _gen(seed)
    K, N, E = c["K"], c["N"], c["E"]
    ids, weights = _chosen(c, g)
    return {"x": _normal(g, (c["rows"] * c["k"], K), std=0.5), "w": [_normal(g, (E, N, K), std=K ** -0.5)], "ids": ids,
            "weights": weights, "residual": _normal(g, (c["rows"], N)) if c["residual"] else None}


def _inputs(c, seed):
    return {"act": _act_inputs, "route": _route_inputs, "gated": _gated_inputs, "down": _down_inputs}[c["kind"]](c, seed)


def _by_expert(ids, E):
    """The pairs in the order of their experts, those without one last, and where each expert's begin."""
    flat = ids.reshape(-1).long()
    key = torch.where((flat >= 0) & (flat < E), flat, E)
    per = (key[:, None] == torch.arange(E, device=DEV)).sum(0)
    return torch.argsort(key, stable=True), torch.cat([torch.zeros(1, dtype=torch.long, device=DEV), torch.cumsum(per, 0)])


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    c, rows = case, case["rows"]
    # outputs are buffers of the program's own, as a decode loop keeps them; the rows of pairs without an expert are not written
    if c["kind"] == "act":
        s["out"] = torch.empty((rows, c["N"]), dtype=DTYPES[c["out"]], device=DEV)
    elif c["kind"] == "gated":
        s["out"] = torch.zeros((rows * c["k"], c["N"]), dtype=torch.bfloat16, device=DEV)
    elif c["kind"] == "down":
        s["out"] = torch.empty((rows, c["N"]), dtype=torch.bfloat16, device=DEV)
    if not own:
        if c["kind"] in ("gated", "down"):
            s["order"], s["offsets"] = _by_expert(s["ids"], c["E"])
            s["most"] = int((s["offsets"][1:] - s["offsets"][:-1]).max())   # rows of the expert that has most
        return s
    from paper_2411_15785_amd import model
    s["model"] = model
    if c["kind"] == "act":
        s["packed"] = model.bctm_pack_weight(s["w"])
        s["xin"] = model.bctm_pack_rows(s["x"]) if c["tiled"] else s["x"]
        del s["w"]
    elif c["kind"] == "route":
        s["experts"] = torch.empty((rows, c["k"]), dtype=torch.int32, device=DEV)
        s["weights"] = torch.empty((rows, c["k"]), dtype=torch.float32, device=DEV)
        s["plan"] = model.ExpertPlan(rows, c["k"], c["E"], DEV)
    else:
        # the router has run by then: its plan is there
        s["plan"] = model.bctm_expert_plan(s["ids"], c["E"])
        s["packed"] = [model.bctm_pack_experts(w) for w in s["w"]]
        if c["kind"] == "down":
            s["workspace"] = torch.empty(model.bctm_expert_workspace(rows, c["k"], c["N"]), dtype=torch.uint8, device=DEV)
        del s["w"]
    return s


# ------------------------------------------------------------------ one pass


def _act_plain(s):
    c = s["case"]
    y = s["x"].float() @ s["w"].float().T
    if s["bias"] is not None:
        y = y + s["bias"].float()
    act = c["act"]
    if act == "relu":
        y = torch.where(y < 0, torch.zeros_like(y), y)
    elif act == "silu":
        y = y / (1.0 + torch.exp(-y))
    elif act == "gelu":
        y = 0.5 * y * (1.0 + torch.erf(y * math.sqrt(0.5)))
    elif act == "gelu_tanh":
        y = 0.5 * y * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (y + 0.044715 * y * y * y)))
    elif act == "sigmoid":
        y = 1.0 / (1.0 + torch.exp(-y))
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return [y.to(DTYPES[c["out"]])]


def _route_plain(s):
    c = s["case"]
    k, E = c["k"], c["E"]
    # with a bias the order is that of sums, which have to be told apart
    x = s["logits"].double() if c["bias"] else s["logits"].float()
    x = torch.where(torch.isnan(x), torch.full_like(x, float("-inf")), x)
    open_ = ~torch.isneginf(x)
    if c["sigmoid"]:
        p = 1.0 / (1.0 + torch.exp(-x))
    else:
        best = x.max(-1, keepdim=True).values
        p = torch.exp(torch.where(x == best, torch.zeros_like(x), x - best))
        p = torch.where(open_, p, torch.zeros_like(p))
        p = p / p.sum(-1, keepdim=True)
    key = torch.where(open_, p + s["bias"].double(), float("-inf")) if c["bias"] else x
    order = torch.argsort(key, dim=-1, descending=True, stable=True)[:, :k]
    has = open_.gather(1, order)
    w = torch.where(has, p.gather(1, order), torch.zeros_like(p[:, :k]))
    if c["normalise"]:
        total = w.sum(-1, keepdim=True)
        w = w / torch.where(total > 0, total, torch.ones_like(total))
    ids = torch.where(has, order, torch.full_like(order, -1)).int()
    by, offsets = _by_expert(ids, E)
    return [ids, (w * c["scale"]).float(), by.int(), offsets.int()]


def _grouped(s, x, w):
    """x [pairs][K] in fp32 times the transposed weights of each pair's expert -> fp32 [pairs][N], 0 for pairs without one."""
    pairs, E = x.shape[0], w.shape[0]
    at = s["offsets"][:-1, None] + torch.arange(s["most"], device=DEV)
    pair = torch.where(at < s["offsets"][1:, None], s["order"][at.clamp(max=pairs - 1)], pairs)
    x = torch.cat([x, torch.zeros_like(x[:1])])
    y = torch.bmm(w.float(), x[pair].transpose(1, 2).contiguous()).transpose(1, 2)
    out = torch.zeros((pairs + 1, w.shape[1]), device=DEV)
    out[pair.reshape(-1)] = y.reshape(E * s["most"], -1)
    return out[:pairs]


def _gated_plain(s):
    x = s["x"].float().repeat_interleave(s["case"]["k"], 0)
    gate, up = _grouped(s, x, s["w"][0]), _grouped(s, x, s["w"][1])
    return [(gate / (1.0 + torch.exp(-gate)) * up).to(torch.bfloat16)]


def _down_plain(s):
    c = s["case"]
    y = _grouped(s, s["x"].float(), s["w"][0]).view(c["rows"], c["k"], -1)
    y = (y * s["weights"][:, :, None]).sum(1)
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return [y.to(torch.bfloat16)]


def run(state):
    s, c = state, state["case"]
    if not own:
        return {"act": _act_plain, "route": _route_plain, "gated": _gated_plain, "down": _down_plain}[c["kind"]](s)
    m = s["model"]
    if c["kind"] == "act":
        return [m.bctm_linear_act(s["xin"], s["packed"], s["bias"], c["act"], s["residual"], out=s["out"])]
    if c["kind"] == "route":
        m.bctm_route(s["logits"], c["k"], bias=s["bias"], sigmoid=c["sigmoid"], normalise=c["normalise"], scale=c["scale"],
                     experts=s["experts"], weights=s["weights"], plan=s["plan"])
        return [s["experts"], s["weights"], s["plan"].order, s["plan"].offsets]
    if c["kind"] == "gated":
        return [m.bctm_expert_swiglu(s["x"], s["packed"][0], s["packed"][1], s["plan"], out=s["out"])]
    return [m.bctm_expert_linear(s["x"], s["packed"][0], s["plan"], s["weights"], s["residual"], out=s["out"],
                                 workspace=s["workspace"])]


def work(case):
    c, rows = case, case["rows"]
    if c["kind"] == "act":
        K, N = c["K"], c["N"]
        values = N * K + rows * K + (N if c["bias"] else 0) + (rows * N if c["residual"] else 0)
        return {"bytes": 2 * values + rows * N * (4 if c["out"] == "f32" else 2), "flops": 2 * rows * N * K}
    if c["kind"] == "route":
        n, pairs = rows * c["E"], rows * c["k"]
        return {"bytes": n * (4 if c["dtype"] == "f32" else 2) + 12 * pairs + 4 * (c["E"] + 1), "flops": 4 * n}
    K, N, E, k = c["K"], c["N"], c["E"], c["k"]
    mats = 2 if c["kind"] == "gated" else 1
    tokens = rows * (1.0 - c["none"])
    pairs = max(1, round(tokens * k))
    used = max(k, round(E * (1.0 - (1.0 - k / E) ** tokens)))   # experts that have a token, if all are as likely
    values = used * mats * N * K + (tokens if c["kind"] == "gated" else pairs) * K
    values += pairs * N if c["kind"] == "gated" else rows * N * (2 if c["residual"] else 1) + 2 * pairs
    return {"bytes": int(2 * values + 4 * rows * k), "flops": 2 * pairs * mats * N * K}


# ------------------------------------------------------------------ the definitions in 64 bits


def _act_exact(c, s):
    y = torch.addmm(s["bias"].double(), s["x"].double(), s["w"].double().t()) if s["bias"] is not None else \
        torch.mm(s["x"].double(), s["w"].double().t())
    y = {"none": lambda v: v, "relu": lambda v: v.clamp(min=0), "silu": lambda v: v * torch.sigmoid(v), "sigmoid": torch.sigmoid,
         "gelu": lambda v: 0.5 * v * torch.erfc(-v / math.sqrt(2.0)),
         "gelu_tanh": lambda v: v * torch.sigmoid(math.sqrt(8.0 / math.pi) * (v + 0.044715 * v ** 3))}[c["act"]](y)
    return [y if s["residual"] is None else y + s["residual"].double()]


def _route_exact(c, s):
    x = s["logits"].double().cpu().numpy()
    bias = None if s["bias"] is None else s["bias"].double().cpu().numpy()
    rows, E, k = c["rows"], c["E"], c["k"]
    may = x > -np.inf   # neither a NaN nor closed
    with np.errstate(all="ignore"):
        if c["sigmoid"]:
            p = np.where(x >= 0, 1.0 / (1.0 + np.exp(-x)), np.exp(x) / (1.0 + np.exp(x)))
        else:
            e = np.where(may, np.exp(x - np.max(np.where(may, x, -np.inf), axis=1, keepdims=True)), 0.0)
            p = e / np.sum(e, axis=1, keepdims=True)
        rank = x if bias is None else p + bias
    first = np.lexsort((np.broadcast_to(np.arange(E), x.shape), -np.where(may, rank, -np.inf)), axis=1)[:, :k]
    some = np.take_along_axis(may, first, 1)
    w = np.where(some, np.take_along_axis(p, first, 1), 0.0)
    if c["normalise"]:
        total = w.sum(1, keepdims=True)
        w = np.divide(w, total, out=np.zeros_like(w), where=total > 0)
    ids = np.where(some, first, -1)
    flat = ids.reshape(-1)
    order = np.concatenate([np.flatnonzero(flat == e) for e in range(E)] + [np.flatnonzero(flat < 0)])
    offsets = np.concatenate([[0], np.cumsum(np.bincount(flat[flat >= 0], minlength=E))])
    return [torch.from_numpy(ids.astype(np.int32)), torch.from_numpy(w * c["scale"]), torch.from_numpy(order.astype(np.int32)),
            torch.from_numpy(offsets.astype(np.int32))]


def _pairs_of(s, e):
    return torch.nonzero(s["ids"].reshape(-1) == e)[:, 0]


def _gated_exact(c, s):
    out = torch.zeros((c["rows"] * c["k"], c["N"]), dtype=torch.float64, device=DEV)
    for e in range(c["E"]):
        p = _pairs_of(s, e)
        x = s["x"][torch.div(p, c["k"], rounding_mode="floor")].double()
        gate = x @ s["w"][0][e].double().t()
        out[p] = gate * torch.sigmoid(gate) * (x @ s["w"][1][e].double().t())
    return [out]


def _down_exact(c, s):
    out = torch.zeros((c["rows"], c["N"]), dtype=torch.float64, device=DEV)
    if s["residual"] is not None:
        out += s["residual"].double()
    weights = s["weights"].reshape(-1).double()
    for e in range(c["E"]):
        p = _pairs_of(s, e)
        y = s["x"][p].double() @ s["w"][0][e].double().t()
        out.index_add_(0, torch.div(p, c["k"], rounding_mode="floor"), weights[p, None] * y)
    return [out]


def exact(case, seed):
    s = _inputs(case, seed)
    return {"act": _act_exact, "route": _route_exact, "gated": _gated_exact, "down": _down_exact}[case["kind"]](case, s)
