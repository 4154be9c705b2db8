"""What every request of a served batch brings of its own, as cases that can be timed and checked.

Three operators between the projections, the bounded caches and the next token:

rope     norms of the queries and write queries of each head, with the position rotation in the same pass
         (model.bctm_qk_norm_rope)
lora     a shared projection with the low-rank adapter of each row's request: one output with a residual
         (model.bctm_linear_lora), several outputs (model.bctm_linear_split_lora) or the gated product of a SwiGLU
         (model.bctm_swiglu_lora)
sample   the next token of each sequence with its own temperature, top-k, top-p and min-p, from a given uniform number
         (model.bctm_sample)

The plain forms are elementary torch operations in 32 bits, rounded once; angles and the sampler's weights and sums are in
64 bits, as an angle of a far position and the border between two tokens need it.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
#: a drawn case stays below these, those of the largest listed ones
MAX_ROPE_ELEMENTS = 16384 * 64 * 128
MAX_LOGITS = 128 * 131072
MAX_LORA_FLOPS = 3.6e11


def _rope(name, rows, Hq, Hkv, d, rot, dtype="bf16", norm=True, interleaved=False, fused=True, far=4096, base=10000.0):
    return {"name": name, "kind": "rope", "rows": rows, "Hq": Hq, "Hkv": Hkv, "d": d, "rot": rot, "dtype": dtype, "norm": norm,
            "interleaved": interleaved, "fused": fused, "far": far, "base": base}


def _lora(name, form, rows, K, N, rank, n_adapters, run_length=1, none=0.0, residual=False, tiled=False):
    """run_length: consecutive rows of one request (1: a decode batch); none: the share of requests without an adapter."""
    return {"name": name, "kind": "lora", "form": form, "rows": rows, "K": K, "N": N, "rank": rank, "n_adapters": n_adapters,
            "run_length": run_length, "none": none, "residual": residual, "tiled": tiled}


def _sample(name, rows, N, dtype="bf16", settings="mixed", pad=0, masked=0.0):
    """settings: mixed (every row its own), nucleus (temperature and top-p), plain (temperature alone); pad: columns of the
    logits behind the vocabulary; masked: the share of rows in which a grammar forbids most tokens."""
    return {"name": name, "kind": "sample", "rows": rows, "N": N, "dtype": dtype, "settings": settings, "pad": pad,
            "masked": masked}


def listed():
    return [
        # one sequence of the 7B-shaped layer: 64 heads, latency
        _rope("rope_one_token", 1, 32, 32, 128, 128),
        # a decode batch with grouped heads, read in place from the fused projection's rows, at far positions
        _rope("rope_decode_gqa", 64, 32, 8, 128, 128, far=1 << 20, base=500000.0),
        # a prompt chunk of 32 sequences x 512 tokens of the 7B-shaped layer, the two projections' own outputs
        _rope("rope_prompt_7b", 16384, 32, 32, 128, 128, fused=False),
        # an fp32 layer that rotates half of each head, neighbours in pairs, and a ragged number of rows
        _rope("rope_f32_partial", 1501, 12, 4, 64, 32, dtype="f32", interleaved=True),
        # a few sequences through a small projection, one of them without an adapter
        _lora("lora_small", "linear", 5, 1024, 1024, 8, 3, none=0.2, residual=True),
        # the fused q | wq | wv projection of the 7B-shaped layer at its serving batch, an adapter for every sequence
        _lora("lora_decode_qkv", "split", 32, 4096, 12288, 16, 32, tiled=True),
        # the gated MLP over a prompt chunk of 4 sequences x 512 tokens
        _lora("lora_prompt_swiglu", "swiglu", 2048, 4096, 11008, 32, 8, run_length=512, tiled=True),
        # the down projection over ragged prompts with a residual, some requests without an adapter
        _lora("lora_prompt_down", "linear", 3587, 11008, 4096, 64, 6, run_length=300, none=0.2, residual=True, tiled=True),
        # one sequence, the 7B-shaped vocabulary, temperature and top-p
        _sample("sample_one", 1, 32000, settings="nucleus"),
        # the serving batch of the 7B-shaped model, every sequence its own settings
        _sample("sample_7b_batch", 32, 32000),
        # a wide vocabulary and a large batch, temperature and top-p: the whole row has to be weighed
        _sample("sample_wide", 128, 131072, settings="nucleus"),
        # fp32 logits of an odd vocabulary in padded rows, most of them under a grammar's mask
        _sample("sample_f32_masked", 24, 50001, dtype="f32", pad=15, masked=0.7),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rope", "lora", "sample"])
    if kind == "rope":
        d = rng.choice([64, 128])
        Hkv = rng.choice([1, 2, 4, 8, 32])
        Hq = Hkv * rng.choice([1, 2, 4, 8]) if Hkv < 32 else 32
        rows = min(_log(rng, 1, 20000), MAX_ROPE_ELEMENTS // ((Hq + Hkv) * d))
        return {k: v for k, v in _rope("", rows, Hq, Hkv, d, rng.choice([d, d, d // 2]), rng.choice(["bf16", "bf16", "f32"]),
                                       rng.random() < 0.8, rng.random() < 0.3, rng.random() < 0.5,
                                       rng.choice([4096, 65536, 1 << 20]), rng.choice([10000.0, 500000.0])).items() if k != "name"}
    if kind == "lora":
        form = rng.choice(["linear", "linear", "split", "swiglu"])
        decode = rng.random() < 0.5
        rows = _log(rng, 1, 127) if decode else _log(rng, 128, 4096)
        K = 32 * _log(rng, 8, 344)
        N = (48 if form == "split" else 16) * _log(rng, 8, 256 if form == "split" else 688)
        while 2.0 * rows * K * N * (2 if form == "swiglu" else 1) > MAX_LORA_FLOPS:
            rows = rows // 2
        n = _log(rng, 1, 32)
        return {k: v for k, v in _lora("", form, rows, K, N, rng.choice([4, 8, 16, 16, 24, 32, 64]), n,
                                       1 if decode else _log(rng, 16, 512), rng.choice([0.0, 0.0, 0.3]),
                                       form == "linear" and rng.random() < 0.5, rng.random() < 0.6).items() if k != "name"}
    N = _log(rng, 1000, 200000)
    rows = max(1, min(_log(rng, 1, 256), MAX_LOGITS // N))
    return {k: v for k, v in _sample("", rows, N, rng.choice(["bf16", "bf16", "f32"]), rng.choice(["mixed", "nucleus", "plain"]),
                                     rng.choice([0, 0, 1, 24]), rng.choice([0.0, 0.0, 0.5])).items() if k != "name"}


# ------------------------------------------------------------------ inputs


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _normal(g, shape, dtype=torch.bfloat16, std=1.0):
    return (torch.randn(shape, generator=g, device=DEV) * std).to(dtype)


def _rope_inputs(c, seed):
    g, t = _gen(seed), DTYPES[c["dtype"]]
    rows, Hq, Hkv, d = c["rows"], c["Hq"], c["Hkv"], c["d"]
    if c["fused"]:   # q | wq | wv side by side in one projection's output
        x = _normal(g, (rows, Hq + 2 * Hkv, d), t)
        q, k = x[:, :Hq], x[:, Hq:Hq + Hkv]
    else:
        q, k = _normal(g, (rows, Hq, d), t), _normal(g, (rows, Hkv, d), t)
    gains = [(1.0 + 0.2 * torch.randn(d, generator=g, device=DEV)).to(t) if c["norm"] else None for _ in range(2)]
    # a chunk of tokens runs on from where its sequence stands; a decode batch has a position for every sequence
    run = 512 if rows > 512 else 1
    start = torch.randint(0, max(1, c["far"] - run), ((rows + run - 1) // run,), generator=g, device=DEV)
    pos = (start[:, None] + torch.arange(run, device=DEV)[None, :]).reshape(-1)[:rows].to(torch.int32).contiguous()
    freq = torch.tensor([c["base"] ** (-2.0 * j / c["rot"]) for j in range(c["rot"] // 2)], dtype=torch.float64, device=DEV)
    return {"q": q, "k": k, "q_gain": gains[0], "k_gain": gains[1], "eps": 1e-6 if c["norm"] else None, "pos": pos, "freq": freq}


def _lora_inputs(c, seed):
    g = _gen(seed)
    rows, K, N, r, n = c["rows"], c["K"], c["N"], c["rank"], c["n_adapters"]
    segs = {"linear": 1, "split": 3, "swiglu": 2}[c["form"]]
    mats = 2 if c["form"] == "swiglu" else 1
    x = _normal(g, (rows, K))
    w = [_normal(g, (N, K), std=K ** -0.5) for _ in range(mats)]
    a = _normal(g, (n, segs, r, K), std=K ** -0.5)
    b = [_normal(g, (n, N, r), std=0.3 * r ** -0.5) for _ in range(mats)]
    scale = 0.5 + torch.rand(n, generator=g, device=DEV)
    requests = (rows + c["run_length"] - 1) // c["run_length"]
    ids = torch.randint(0, n, (requests,), generator=g, device=DEV)
    if c["run_length"] == 1 and n >= rows:
        ids = torch.randperm(n, generator=g, device=DEV)[:rows]
    ids = torch.where(torch.rand(requests, generator=g, device=DEV) < c["none"], torch.full_like(ids, -1), ids)
    ids = ids.repeat_interleave(c["run_length"])[:rows].to(torch.int32).contiguous()
    res = _normal(g, (rows, N)) if c["residual"] else None
    return {"x": x, "w": w, "a": a, "b": b, "scale": scale, "ids": ids, "residual": res}


def _sample_inputs(c, seed):
    g = _gen(seed)
    rows, N = c["rows"], c["N"]
    spread = 1.5 + 1.5 * torch.rand((rows, 1), generator=g, device=DEV)
    x = torch.randn((rows, N + c["pad"]), generator=g, device=DEV) * spread
    # a handful of likely tokens in each row, as a trained head gives them
    likely = torch.randint(0, N, (rows, 24), generator=g, device=DEV)
    x.scatter_add_(1, likely, 8.0 * torch.rand((rows, 24), generator=g, device=DEV))
    if c["masked"]:
        forbid = (torch.rand((rows, N + c["pad"]), generator=g, device=DEV) < 0.97) & \
                 (torch.rand((rows, 1), generator=g, device=DEV) < c["masked"])
        x.masked_fill_(forbid, float("-inf"))
    x = x.to(DTYPES[c["dtype"]])

    def pick(values, dtype):
        v = torch.tensor(values, dtype=dtype, device=DEV)
        return v[torch.randint(0, len(values), (rows,), generator=g, device=DEV)].contiguous()

    mixed = c["settings"] == "mixed"
    return {"x": x, "N": N, "u": torch.rand(rows, generator=g, device=DEV),
            "t": pick([0.0, 0.6, 0.8, 1.0, 1.0, 1.3] if mixed else [0.7, 0.9, 1.0, 1.2], torch.float32),
            "top_k": pick([0, 0, 20, 50, 200], torch.int32) if mixed else None,
            "top_p": pick([1.0, 0.95, 0.9, 0.8] if mixed else [0.98, 0.95, 0.9], torch.float32) if c["settings"] != "plain" else None,
            "min_p": pick([0.0, 0.0, 0.02, 0.1], torch.float32) if mixed else None}


def _inputs(c, seed):
    return {"rope": _rope_inputs, "lora": _lora_inputs, "sample": _sample_inputs}[c["kind"]](c, seed)


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if not own:
        return s
    from paper_2411_15785_amd import model
    s["model"] = model
    if case["kind"] == "rope":
        # outputs are buffers of the program's own, as a decode loop keeps them
        s["out"] = [torch.empty(x.shape, dtype=x.dtype, device=DEV) for x in (s["q"], s["k"])]
    elif case["kind"] == "lora":
        rows, N = case["rows"], case["N"]
        s["packed"] = [model.bctm_pack_weight(w) for w in s["w"]]
        s["adapters"] = model.bctm_lora_pack(s["a"], s["b"], s["scale"])
        s["xin"] = model.bctm_pack_rows(s["x"]) if case["tiled"] else s["x"]
        widths = [N // 3] * 3 if case["form"] == "split" else [N]
        s["out"] = [torch.empty((rows, n), dtype=torch.bfloat16, device=DEV) for n in widths]
        del s["w"], s["a"], s["b"]
    else:
        s["ids"] = torch.empty(case["rows"], dtype=torch.int32, device=DEV)
        s["prob"] = torch.empty(case["rows"], dtype=torch.float32, device=DEV)
    return s


# ------------------------------------------------------------------ one pass


def _rope_plain(s):
    c = s["case"]
    half = c["rot"] // 2
    angle = s["pos"].double()[:, None, None] * s["freq"]
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    outs = []
    for x, gain in ((s["q"], s["q_gain"]), (s["k"], s["k_gain"])):
        y = x.float()
        if c["norm"]:
            y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + s["eps"]) * gain.float()
        a, b = (y[..., 0:c["rot"]:2], y[..., 1:c["rot"]:2]) if c["interleaved"] else (y[..., :half], y[..., half:c["rot"]])
        ra, rb = a * cos - b * sin, a * sin + b * cos
        turned = torch.stack((ra, rb), -1).flatten(-2) if c["interleaved"] else torch.cat((ra, rb), -1)
        outs.append(torch.cat((turned, y[..., c["rot"]:]), -1).to(x.dtype))
    return outs


def _lora_plain(s):
    c = s["case"]
    rows, n, r = c["rows"], c["n_adapters"], c["rank"]
    x, ids = s["x"].float(), s["ids"].long()
    mine = (ids[:, None] == torch.arange(n, device=DEV)) * s["scale"]
    low = (x @ s["a"].float().reshape(-1, c["K"]).T).view(rows, n, -1, r) * mine[:, :, None, None]

    def product(w, b, start, stop, seg):
        low_seg = low[:, :, seg].reshape(rows, n * r)
        y = x @ w[start:stop].float().T
        return y + low_seg @ b[:, start:stop].float().permute(0, 2, 1).reshape(n * r, stop - start)

    N = c["N"]
    if c["form"] == "swiglu":
        gate, up = (product(s["w"][i], s["b"][i], 0, N, i) for i in range(2))
        return [(gate * torch.sigmoid(gate) * up).to(torch.bfloat16)]
    if c["form"] == "split":
        return [product(s["w"][0], s["b"][0], i * N // 3, (i + 1) * N // 3, i).to(torch.bfloat16) for i in range(3)]
    y = product(s["w"][0], s["b"][0], 0, N, 0)
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return [y.to(torch.bfloat16)]


def _sample_plain(s):
    c = s["case"]
    rows, N = c["rows"], s["N"]
    x = s["x"][:, :N].float()
    x = torch.where(torch.isnan(x), torch.full_like(x, float("-inf")), x)
    v, order = torch.sort(x, dim=-1, descending=True, stable=True)
    t = s["t"].double()[:, None]
    v, first = v.double(), v[:, :1].double()
    below = torch.where(v == first, torch.zeros_like(v), v - first)
    w = torch.exp(below / torch.where(t > 0, t, torch.ones_like(t)))
    w = torch.where(torch.isneginf(v), torch.zeros_like(w), w)
    cum = torch.cumsum(w, -1)
    keep = torch.full((rows,), N, dtype=torch.long, device=DEV)
    if s["top_k"] is not None:
        k = s["top_k"].long()
        keep = torch.where((k > 0) & (k < N), k, keep)
    if s["top_p"] is not None:
        p = s["top_p"].double()
        target = p * cum.gather(1, (keep - 1)[:, None])[:, 0]
        by_p = (cum < target[:, None]).sum(-1) + 1
        keep = torch.where(p < 1, torch.minimum(keep, by_p), keep)
    if s["min_p"] is not None:
        keep = torch.minimum(keep, (w >= s["min_p"].double()[:, None]).sum(-1))
    keep = torch.clamp(keep, min=1)
    keep = torch.where(s["t"] > 0, keep, torch.ones_like(keep))
    kept = cum.gather(1, (keep - 1)[:, None])
    drawn = torch.minimum((cum <= s["u"].double()[:, None] * kept).sum(-1), keep - 1)[:, None]
    ids, prob = order.gather(1, drawn)[:, 0], (w.gather(1, drawn) / kept)[:, 0]
    left = ~torch.isneginf(first[:, 0])
    return [torch.where(left, ids, torch.full_like(ids, -1)).int(), torch.where(left, prob, torch.zeros_like(prob)).float()]


def run(state):
    s, c = state, state["case"]
    if not own:
        return {"rope": _rope_plain, "lora": _lora_plain, "sample": _sample_plain}[c["kind"]](s)
    m = s["model"]
    if c["kind"] == "rope":
        return list(m.bctm_qk_norm_rope(s["q"], s["k"], q_gain=s["q_gain"], k_gain=s["k_gain"], eps=s["eps"], positions=s["pos"],
                                        inv_freq=s["freq"], interleaved=c["interleaved"], q_out=s["out"][0], k_out=s["out"][1]))
    if c["kind"] == "lora":
        if c["form"] == "swiglu":
            return [m.bctm_swiglu_lora(s["xin"], s["packed"][0], s["packed"][1], s["adapters"], s["ids"], out=s["out"][0])]
        if c["form"] == "split":
            return list(m.bctm_linear_split_lora(s["xin"], s["packed"][0], s["adapters"], s["ids"], s["out"]))
        return [m.bctm_linear_lora(s["xin"], s["packed"][0], s["adapters"], s["ids"], s["residual"], out=s["out"][0])]
    x = s["x"] if c["pad"] == 0 else s["x"][:, :s["N"]]
    return list(m.bctm_sample(x, s["u"], temperature=s["t"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"],
                              out=s["ids"], prob=s["prob"]))


def work(case):
    c = case
    if c["kind"] == "rope":
        n = c["rows"] * (c["Hq"] + c["Hkv"]) * c["d"]
        size = 4 if c["dtype"] == "f32" else 2
        return {"bytes": 2 * n * size + 4 * c["rows"] + 4 * c["rot"], "flops": n * (4 if c["norm"] else 0) + 3 * n * c["rot"] // c["d"]}
    if c["kind"] == "lora":
        rows, K, N, r = c["rows"], c["K"], c["N"], c["rank"]
        segs, mats = {"linear": (1, 1), "split": (3, 1), "swiglu": (2, 2)}[c["form"]]
        requests = (rows + c["run_length"] - 1) // c["run_length"]
        used = min(c["n_adapters"], max(1, round(requests * (1.0 - c["none"]))))
        values = mats * N * K + rows * K + rows * N * (2 if c["residual"] else 1) + used * r * (segs * K + mats * N)
        return {"bytes": 2 * values + 4 * rows, "flops": 2 * rows * (mats * N * K + r * (segs * K + mats * N))}
    n = c["rows"] * c["N"]
    return {"bytes": n * (4 if c["dtype"] == "f32" else 2) + 28 * c["rows"], "flops": 4 * n}


# ------------------------------------------------------------------ the definitions in 64 bits


def _rope_exact(c, s):
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV), s["pos"].double()[:, None] * s["freq"][None, :])
    outs = []
    for x, gain in ((s["q"], s["q_gain"]), (s["k"], s["k_gain"])):
        y = x.double()
        if gain is not None:
            y = y / torch.sqrt(y.square().sum(-1, keepdim=True) / c["d"] + s["eps"]) * gain.double()
        pairs = y[..., :c["rot"]].unflatten(-1, (-1, 2) if c["interleaved"] else (2, -1))
        if not c["interleaved"]:
            pairs = pairs.transpose(-1, -2)
        z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn[:, None, :])
        if not c["interleaved"]:
            z = z.transpose(-1, -2)
        y[..., :c["rot"]] = z.flatten(-2)
        outs.append(y)
    return outs


def _lora_exact(c, s):
    x = s["x"].double()
    widths = [c["N"] // 3] * 3 if c["form"] == "split" else [c["N"]]

    def whole(w, b, segments):
        y = x @ w.double().T
        for i in range(c["n_adapters"]):
            mine = torch.nonzero(s["ids"] == i)[:, 0]
            if mine.numel():
                for seg, (n0, n1) in segments:
                    low = x[mine] @ s["a"][i, seg].double().T
                    y[mine, n0:n1] += s["scale"][i].double() * (low @ b[i, n0:n1].double().T)
        return y

    if c["form"] == "swiglu":
        gate, up = (whole(s["w"][i], s["b"][i], [(i, (0, c["N"]))]) for i in range(2))
        return [gate / (1.0 + torch.exp(-gate)) * up]
    ends = [sum(widths[:i + 1]) for i in range(len(widths))]
    y = whole(s["w"][0], s["b"][0], [(i, (e - n, e)) for i, (e, n) in enumerate(zip(ends, widths))])
    if s["residual"] is not None:
        y = y + s["residual"].double()
    return list(torch.split(y, widths, dim=1))


def _sample_exact(c, s):
    x = s["x"][:, :s["N"]].double().cpu().numpy()
    at = {k: None if s[k] is None else s[k].cpu().numpy().astype(np.float64) for k in ("u", "t", "top_k", "top_p", "min_p")}
    ids, probs = np.full(c["rows"], -1, np.int32), np.zeros(c["rows"])
    for r in range(c["rows"]):
        allowed = np.flatnonzero(x[r] > -np.inf)   # neither a NaN nor a forbidden token
        if allowed.size == 0:
            continue
        best = x[r, allowed].max()
        if not at["t"][r] > 0:
            ids[r], probs[r] = allowed[np.argmax(x[r, allowed])], 1.0
            continue
        ranked = allowed[np.argsort(-x[r, allowed], kind="stable")]
        with np.errstate(invalid="ignore"):
            w = np.where(x[r, ranked] == best, 1.0, np.exp((x[r, ranked] - best) / at["t"][r]))
        cum = np.cumsum(w.astype(np.longdouble))
        n = ranked.size
        if at["top_k"] is not None and 0 < at["top_k"][r] < n:
            n = int(at["top_k"][r])
        most = n
        if at["top_p"] is not None and at["top_p"][r] < 1:
            most = min(n, int(np.searchsorted(cum[:n], at["top_p"][r] * cum[n - 1], side="left")) + 1)
        if at["min_p"] is not None:
            most = min(most, int(np.count_nonzero(w >= at["min_p"][r])))
        most = max(1, most)
        j = min(most - 1, int(np.searchsorted(cum[:most], at["u"][r] * cum[most - 1], side="right")))
        ids[r], probs[r] = ranked[j], w[j] / cum[most - 1]
    return [torch.from_numpy(ids), torch.from_numpy(probs)]


def exact(case, seed):
    s = _inputs(case, seed)
    return {"rope": _rope_exact, "lora": _lora_exact, "sample": _sample_exact}[case["kind"]](case, s)
