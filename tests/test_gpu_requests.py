"""Head norms, rotation, adapters and sampling together, as BctStack.forward runs them for a batch of requests: against the
oracle's stack, chunk and decode steps, and captured in a graph.  Logits: within 2 % of the row's largest, what bf16 activations
allow through these layers (as for the plain stack).  Tokens: exactly those of the logits that the GPU returned."""
import numpy as np
import pytest
import torch

import bct_synth as syn
from _util import to_dev, to_np
from oracle import model_ref as R
from test_gpu_sample import reference, uniform

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def M():
    from paper_2411_15785_amd import model
    model.mlib()
    return model


def dev(a):
    return to_dev(a, "bf16")


SHAPES = {
    "gqa": dict(n_layers=3, dim=256, n_q_heads=4, n_kv_heads=2, head_dim=64, ffn=704, vocab=512, capacity_M=128, batch=5,
                head_norm=True, rope_base=10000.0),
    "partial": dict(n_layers=2, dim=256, n_q_heads=2, n_kv_heads=2, head_dim=128, ffn=512, vocab=320, capacity_M=192, batch=3,
                    rope_base=500000.0, rotary_dim=64, rope_interleaved=True),
    "norm": dict(n_layers=2, dim=128, n_q_heads=2, n_kv_heads=1, head_dim=64, ffn=256, vocab=256, capacity_M=64, batch=33, head_norm=True),
}


class Pair:
    def __init__(self, M, name, n=4, rank=8, T=0):
        self.s = s = M.StackShape(**SHAPES[name])
        w = syn.make_stack_weights(s, seed=21)
        wd = {"embed": dev(w["embed"]), "final_norm": dev(w["final_norm"]), "head": dev(w["head"]), "keys": [dev(k) for k in w["keys"]],
              "layers": [{k: dev(v) for k, v in lw.items()} for lw in w["layers"]]}
        self.ref, self.gpu = R.RefStack(s, w), M.BctStack(s, wd, max_prefill_T=T)
        self.twin = M.BctStack(s, wd, max_prefill_T=T)
        g = np.random.RandomState(5)
        shapes = s.weight_shapes()
        self.n, self.lora, packed = n, [], []
        for l in range(s.n_layers):
            scale = (0.5 + g.rand(n)).astype(np.float32)
            d = {}
            for p in ("w_q", "w_wq", "w_wv", "w_o", "w_gate", "w_up", "w_down"):
                N, K = shapes[p]
                d[p] = (syn.pack(g.randn(n, rank, K) * K ** -0.5, "bf16"), syn.pack(g.randn(n, N, rank) * 0.5 * rank ** -0.5, "bf16"), scale)
            self.lora.append(d)
            sc = torch.from_numpy(scale).cuda()
            stack = lambda names: dev(np.stack([d[p][0] for p in names], 1))
            packed.append({
                "qkv": M.bctm_lora_pack(stack(("w_q", "w_wq", "w_wv")), dev(np.concatenate([d[p][1] for p in ("w_q", "w_wq", "w_wv")], 1)), sc),
                "o": M.bctm_lora_pack(stack(("w_o",)), dev(d["w_o"][1]), sc),
                "gate_up": M.bctm_lora_pack(stack(("w_gate", "w_up")), (dev(d["w_gate"][1]), dev(d["w_up"][1])), sc),
                "down": M.bctm_lora_pack(stack(("w_down",)), dev(d["w_down"][1]), sc)})
        self.gpu.set_adapters(packed)
        self.twin.set_adapters(packed)

    def batch(self, step, T=1, at=0):
        """ids, positions, adapters of every row; sequence b stands at + 100 b and has adapter b % (n + 1), one of them none."""
        s = self.s
        ids = syn.make_token_ids(31, step, s.batch * T, s.vocab)
        pos = (np.arange(s.batch)[:, None] * 100 + at + np.arange(T)[None, :]).reshape(-1).astype(np.int32)
        ad = np.repeat(np.arange(s.batch) % (self.n + 1), T).astype(np.int32)
        return ids, (pos if s.rope_base else None), ad

    def settings(self, M, rows, step):
        g = np.random.RandomState(100 + step)
        h = dict(t=g.choice([0.0, 0.7, 1.0], rows).astype(np.float32), k=g.choice([0, 5, 50], rows).astype(np.int32),
                 p=g.choice([0.8, 0.95, 1.0], rows).astype(np.float32), m=g.choice([0.0, 0.05], rows).astype(np.float32),
                 u=uniform(rows, step))
        d = {k: torch.from_numpy(v).cuda() for k, v in h.items()}
        return h, M.Sampling(d["u"], d["t"], d["k"], d["p"], d["m"], torch.empty(rows, device="cuda"))


def to(a):
    return None if a is None else torch.from_numpy(a).cuda()


def check(got, ref_bits, h, prob, what):
    ids, logits = got
    bits = to_np(logits, "bf16")
    a, b = R.bf16_to_f64(bits), R.bf16_to_f64(ref_bits)
    err = np.max(np.abs(a - b) / np.max(np.abs(b), axis=1, keepdims=True))
    assert err <= 2e-2, f"{what}: logits differ by {err:.3e} of the row maximum"
    want = [reference(a[r], float(h["u"][r]), float(h["t"][r]), int(h["k"][r]), float(h["p"][r]), float(h["m"][r])) for r in range(len(a))]
    assert np.array_equal(ids.cpu().numpy(), [w for w, _ in want]), what
    assert np.allclose(prob.cpu().numpy(), [p for _, p in want], rtol=2.0 ** -23, atol=0), what


@pytest.mark.parametrize("name", SHAPES)
def test_chunk_then_decode(M, name):
    T = 37
    p = Pair(M, name, T=T)
    s = p.s
    ids, pos, ad = p.batch(0, T)
    h, smp = p.settings(M, s.batch * T, 0)
    _, lg = p.ref.forward(ids, T=T, positions=pos, adapters=ad, lora=p.lora)
    got = p.gpu.forward(to(ids), T=T, positions=to(pos), adapters=to(ad), sampling=smp)
    check(got, lg, h, smp.prob, "chunk")
    # the last tokens alone: the same rows
    h1, s1 = p.settings(M, s.batch, 1)
    last = np.arange(s.batch) * T + T - 1
    got1 = p.twin.forward(to(ids), T=T, head="last", positions=to(pos), adapters=to(ad), sampling=s1)
    check(got1, lg[last], h1, s1.prob, "last tokens of the chunk")
    for step in range(1, 4):
        ids, pos, ad = p.batch(step, at=T + step)
        h, smp = p.settings(M, s.batch, step)
        _, lg = p.ref.forward(ids, positions=pos, adapters=ad, lora=p.lora)
        for stack in (p.gpu, p.twin):
            got = stack.forward(to(ids), positions=to(pos), adapters=to(ad), sampling=smp)
            check(got, lg, h, smp.prob, f"decode {step}")


def test_without_the_options_nothing_changes(M):
    """No adapter on any row, greedy settings: the bits of the plain call."""
    p = Pair(M, "gqa")
    ids, pos, _ = p.batch(0)
    off = torch.full((p.s.batch,), -1, dtype=torch.int32, device="cuda")
    a = p.gpu.forward(to(ids), positions=to(pos), adapters=off,
                      sampling=M.Sampling(torch.zeros(p.s.batch, device="cuda"), torch.zeros(p.s.batch, device="cuda")))
    b = p.twin.forward(to(ids), positions=to(pos))
    assert torch.equal(a[1].view(torch.int16), b[1].view(torch.int16)) and torch.equal(a[0], b[0])


def test_captured_steps_feed_themselves(M):
    """A decode step captured once and replayed: its tokens are the next step's ids, positions advance, numbers and adapters
    change between replays; an eager stack does the same."""
    p = Pair(M, "gqa")
    s = p.s
    ids, pos, ad = (to(a) for a in p.batch(0))
    h, smp = p.settings(M, s.batch, 0)
    eager_ids = ids.clone()
    run = lambda stack, i: stack.forward(i, next_ids=i, positions=pos, adapters=ad, sampling=smp)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run(p.gpu, ids)
    torch.cuda.current_stream().wait_stream(side)
    _, eager_logits = run(p.twin, eager_ids)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        _, logits = run(p.gpu, ids)
    for step in range(1, 6):
        pos.add_(1)
        smp.uniform.copy_(to(uniform(s.batch, 50 + step)))
        ad.copy_(torch.roll(ad, 1))
        g.replay()
        _, eager_logits = run(p.twin, eager_ids)
        torch.cuda.synchronize()
        assert torch.equal(logits.view(torch.int16), eager_logits.view(torch.int16)), step
        assert torch.equal(ids, eager_ids), step


def test_refusals(M):
    p = Pair(M, "gqa")
    ids, pos, ad = (to(a) for a in p.batch(0))
    with pytest.raises(ValueError):
        p.gpu.forward(ids)                                        # positions are missing
    with pytest.raises(ValueError):
        p.gpu.forward(ids, positions=pos.long())
    with pytest.raises(ValueError):
        p.gpu.forward(ids, positions=pos, adapters=ad[:-1])
    with pytest.raises(ValueError):
        p.gpu.forward(ids, positions=pos, sampling=M.Sampling(torch.zeros(1, device="cuda")))
    with pytest.raises(ValueError):
        p.gpu.set_adapters([{}])                                  # one layer of three
    with pytest.raises(ValueError):
        p.gpu.set_adapters([{"o": p.gpu.adapters[0]["down"]}, {}, {}])
    p.gpu.set_adapters(None)
    with pytest.raises(ValueError):
        p.gpu.forward(ids, positions=pos, adapters=ad)
    with pytest.raises(ValueError):
        M.StackShape(**{**SHAPES["gqa"], "rotary_dim": 24})


def test_a_captured_step_outlives_its_adapters(M):
    """A step captured with adapters goes on with them after others have been set, whatever is allocated in between."""
    p = Pair(M, "gqa")
    s, packed = p.s, p.gpu.adapters
    ids, pos, ad = (to(a) for a in p.batch(0))
    run = lambda stack: stack.forward(ids, positions=pos, adapters=ad)
    run(p.gpu)
    run(p.twin)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        _, logits = run(p.gpu)
    p.gpu.set_adapters(None)
    size = packed[0]["qkv"].workspace_bytes(s.batch)
    others = [torch.full((size,), 7, dtype=torch.uint8, device="cuda") for _ in range(64)]
    for step in range(3):
        ids.copy_(to(p.batch(step)[0]))
        g.replay()
        _, want = run(p.twin)
        torch.cuda.synchronize()
        assert torch.equal(logits.view(torch.int16), want.view(torch.int16)), step
    assert all(bool((o == 7).all()) for o in others)


def test_a_refused_call_changes_nothing(M):
    """Wrong vectors of any kind are refused before a layer's cache has taken the tokens: the next call is as if there had been none."""
    p = Pair(M, "gqa")
    s, packed = p.s, p.gpu.adapters
    for stack in (p.gpu, p.twin):      # adapters behind the cache alone
        stack.set_adapters([{"down": d["down"]} for d in packed])
    ids, pos, ad = (to(a) for a in p.batch(0))
    n, f = s.batch, lambda k: torch.zeros(k, device="cuda")
    u = f(n)
    for kw in (dict(positions=pos[:-1]), dict(positions=pos.cpu()), dict(adapters=ad[:-1]), dict(adapters=ad.long()), dict(adapters=ad.cpu()),
               dict(adapters=torch.stack([ad, ad], 1)[:, 0]), dict(sampling=M.Sampling(None)), dict(sampling=M.Sampling(f(n + 1))),
               dict(sampling=M.Sampling(u, temperature=f(1))), dict(sampling=M.Sampling(u, top_k=f(n))), dict(sampling=M.Sampling(u, top_p=u.double())),
               dict(sampling=M.Sampling(u, min_p=u.cpu())), dict(sampling=M.Sampling(u, prob=f(n + 1))),
               dict(sampling=M.Sampling(u), next_ids=torch.empty(n + 1, dtype=torch.int32, device="cuda"))):
        with pytest.raises(ValueError):
            p.gpu.forward(ids, **{**dict(positions=pos), **kw})
    _, a = p.gpu.forward(ids, positions=pos, adapters=ad, sampling=M.Sampling(u, prob=True))
    _, b = p.twin.forward(ids, positions=pos, adapters=ad)
    assert torch.equal(a.view(torch.int16), b.view(torch.int16))
