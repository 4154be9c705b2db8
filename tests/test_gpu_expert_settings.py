"""Settings of a stack with experts beyond those of test_gpu_expert_stack.py: a selection bias in float32, and many lengths of chunks."""
import numpy as np
import pytest
import torch

import bct_synth as syn
from _util import to_dev, to_np
from oracle import model_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def M():
    from paper_2411_15785_amd import model
    model.mlib()
    return model


SHAPE = dict(n_layers=2, dim=256, n_q_heads=4, n_kv_heads=2, head_dim=64, ffn=96, vocab=320, capacity_M=128, batch=5, n_experts=40,
             experts_per_token=6, router_sigmoid=True, router_bias=True, router_scale=2.5)


def weights_of(s, bias=None, level=False):
    """The oracle's weights and the GPU's; bias: each layer's selection bias, float32; level: routers of zeros, whose scores are all 1/2."""
    w = syn.make_stack_weights(s, seed=35)
    for lw in w["layers"]:
        if bias is not None:
            lw["router_bias"] = bias
        if level:
            lw["w_router"] = np.zeros_like(lw["w_router"])
    dev = lambda a: to_dev(a, "f32" if a.dtype == np.float32 else "bf16")
    wd = {n: dev(w[n]) for n in ("embed", "final_norm", "head")}
    return w, {**wd, "keys": [dev(k) for k in w["keys"]], "layers": [{n: dev(v) for n, v in lw.items()} for lw in w["layers"]]}


def recorded(M, monkeypatch):
    seen, route = [], M.bctm_route

    def record(*a, **kw):
        out = route(*a, **kw)
        seen.append(out[0].cpu().numpy().astype(np.int64))
        return out

    monkeypatch.setattr(M, "bctm_route", record)
    return seen


def test_a_bias_in_float32_decides_where_bf16_would_not(M, monkeypatch):
    """Equal scores, and a bias whose steps are a thousandth of a bf16 spacing: the choice is the bias' own order.  Once as a column
    of all layers' biases, which is not contiguous."""
    s = M.StackShape(**SHAPE)
    bias = (0.5 + 2.0 ** -20 * np.random.default_rng(3).permutation(s.n_experts)).astype(np.float32)
    w, wd = weights_of(s, bias, level=True)
    wd["layers"][1]["router_bias"] = torch.from_numpy(bias).cuda()[:, None].repeat(1, 3)[:, 1]
    assert not wd["layers"][1]["router_bias"].is_contiguous()
    assert len(set(torch.from_numpy(bias).bfloat16().tolist())) == 1
    seen = recorded(M, monkeypatch)
    ids = syn.make_token_ids(31, 0, s.batch, s.vocab)
    M.BctStack(s, wd).forward(torch.from_numpy(ids).cuda())
    want = np.argsort(-bias)[:s.experts_per_token]
    assert len(seen) == s.n_layers and all((c == want).all() for c in seen)


def test_a_stack_with_a_bias_in_float32(M, monkeypatch):
    """Against the oracle with the GPU's choices, which have to be ones that its scores allow (2 % of a logit's scale, as in
    test_gpu_expert_stack.py)."""
    s = M.StackShape(**SHAPE)
    w, wd = weights_of(s, np.random.default_rng(4).normal(0, 0.1, s.n_experts).astype(np.float32))
    ref, gpu, seen = R.RefStack(s, w), M.BctStack(s, wd, max_prefill_T=9), recorded(M, monkeypatch)
    for step, T in enumerate((9, 1)):
        ids = syn.make_token_ids(31, step, s.batch * T, s.vocab)
        seen.clear()
        _, logits = gpu.forward(torch.from_numpy(ids).cuda(), T=T)
        _, want = ref.forward(ids, T=T, choices=list(seen), margin=0.02)
        a, b = R.bf16_to_f64(to_np(logits, "bf16")), R.bf16_to_f64(want)
        assert np.max(np.abs(a - b) / np.max(np.abs(b), axis=1, keepdims=True)) <= 2e-2


def test_other_types_of_a_bias_are_refused(M):
    s = M.StackShape(**SHAPE)
    _, wd = weights_of(s)
    M.BctStack(s, wd)   # bf16 as before
    for bad in (torch.float64, torch.float16):
        wd["layers"][1]["router_bias"] = torch.zeros(s.n_experts, dtype=bad, device="cuda")
        with pytest.raises(ValueError, match="router_bias"):
            M.BctStack(s, wd)


def test_chunks_of_many_lengths_share_the_large_buffers(M):
    """After a chunk of the longest length, shorter ones take no workspace and no gated rows of their own."""
    s = M.StackShape(**{**SHAPE, "batch": 8, "ffn": 256})
    _, wd = weights_of(s)
    gpu = M.BctStack(s, wd, max_prefill_T=64)
    run = lambda T: gpu.forward(torch.from_numpy(syn.make_token_ids(31, T, s.batch * T, s.vocab)).cuda(), T=T, head="last")
    run(64)
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    lengths = range(33, 64)
    for T in lengths:
        run(T)
    torch.cuda.synchronize()
    own = sum(M.bctm_expert_workspace(s.batch * T, s.experts_per_token, s.dim) + 2 * s.batch * T * s.experts_per_token * s.ffn for T in lengths)
    # seven bf16 rows of a token as wide as the stream and its heads, one tiled, plan, logits and choice: a fifth of the two
    assert torch.cuda.memory_allocated() - before < own / 2


def test_longer_chunks_take_at_most_four_times_the_largest(M):
    s = M.StackShape(**{**SHAPE, "batch": 8})
    gpu = M.BctStack(s, weights_of(s)[1], max_prefill_T=64)
    for T in range(2, 65):
        gpu.forward(torch.from_numpy(syn.make_token_ids(31, T, s.batch * T, s.vocab)).cuda(), T=T, head="last")
    kept = gpu._bufs[("shared", "workspace")]
    assert sum(t.numel() for t in kept) <= 4 * M.bctm_expert_workspace(s.batch * 64, s.experts_per_token, s.dim)


def test_a_captured_step_goes_on_after_longer_chunks(M):
    """The buffers grow between the replays of a decode step, which has the addresses of the smaller ones."""
    s = M.StackShape(**SHAPE)
    _, wd = weights_of(s)
    a, b = M.BctStack(s, wd, max_prefill_T=40), M.BctStack(s, wd, max_prefill_T=40)
    ids = torch.from_numpy(syn.make_token_ids(31, 0, s.batch, s.vocab)).cuda()
    eager = ids.clone()
    step = lambda stack, i: stack.forward(i, next_ids=i)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(a, ids)
    torch.cuda.current_stream().wait_stream(side)
    step(b, eager)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        _, logits = step(a, ids)
    for T in (3, 40, 17, 29):
        chunk = torch.from_numpy(syn.make_token_ids(31, T, s.batch * T, s.vocab)).cuda()
        for stack in (a, b):
            stack.forward(chunk, T=T, head="last")
        for _ in range(2):
            g.replay()
            _, want = step(b, eager)
            torch.cuda.synchronize()
            assert torch.equal(logits.view(torch.int16), want.view(torch.int16)) and torch.equal(ids, eager), T


@pytest.mark.parametrize("what", ["ExpertPlan", "bctm_expert_workspace"])
def test_a_step_whose_buffers_are_not_to_be_had_changes_nothing(M, what, monkeypatch):
    """The caches take a step's tokens layer by layer: a plan or workspace that is refused has to be refused before."""
    s = M.StackShape(**SHAPE)
    _, wd = weights_of(s)
    a, b = M.BctStack(s, wd, max_prefill_T=9), M.BctStack(s, wd, max_prefill_T=9)
    chunk = torch.from_numpy(syn.make_token_ids(31, 0, s.batch * 9, s.vocab)).cuda()
    ids = torch.from_numpy(syn.make_token_ids(31, 1, s.batch, s.vocab)).cuda()

    def refuse(*args):
        raise MemoryError

    with monkeypatch.context() as m:
        m.setattr(M, what, refuse)
        with pytest.raises(MemoryError):
            a.forward(chunk, T=9)
    for stack in (a, b):
        stack.forward(ids)
    (_, got), (_, want) = a.forward(chunk, T=9), b.forward(chunk, T=9)
    assert torch.equal(got.view(torch.int16), want.view(torch.int16))
