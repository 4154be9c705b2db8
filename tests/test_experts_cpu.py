"""Refusals of the layers with experts and of the projection with an epilogue: the C entry points check their arguments before the
first HIP call, so no GPU is needed."""
import ctypes

import pytest

import paper_2411_15785_amd as P
from paper_2411_15785_amd import model


@pytest.fixture(scope="module")
def ML():
    return model.mlib()


A, B, C, D, E, F, G = (ctypes.c_void_p(0x1000000 * i) for i in range(1, 8))
odd = ctypes.c_void_p(0x1000008)
BF16, F32 = 1, 0
INVALID, UNSUPPORTED, MISALIGNED, SMALL = P.BCT_ERR_INVALID_ARG, P.BCT_ERR_UNSUPPORTED, P.BCT_ERR_MISALIGNED, P.BCT_ERR_BUFFER_TOO_SMALL


def call(f, defaults, kw):
    assert set(kw) <= set(defaults)
    return f(*{**defaults, **kw}.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(rows=0), INVALID), (dict(x=None), INVALID), (dict(w=None), INVALID), (dict(out=None), INVALID), (dict(K=0), INVALID),
    (dict(N=0), INVALID), (dict(K=48), UNSUPPORTED), (dict(N=24), UNSUPPORTED), (dict(act=6), INVALID), (dict(flags=4), INVALID),
    (dict(flags=32), INVALID), (dict(flags=2 | 16), INVALID), (dict(flags=2, N=80), UNSUPPORTED), (dict(out=A), INVALID),
    (dict(out=D, flags=16), INVALID), (dict(out=D, flags=2), INVALID), (dict(x=odd), MISALIGNED), (dict(bias=odd), MISALIGNED),
    (dict(res=odd), MISALIGNED), (dict(out=odd), MISALIGNED)])
def test_linear_act_refusals(ML, kw, status):
    d = dict(x=A, w=B, bias=C, res=D, out=E, rows=4, K=64, N=96, act=1, flags=0)
    assert call(ML.bctm_linear_act, d, kw) == status
    assert ML.bctm_last_error() != b""


SIZES = [(dict(rows=0), INVALID), (dict(k=0), INVALID), (dict(n=0, k=0), INVALID), (dict(n=513), UNSUPPORTED), (dict(k=17), UNSUPPORTED),
         (dict(n=3, k=4), UNSUPPORTED), (dict(rows=0x7FFFFFFF, k=2), UNSUPPORTED), (dict(rows=0xFFFFFFFF, k=1), UNSUPPORTED)]


def plan_bytes(ML, rows, k, n):
    v = ctypes.c_size_t(0)
    st = ML.bctm_expert_plan_bytes(rows, k, n, ctypes.byref(v), None)
    return st, v.value


@pytest.mark.parametrize("kw,status", SIZES)
def test_plan_sizes(ML, kw, status):
    d = dict(rows=4, k=2, n=16, **{})
    d.update(kw)
    assert plan_bytes(ML, d["rows"], d["k"], d["n"])[0] == status
    assert ML.bctm_expert_plan_bytes(4, 2, 16, None, None) == INVALID


def test_a_plan_grows_with_its_sizes(ML):
    for rows, k, n in ((1, 1, 1), (64, 8, 64), (65, 8, 64), (100000, 16, 512)):
        order = ctypes.c_size_t(0)
        v = ctypes.c_size_t(0)
        assert ML.bctm_expert_plan_bytes(rows, k, n, ctypes.byref(v), ctypes.byref(order)) == 0
        assert order.value >= n + 1 and v.value >= 4 * (order.value + rows * k) and v.value % 16 == 0
        assert plan_bytes(ML, rows + 1, k, n)[1] >= v.value


@pytest.mark.parametrize("kw,status", SIZES + [
    (dict(x=None), INVALID), (dict(ids=None), INVALID), (dict(w=None), INVALID), (dict(ld=15), INVALID), (dict(ld=1 << 60), INVALID),
    (dict(dtype=2), UNSUPPORTED), (dict(flags=4), INVALID), (dict(scale=float("nan")), INVALID), (dict(scale=float("inf")), INVALID),
    (dict(plan=odd), MISALIGNED), (dict(x=ctypes.c_void_p(0x1000002)), MISALIGNED), (dict(x=ctypes.c_void_p(0x1000001), dtype=BF16), MISALIGNED),
    (dict(bias=ctypes.c_void_p(0x1000002)), MISALIGNED), (dict(ids=ctypes.c_void_p(0x1000002)), MISALIGNED),
    (dict(w=ctypes.c_void_p(0x1000001)), MISALIGNED), (dict(size=16), SMALL)])
def test_route_refusals(ML, kw, status):
    d = dict(x=A, ld=16, bias=B, ids=C, w=D, plan=E, size=1 << 20, rows=4, n=16, k=2, scale=1.0, dtype=F32, flags=3)
    if "n" in kw:
        kw = {**kw, "ld": 600}
    assert call(ML.bctm_route, d, kw) == status
    assert ML.bctm_last_error() != b""


@pytest.mark.parametrize("kw,status", SIZES + [
    (dict(ids=None), INVALID), (dict(plan=None), INVALID), (dict(plan=odd), MISALIGNED), (dict(ids=ctypes.c_void_p(0x1000002)), MISALIGNED),
    (dict(size=16), SMALL)])
def test_plan_refusals(ML, kw, status):
    d = dict(ids=A, plan=B, size=1 << 20, rows=4, n=16, k=2)
    assert call(ML.bctm_expert_plan, d, kw) == status


PRODUCTS = SIZES + [(dict(x=None), INVALID), (dict(w=None), INVALID), (dict(out=None), INVALID), (dict(plan=None), INVALID), (dict(K=0), INVALID),
                    (dict(N=0), INVALID), (dict(K=16), UNSUPPORTED), (dict(N=8), UNSUPPORTED), (dict(out=A), INVALID), (dict(x=odd), MISALIGNED),
                    (dict(w=odd), MISALIGNED), (dict(out=odd), MISALIGNED), (dict(plan=odd), MISALIGNED), (dict(K=1 << 25), UNSUPPORTED),
                    (dict(N=1 << 25), UNSUPPORTED), (dict(rows=1 << 30, k=1, N=1 << 20), UNSUPPORTED), (dict(rows=100 << 20, k=1, K=4096, N=4096), UNSUPPORTED)]


@pytest.mark.parametrize("kw,status", PRODUCTS + [(dict(up=None), INVALID), (dict(up=odd), MISALIGNED)])
def test_expert_swiglu_refusals(ML, kw, status):
    d = dict(x=A, w=B, up=C, out=D, plan=E, rows=4, k=2, n=16, K=64, N=48)
    assert call(ML.bctm_expert_swiglu, d, kw) == status
    assert ML.bctm_last_error() != b""


@pytest.mark.parametrize("kw,status", PRODUCTS + [
    (dict(weights=None), INVALID), (dict(ws=None), INVALID), (dict(ws=odd), MISALIGNED), (dict(res=odd), MISALIGNED),
    (dict(weights=ctypes.c_void_p(0x1000002)), MISALIGNED), (dict(size=8 * 48 * 4 - 1), SMALL)])
def test_expert_linear_refusals(ML, kw, status):
    d = dict(x=A, w=B, plan=C, weights=D, res=E, out=F, ws=G, size=1 << 62, rows=4, k=2, n=16, K=64, N=48)
    assert call(ML.bctm_expert_linear, d, kw) == status
    assert ML.bctm_last_error() != b""


def test_workspace(ML):
    v = ctypes.c_size_t(0)
    assert ML.bctm_expert_workspace(4, 2, 48, ctypes.byref(v)) == 0 and v.value >= 8 * 48 * 4
    assert ML.bctm_expert_workspace(0, 2, 48, ctypes.byref(v)) == INVALID
    assert ML.bctm_expert_workspace(4, 2, 40, ctypes.byref(v)) == UNSUPPORTED
    assert ML.bctm_expert_workspace(4, 2, 48, None) == INVALID
    assert ML.bctm_expert_workspace(4, 17, 48, ctypes.byref(v)) == UNSUPPORTED
    assert ML.bctm_expert_workspace(0xFFFFFFFF, 16, 48, ctypes.byref(v)) == UNSUPPORTED


def test_python_wrappers_refuse_what_is_not_on_the_gpu():
    import torch
    x = torch.zeros((4, 64), dtype=torch.bfloat16)
    for f in (lambda: model.bctm_route(torch.zeros((4, 16)), 2), lambda: model.bctm_expert_plan(torch.zeros((4, 2), dtype=torch.int32), 16),
              lambda: model.bctm_pack_experts(torch.zeros((2, 16, 64), dtype=torch.bfloat16)),
              lambda: model.bctm_expert_swiglu(x, None, None, None), lambda: model.bctm_expert_linear(x, None, None, None),
              lambda: model.bctm_linear_act(x, None)):
        with pytest.raises(ValueError):
            f()
    with pytest.raises(model.BctModelError):
        model.ExpertPlan(4, 3, 2, "cpu")


@pytest.mark.parametrize("scale", [float("inf"), float("-inf"), float("nan"), 1e39])
def test_a_stack_refuses_a_scale_that_the_router_would(scale):
    """With the shape, not in the middle of a step."""
    shape = dict(n_layers=1, dim=64, n_q_heads=1, n_kv_heads=1, head_dim=64, ffn=64, vocab=64, capacity_M=64, batch=1, n_experts=4, experts_per_token=2)
    model.StackShape(**shape, router_scale=-2.5)
    with pytest.raises(ValueError, match="router_scale"):
        model.StackShape(**shape, router_scale=scale)
