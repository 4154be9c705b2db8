"""Refusals of the per-request operators (head norms with rotation, adapters, sampling): the C entry points check their
arguments before the first HIP call, so no GPU is needed."""
import ctypes
import weakref

import pytest

import paper_2411_15785_amd as P
from paper_2411_15785_amd import model


@pytest.fixture(scope="module")
def ML():
    return model.mlib()


A, B, C, D, E = (ctypes.c_void_p(0x1000000 * i) for i in range(1, 6))
BF16, F32, NORM, PAIRS = 1, 0, model.BCTM_HEAD_NORM, model.BCTM_ROPE_INTERLEAVED


def rope(ML, **kw):
    a = dict(q=A, qo=B, qg=None, hq=4, ldq=512, ldqo=512, k=C, ko=D, kg=None, hk=2, ldk=256, ldko=256, pos=E, freq=E, rot=128, rows=3,
             d=128, eps=1e-6, dtype=BF16, flags=NORM)
    assert set(kw) <= set(a)
    a.update(kw)
    return ML.bctm_qk_norm_rope(*a.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(rows=0), P.BCT_ERR_INVALID_ARG), (dict(q=None), P.BCT_ERR_INVALID_ARG), (dict(qo=None), P.BCT_ERR_INVALID_ARG),
    (dict(hq=0), P.BCT_ERR_INVALID_ARG), (dict(hk=0), P.BCT_ERR_INVALID_ARG), (dict(k=None), P.BCT_ERR_INVALID_ARG),
    (dict(ko=None), P.BCT_ERR_INVALID_ARG), (dict(dtype=2), P.BCT_ERR_UNSUPPORTED), (dict(flags=NORM | 1), P.BCT_ERR_INVALID_ARG),
    (dict(flags=0, rot=0, pos=None, freq=None), P.BCT_ERR_INVALID_ARG), (dict(flags=0, qg=E), P.BCT_ERR_INVALID_ARG),
    (dict(eps=-1.0), P.BCT_ERR_INVALID_ARG), (dict(eps=float("nan")), P.BCT_ERR_INVALID_ARG),
    (dict(d=120), P.BCT_ERR_UNSUPPORTED), (dict(d=272, ldq=1088, ldqo=1088, ldk=544, ldko=544), P.BCT_ERR_UNSUPPORTED),
    (dict(rot=144), P.BCT_ERR_UNSUPPORTED), (dict(rot=24), P.BCT_ERR_UNSUPPORTED), (dict(pos=None), P.BCT_ERR_INVALID_ARG),
    (dict(freq=None), P.BCT_ERR_INVALID_ARG), (dict(rot=0), P.BCT_ERR_INVALID_ARG), (dict(ldq=504), P.BCT_ERR_INVALID_ARG),
    (dict(ldko=248), P.BCT_ERR_INVALID_ARG), (dict(ldq=516), P.BCT_ERR_MISALIGNED), (dict(q=ctypes.c_void_p(0x1000008)), P.BCT_ERR_MISALIGNED),
    (dict(freq=ctypes.c_void_p(0x5000008)), P.BCT_ERR_MISALIGNED),
    # outputs over inputs: half a row further, another distance, the other input, each other
    (dict(qo=ctypes.c_void_p(0x1000000 + 512)), P.BCT_ERR_INVALID_ARG), (dict(qo=A, ldqo=640), P.BCT_ERR_INVALID_ARG),
    (dict(qo=C), P.BCT_ERR_INVALID_ARG), (dict(ko=A), P.BCT_ERR_INVALID_ARG), (dict(ko=B), P.BCT_ERR_INVALID_ARG),
    (dict(ko=ctypes.c_void_p(0x2000000 + 2 * 512 * 2 + 768)), P.BCT_ERR_INVALID_ARG),
    # side by side in one row, but one head too far to the left
    (dict(qo=A, k=ctypes.c_void_p(0x1000000 + 768), ko=ctypes.c_void_p(0x1000000 + 768), ldq=1024, ldqo=1024, ldk=1024, ldko=1024),
     P.BCT_ERR_INVALID_ARG),
    (dict(rows=0xFFFFFFFF, hq=0xFFFF0, ldq=0x7FFFF00, ldqo=0x7FFFF00, q=A, qo=A, k=None, ko=None, hk=0), P.BCT_ERR_UNSUPPORTED),
])
def test_rope_refusals(ML, kw, status):
    assert rope(ML, **kw) == status
    assert ML.bctm_last_error() != b""


def sample(ML, **kw):
    a = dict(x=A, ld=1000, t=None, k=None, p=None, m=None, u=B, ids=C, prob=None, rows=4, N=1000, dtype=BF16)
    assert set(kw) <= set(a)
    a.update(kw)
    return ML.bctm_sample(*a.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(x=None), P.BCT_ERR_INVALID_ARG), (dict(u=None), P.BCT_ERR_INVALID_ARG), (dict(ids=None), P.BCT_ERR_INVALID_ARG),
    (dict(rows=0), P.BCT_ERR_INVALID_ARG), (dict(N=0), P.BCT_ERR_INVALID_ARG), (dict(dtype=7), P.BCT_ERR_UNSUPPORTED),
    (dict(ld=999), P.BCT_ERR_INVALID_ARG), (dict(N=(1 << 22) + 1, ld=1 << 23), P.BCT_ERR_UNSUPPORTED),
    (dict(ld=1 << 60), P.BCT_ERR_UNSUPPORTED), (dict(rows=1 << 31), P.BCT_ERR_UNSUPPORTED),
    (dict(x=ctypes.c_void_p(0x1000001)), P.BCT_ERR_MISALIGNED), (dict(x=ctypes.c_void_p(0x1000002), dtype=F32), P.BCT_ERR_MISALIGNED),
])
def test_sample_refusals(ML, kw, status):
    assert sample(ML, **kw) == status
    assert ML.bctm_last_error() != b""


def lora_args(**kw):
    l = model._bctm_lora(0x6000000, 0x7000000, None, None, 0x8000000, 4, 16, 0x9000000, 1 << 20)
    for k, v in kw.items():
        assert k in dict(l._fields_)
        setattr(l, k, v)
    return ctypes.byref(l)


@pytest.mark.parametrize("kw,status", [
    (dict(a=None), P.BCT_ERR_INVALID_ARG), (dict(b=None), P.BCT_ERR_INVALID_ARG), (dict(adapter=None), P.BCT_ERR_INVALID_ARG),
    (dict(n_adapters=0), P.BCT_ERR_INVALID_ARG), (dict(rank=0), P.BCT_ERR_INVALID_ARG), (dict(rank=24), P.BCT_ERR_UNSUPPORTED),
    (dict(rank=272), P.BCT_ERR_UNSUPPORTED), (dict(n_adapters=1 << 31), P.BCT_ERR_UNSUPPORTED),
    (dict(a=0x6000008), P.BCT_ERR_MISALIGNED), (dict(b=0x7000008), P.BCT_ERR_MISALIGNED), (dict(workspace=0x9000004), P.BCT_ERR_MISALIGNED),
    (dict(workspace=None), P.BCT_ERR_BUFFER_TOO_SMALL), (dict(workspace_bytes=255), P.BCT_ERR_BUFFER_TOO_SMALL),
])
def test_adapter_refusals(ML, kw, status):
    assert ML.bctm_linear_lora(A, B, None, C, 4, 64, 32, 0, lora_args(**kw), None) == status
    assert ML.bctm_linear_split_lora(A, B, C, 16, D, 16, None, 0, 4, 64, 0, lora_args(**kw), None) == status
    up = dict(b_up=0xA000000)
    assert ML.bctm_swiglu_lora(A, B, C, D, 4, 64, 32, 0, lora_args(**{**up, **kw}), None) == status
    assert ML.bctm_last_error() != b""


def test_adapter_calls_refuse_what_the_projections_refuse(ML):
    l = lora_args()
    assert ML.bctm_linear_lora(A, B, None, C, 4, 72, 32, 0, l, None) == P.BCT_ERR_UNSUPPORTED
    assert ML.bctm_linear_lora(A, B, None, A, 4, 64, 32, 0, l, None) == P.BCT_ERR_INVALID_ARG
    assert ML.bctm_linear_lora(A, B, None, C, 4, 64, 32, 2, l, None) == P.BCT_ERR_INVALID_ARG
    assert ML.bctm_linear_lora(A, B, None, C, 4, 64, 32, 0, None, None) == P.BCT_ERR_INVALID_ARG
    assert ML.bctm_linear_split_lora(A, B, C, 16, D, 16, None, 0, 4, 64, 0, None, None) == P.BCT_ERR_INVALID_ARG
    assert ML.bctm_linear_split_lora(A, B, C, 16, None, 16, None, 0, 4, 64, 0, l, None) == P.BCT_ERR_INVALID_ARG
    assert ML.bctm_swiglu_lora(A, B, C, D, 4, 64, 32, 0, None, None) == P.BCT_ERR_INVALID_ARG
    assert ML.bctm_swiglu_lora(A, B, C, D, 4, 64, 32, 0, l, None) == P.BCT_ERR_INVALID_ARG                       # no b_up
    assert ML.bctm_linear_lora(A, B, None, C, 4, 64, 32, 0, lora_args(b_up=0xA000000), None) == P.BCT_ERR_INVALID_ARG
    size = ctypes.c_size_t(0)
    assert ML.bctm_lora_workspace(4, 64, 16, 1, ctypes.byref(size)) == 0 and size.value >= 4 * 16 * 4
    assert ML.bctm_lora_workspace(4, 64, 16, 4, ctypes.byref(size)) == P.BCT_ERR_UNSUPPORTED
    assert ML.bctm_lora_workspace(4, 65, 16, 1, ctypes.byref(size)) == P.BCT_ERR_UNSUPPORTED
    assert ML.bctm_lora_workspace(0, 64, 16, 1, ctypes.byref(size)) == P.BCT_ERR_INVALID_ARG
    assert ML.bctm_lora_workspace(4, 64, 16, 1, None) == P.BCT_ERR_INVALID_ARG
    assert ML.bctm_lora_pack(A, B, 24, 16, None) == P.BCT_ERR_UNSUPPORTED
    assert ML.bctm_lora_pack(A, B, 32, 24, None) == P.BCT_ERR_UNSUPPORTED
    assert ML.bctm_lora_pack(A, A, 32, 16, None) == P.BCT_ERR_INVALID_ARG
    assert ML.bctm_lora_pack(A, None, 32, 16, None) == P.BCT_ERR_INVALID_ARG
    assert ML.bctm_lora_pack(A, ctypes.c_void_p(0x2000008), 32, 16, None) == P.BCT_ERR_MISALIGNED


@pytest.mark.parametrize("K,rank,segments", [(4096, 16, 1), (11008, 64, 3), (64, 256, 2), (2048, 48, 2)])
def test_workspace_serves_fewer_rows(ML, K, rank, segments):
    size, before = ctypes.c_size_t(0), 0
    for rows in sorted({r + d for e in range(18) for r in (1 << e, 3 << e) for d in (-1, 0, 1) if r + d > 0}):
        assert ML.bctm_lora_workspace(rows, K, rank, segments, ctypes.byref(size)) == 0
        assert size.value >= before, rows
        before = size.value


@pytest.mark.parametrize("name", ["ldq", "ldqo", "ldk", "ldko"])
def test_row_distances_beyond_32_bits_arrive_whole(ML, name):
    """Cut to 32 bits, the first of these distances would be that of a valid call, and the second would be below the width."""
    for far in ((1 << 49) + 512, (1 << 62) + 8):
        assert rope(ML, **{name: far}) == P.BCT_ERR_UNSUPPORTED, far
        assert b"matrix too large" in ML.bctm_last_error()


def test_new_adapters_leave_the_workspaces_of_old_ones():
    """What a step on another stream or a captured one uses is not given back; one that is large enough serves on."""
    torch = pytest.importorskip("torch")
    s = model.StackShape(n_layers=2, dim=64, n_q_heads=1, n_kv_heads=1, head_dim=32, ffn=64, vocab=16, capacity_M=64, batch=3)
    stack = object.__new__(model.BctStack)     # no GPU: the bookkeeping alone
    stack.shape, stack.device, stack.embed = s, torch.device("cpu"), torch.empty(0)
    stack.adapters, stack._bufs, stack._lora_now = None, {}, {}
    adapters = lambda rank: [{"o": model.LoraWeights(torch.empty(0), None, None, None, 1, 1, rank, s.q_width, s.dim)} for _ in range(2)]
    stack.set_adapters(adapters(16))
    small = stack._lora_workspace(3)
    assert stack._lora_workspace(3) is small
    held = weakref.ref(small)
    where = small.data_ptr()
    del small
    stack.set_adapters(adapters(64))
    large = stack._lora_workspace(3)
    assert large.numel() >= adapters(64)[0]["o"].workspace_bytes(3) and large.data_ptr() != where
    stack.set_adapters(None)
    assert held() is not None
    stack.set_adapters(adapters(16))
    assert stack._lora_workspace(3) is large and held() is not None


def test_no_more_ranks_are_used_than_there_are(ML):
    assert ML.bctm_linear_lora(A, B, None, C, 4, 64, 32, 0, lora_args(used=17), None) == P.BCT_ERR_INVALID_ARG
    assert b"ranks" in ML.bctm_last_error()


def test_set_adapters_are_those_that_were_checked():
    torch = pytest.importorskip("torch")
    s = model.StackShape(n_layers=1, dim=64, n_q_heads=1, n_kv_heads=1, head_dim=32, ffn=64, vocab=16, capacity_M=64, batch=3)
    stack = object.__new__(model.BctStack)     # no GPU: the bookkeeping alone
    stack.shape, stack.embed, stack._lora_now = s, torch.empty(0), {}
    own = [{"o": model.LoraWeights(torch.empty(0), None, None, None, 1, 1, 16, s.q_width, s.dim)}]
    stack.set_adapters(own)
    own[0]["down"] = None
    assert set(stack.adapters[0]) == {"o"}
