"""ctypes binding of the bctm_ entry points (include/bct_model.h) and a driver that
chains them with the bounded-cache attention into a Llama-shaped decoder.

The driver holds weights and activations as torch tensors (device memory) and
calls the library once per operation on torch's current stream; it does no
arithmetic of its own.  There is no CPU fallback.
"""
from __future__ import annotations

import ctypes
import math
from dataclasses import dataclass

from . import binding
from .binding import BCT_OK, BctCache, BctError, _dptr, _launch, _torch

MODEL_EXPORTS = ["bctm_embed", "bctm_rmsnorm", "bctm_pack_weight", "bctm_pack_rows", "bctm_linear", "bctm_linear_split",
                 "bctm_swiglu", "bctm_linear_plan", "bctm_linear_tile", "bctm_qk_norm_rope",
                 "bctm_lora_workspace", "bctm_lora_pack", "bctm_linear_lora", "bctm_linear_split_lora", "bctm_swiglu_lora",
                 "bctm_linear_act", "bctm_expert_plan_bytes", "bctm_route", "bctm_expert_plan", "bctm_expert_swiglu",
                 "bctm_expert_tile", "bctm_expert_workspace", "bctm_expert_linear", "bctm_argmax", "bctm_sample", "bctm_last_error"]

BCTM_KERNEL_STREAMING, BCTM_KERNEL_STREAMING_WIDE, BCTM_KERNEL_TILE128, BCTM_KERNEL_TILE256 = 0, 1, 2, 3
BCTM_KERNEL_STREAMING_TRIPLE = 4

BCTM_X_TILED = 1
BCTM_OUT_TILED = 2
BCTM_HEAD_NORM = 4
BCTM_ROPE_INTERLEAVED = 8
BCTM_OUT_F32 = 16
BCTM_ACTS = {"none": 0, "relu": 1, "silu": 2, "gelu": 3, "gelu_tanh": 4, "sigmoid": 5}
BCTM_ROUTE_SIGMOID = 1
BCTM_ROUTE_NORMALISE = 2


class _bctm_lora(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("a", "b", "b_up", "scale", "adapter")] + \
        [("n_adapters", ctypes.c_uint32), ("rank", ctypes.c_uint32), ("workspace", ctypes.c_void_p),
         ("workspace_bytes", ctypes.c_size_t), ("used", ctypes.c_uint32)]


_ready = False


def mlib() -> ctypes.CDLL:
    """libbct.so with the bctm_ prototypes set."""
    global _ready
    L = binding.lib()
    if _ready:
        return L
    vp, u32 = ctypes.c_void_p, ctypes.c_uint32
    L.bctm_embed.argtypes = [vp, vp, vp, u32, u32, u32, vp]
    L.bctm_rmsnorm.argtypes = [vp, vp, vp, u32, u32, ctypes.c_float, u32, vp]
    L.bctm_pack_weight.argtypes = [vp, vp, u32, u32, vp]
    L.bctm_pack_rows.argtypes = [vp, vp, u32, u32, vp]
    L.bctm_linear.argtypes = [vp, vp, vp, vp, u32, u32, u32, u32, vp]
    L.bctm_linear_split.argtypes = [vp, vp, vp, u32, vp, u32, vp, u32, u32, u32, u32, vp]
    L.bctm_swiglu.argtypes = [vp, vp, vp, vp, u32, u32, u32, u32, vp]
    L.bctm_linear_plan.argtypes = [u32, u32, u32, u32, ctypes.POINTER(u32)]
    L.bctm_linear_tile.argtypes = [u32, u32, u32, u32, u32] + [ctypes.POINTER(u32)] * 3
    sz = ctypes.c_size_t   # a number too wide for its argument would be cut without a word
    L.bctm_qk_norm_rope.argtypes = [vp, vp, vp, u32, sz, sz] * 2 + [vp, vp, u32, u32, u32, ctypes.c_float, ctypes.c_int32, u32, vp]
    L.bctm_argmax.argtypes = [vp, vp, u32, u32, vp]
    lora = ctypes.POINTER(_bctm_lora)
    L.bctm_lora_workspace.argtypes = [u32, u32, u32, u32, ctypes.POINTER(ctypes.c_size_t)]
    L.bctm_lora_pack.argtypes = [vp, vp, u32, u32, vp]
    L.bctm_linear_lora.argtypes = L.bctm_linear.argtypes[:-1] + [lora, vp]
    L.bctm_linear_split_lora.argtypes = L.bctm_linear_split.argtypes[:-1] + [lora, vp]
    L.bctm_swiglu_lora.argtypes = L.bctm_swiglu.argtypes[:-1] + [lora, vp]
    L.bctm_sample.argtypes = [vp, ctypes.c_size_t] + [vp] * 7 + [u32, u32, ctypes.c_int32, vp]
    L.bctm_linear_act.argtypes = [vp] * 5 + [u32] * 5 + [vp]
    L.bctm_expert_plan_bytes.argtypes = [u32] * 3 + [ctypes.POINTER(sz)] * 2
    L.bctm_route.argtypes = [vp, sz] + [vp] * 4 + [sz, u32, u32, u32, ctypes.c_float, ctypes.c_int32, u32, vp]
    L.bctm_expert_plan.argtypes = [vp, vp, sz, u32, u32, u32, vp]
    L.bctm_expert_swiglu.argtypes = [vp] * 5 + [u32] * 5 + [vp]
    L.bctm_expert_tile.argtypes = [u32] * 6 + [ctypes.POINTER(u32)] * 2
    L.bctm_expert_workspace.argtypes = [u32] * 3 + [ctypes.POINTER(sz)]
    L.bctm_expert_linear.argtypes = [vp] * 7 + [sz] + [u32] * 5 + [vp]
    for n in MODEL_EXPORTS[:-1]:
        getattr(L, n).restype = ctypes.c_int
    L.bctm_last_error.argtypes = []
    L.bctm_last_error.restype = ctypes.c_char_p
    _ready = True
    return L


class BctModelError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        L = mlib()
        super().__init__(f"{where}: {L.bct_strerror(status).decode()} ({status}): {L.bctm_last_error().decode()}")


def _ck(st, where):
    if st != BCT_OK:
        raise BctModelError(st, where)


def _bf16_2d(t, name, cols=None):
    torch = _torch()
    if t.dtype != torch.bfloat16 or t.dim() != 2 or not t.is_contiguous() or not t.is_cuda or \
            (cols is not None and t.shape[1] != cols):
        raise ValueError(f"{name}: expected a contiguous 2-D bf16 device tensor"
                         + (f" with {cols} columns" if cols is not None else "")
                         + f", got {t.dtype} {tuple(t.shape)} on {t.device}")


def bctm_embed(ids, table, out=None):
    torch = _torch()
    _bf16_2d(table, "table")
    if ids.dtype != torch.int32 or ids.dim() != 1 or not ids.is_contiguous() or ids.device != table.device:
        raise ValueError("ids: expected a contiguous 1-D int32 tensor on the table's device")
    if out is None:
        out = torch.empty((ids.numel(), table.shape[1]), dtype=torch.bfloat16, device=table.device)
    _bf16_2d(out, "out", table.shape[1])
    if out.shape[0] != ids.numel():
        raise ValueError("out: one row per id")
    _ck(_launch(mlib().bctm_embed, table.device, _dptr(ids), _dptr(table), _dptr(out), ids.numel(), table.shape[0],
                table.shape[1]), "bctm_embed")
    return out


def bctm_linear_plan(rows, K, N, swiglu=False):
    """The kernel a projection of this shape runs in (one of the BCTM_KERNEL_ values); host logic, no GPU."""
    k = ctypes.c_uint32(0)
    _ck(mlib().bctm_linear_plan(rows, K, N, 1 if swiglu else 0, ctypes.byref(k)), "bctm_linear_plan")
    return k.value


def bctm_linear_tile(rows, K, N, swiglu=False, tiled=False):
    """(rows, features, parts of K) that the launch of this shape gives one workgroup; tiled: x is a TiledRows."""
    v = [ctypes.c_uint32(0) for _ in range(3)]
    _ck(mlib().bctm_linear_tile(rows, K, N, 1 if swiglu else 0, BCTM_X_TILED if tiled else 0,
                                *(ctypes.byref(a) for a in v)), "bctm_linear_tile")
    return tuple(a.value for a in v)


class TiledRows:
    """A [rows][K] activation matrix in the tiled order the projections read (include/bct_model.h):
    data holds 32 * ceil(rows / 32) * K bf16."""

    def __init__(self, rows, K, device, data=None):
        torch = _torch()
        n = 32 * ((rows + 31) // 32) * K
        if data is None:
            # zeros, not empty: rows past the end are read (never stored) and should be finite
            data = torch.zeros(n, dtype=torch.bfloat16, device=device)
        if data.dtype != torch.bfloat16 or data.numel() != n or not data.is_contiguous():
            raise ValueError(f"tiled data: expected {n} contiguous bf16")
        self.data, self.rows, self.K = data, rows, K


def bctm_pack_rows(x, out=None):
    _bf16_2d(x, "x")
    rows, K = x.shape
    if out is None:
        out = TiledRows(rows, K, x.device)
    if (out.rows, out.K) != (rows, K):
        raise ValueError("out: tiled buffer of x's shape")
    _ck(_launch(mlib().bctm_pack_rows, x.device, _dptr(x), _dptr(out.data), rows, K), "bctm_pack_rows")
    return out


def bctm_rmsnorm(x, gain, eps, out=None, tiled=False):
    """out: a tensor of x's shape, or (tiled=True) a TiledRows."""
    torch = _torch()
    _bf16_2d(x, "x")
    if gain.dtype != torch.bfloat16 or tuple(gain.shape) != (x.shape[1],) or not gain.is_contiguous() \
            or gain.device != x.device:
        raise ValueError("gain: expected a contiguous bf16 vector of x's row length on x's device")
    if tiled:
        if out is None:
            out = TiledRows(x.shape[0], x.shape[1], x.device)
        if not isinstance(out, TiledRows) or (out.rows, out.K) != tuple(x.shape):
            raise ValueError("out: a TiledRows of x's shape")
        dst = out.data
    else:
        if out is None:
            out = torch.empty_like(x)
        _bf16_2d(out, "out", x.shape[1])
        if out.shape[0] != x.shape[0]:
            raise ValueError("out: x's shape")
        dst = out
    _ck(_launch(mlib().bctm_rmsnorm, x.device, _dptr(x), _dptr(gain), _dptr(dst), x.shape[0], x.shape[1],
                eps, BCTM_OUT_TILED if tiled else 0), "bctm_rmsnorm")
    return out


def _heads(t, name, dtype, device):
    """t [rows][heads][d] with contiguous heads, its rows at any distance (a part of a wider row) -> shape, that distance."""
    shape, stride = t.shape, t.stride()
    if t.dtype is not dtype or len(shape) != 3 or t.get_device() != device or stride[2] != 1 or \
            (stride[1] != shape[2] and shape[1] > 1):
        raise ValueError(f"{name}: expected {dtype} [rows][heads][d] on cuda:{device}, heads side by side, got {t.dtype} "
                         f"{tuple(shape)} strides {stride} on {t.device}")
    if shape[0] >> 32:
        raise ValueError(f"{name}: more rows than one call takes")
    # the distance of a single row is not looked at
    return shape, stride[0] if shape[0] > 1 else shape[1] * shape[2]


def bctm_qk_norm_rope(q, k=None, q_gain=None, k_gain=None, eps=None, positions=None, inv_freq=None, interleaved=False,
                      q_out=None, k_out=None):
    """Queries [rows][Hq][d] and write queries [rows][Hkv][d] (or None), float32 or bf16: each head normalised (eps given) and
    turned by its row's position (positions int32 [rows] with inv_freq float64 [rotary_dim / 2], radians per position)
    -> (q_out, k_out).  q and k may be parts of wider rows; q_out=q and k_out=k work in place."""
    torch = _torch()
    dtype, device = q.dtype, q.get_device()
    if device < 0 or (dtype is not torch.bfloat16 and dtype is not torch.float32):
        raise ValueError(f"q: expected float32 or bf16 on the GPU, got {dtype} on {q.device}")
    qs, ldq = _heads(q, "q", dtype, device)
    rows, hq, d = qs
    if q_out is None:
        q_out = torch.empty(qs, dtype=dtype, device=q.device)
    qos, ldqo = (qs, ldq) if q_out is q else _heads(q_out, "q_out", dtype, device)
    hk = ldk = ldko = 0
    if k is not None:
        ks, ldk = _heads(k, "k", dtype, device)
        if ks[0] != rows or ks[2] != d:
            raise ValueError("k: one row per row of q, heads of the same size")
        if k_out is None:
            k_out = torch.empty(ks, dtype=dtype, device=q.device)
        kos, ldko = (ks, ldk) if k_out is k else _heads(k_out, "k_out", dtype, device)
        hk = ks[1]
        if kos != ks:
            raise ValueError("k_out: the shape of k")
    elif k_out is not None:
        raise ValueError("k_out goes with k")
    if qos != qs:
        raise ValueError("q_out: the shape of q")
    for g, n in ((q_gain, "q_gain"), (k_gain, "k_gain")):
        if g is not None and (g.dtype is not dtype or g.shape != (d,) or not g.is_contiguous() or g.get_device() != device):
            raise ValueError(f"{n}: expected a contiguous {dtype} vector of {d} on cuda:{device}")
    rot = 0
    if positions is not None and inv_freq is not None:
        if positions.dtype is not torch.int32 or positions.shape != (rows,) or not positions.is_contiguous() or \
                positions.get_device() != device:
            raise ValueError(f"positions: expected a contiguous int32 vector of {rows} on cuda:{device}")
        if inv_freq.dtype is not torch.float64 or inv_freq.dim() != 1 or not inv_freq.is_contiguous() or \
                inv_freq.get_device() != device:
            raise ValueError(f"inv_freq: expected a contiguous float64 vector on cuda:{device}")
        rot = 2 * inv_freq.numel()
    elif positions is not inv_freq:
        raise ValueError("positions and inv_freq: both or neither")
    if eps is not None and not eps >= 0:
        raise ValueError("eps must not be negative")
    flags = (BCTM_HEAD_NORM if eps is not None else 0) | (BCTM_ROPE_INTERLEAVED if interleaved else 0)
    st = _launch(mlib().bctm_qk_norm_rope, q.device, q.data_ptr(), q_out.data_ptr(), _dptr(q_gain), hq, ldq, ldqo, _dptr(k),
                 _dptr(k_out), _dptr(k_gain), hk, ldk, ldko, _dptr(positions), _dptr(inv_freq), rot, rows, d, eps or 0.0,
                 binding.BCT_F32 if dtype is torch.float32 else binding.BCT_BF16, flags)
    _ck(st, "bctm_qk_norm_rope")
    return q_out, k_out


class PackedWeight:
    """A weight matrix [N][K] in the tiled layout bctm_linear / bctm_swiglu stream (bctm_pack_weight)."""

    def __init__(self, data, N, K):
        self.data, self.N, self.K = data, N, K


def bctm_pack_weight(*ws):
    """One or more matrices [N_i][K] -> one PackedWeight of sum N_i features, matrix after matrix."""
    torch = _torch()
    for w in ws:
        _bf16_2d(w, "w", ws[0].shape[1])
    K = ws[0].shape[1]
    N = sum(w.shape[0] for w in ws)
    data = torch.empty(N * K, dtype=torch.bfloat16, device=ws[0].device)
    off = 0
    for w in ws:
        _ck(_launch(mlib().bctm_pack_weight, ws[0].device, _dptr(w), _dptr(data[off:]), w.shape[0], K), "bctm_pack_weight")
        off += w.shape[0] * K
    return PackedWeight(data, N, K)


def _packed(w, name, K):
    if not isinstance(w, PackedWeight):
        raise ValueError(f"{name}: expected a PackedWeight (bctm_pack_weight)")
    if w.K != K:
        raise ValueError(f"{name}: packed for {w.K} inputs, x has {K}")


def _x_arg(x):
    """-> (data tensor, rows, K, flag) of a row-major tensor or a TiledRows."""
    if isinstance(x, TiledRows):
        return x.data, x.rows, x.K, BCTM_X_TILED
    _bf16_2d(x, "x")
    return x, x.shape[0], x.shape[1], 0


def _linear_args(x, w, residual, out):
    torch = _torch()
    xd, rows, K, xf = _x_arg(x)
    _packed(w, "w", K)
    N = w.N
    if out is None:
        out = torch.empty((rows, N), dtype=torch.bfloat16, device=xd.device)
    _bf16_2d(out, "out", N)
    if residual is not None:
        _bf16_2d(residual, "residual", N)
    if out.shape[0] != rows or (residual is not None and residual.shape[0] != rows):
        raise ValueError("out / residual: one row per row of x")
    return out, (xd.device, _dptr(xd), _dptr(w.data), _dptr(residual), _dptr(out), rows, K, N, xf)


def bctm_linear(x, w, residual=None, out=None):
    """x: a [rows][K] tensor or a TiledRows; out / residual row-major [rows][N]."""
    out, args = _linear_args(x, w, residual, out)
    _ck(_launch(mlib().bctm_linear, *args), "bctm_linear")
    return out


def _split_args(x, w, outs):
    xd, rows, K, xf = _x_arg(x)
    _packed(w, "w", K)
    if len(outs) not in (2, 3) or sum(o.shape[1] for o in outs) != w.N:
        raise ValueError("outs: two or three tensors whose widths add up to the weight's features")
    for o in outs:
        _bf16_2d(o, "out")
        if o.shape[0] != rows:
            raise ValueError("outs: one row per row of x")
    o2, n2 = (outs[2], outs[2].shape[1]) if len(outs) == 3 else (None, 0)
    return (xd.device, _dptr(xd), _dptr(w.data), _dptr(outs[0]), outs[0].shape[1], _dptr(outs[1]), outs[1].shape[1], _dptr(o2), n2,
            rows, K, xf)


def bctm_linear_split(x, w, outs):
    """One projection into two or three row-major outputs whose widths add up to w.N."""
    _ck(_launch(mlib().bctm_linear_split, *_split_args(x, w, outs)), "bctm_linear_split")
    return outs


def _swiglu_args(x, w_gate, w_up, out, tiled):
    torch = _torch()
    xd, rows, K, xf = _x_arg(x)
    _packed(w_gate, "w_gate", K)
    _packed(w_up, "w_up", K)
    if w_gate.N != w_up.N:
        raise ValueError("w_gate and w_up: same shape")
    N = w_gate.N
    if tiled:
        if out is None:
            out = TiledRows(rows, N, xd.device)
        if not isinstance(out, TiledRows) or (out.rows, out.K) != (rows, N):
            raise ValueError("out: a TiledRows [rows][N]")
        dst = out.data
    else:
        if out is None:
            out = torch.empty((rows, N), dtype=torch.bfloat16, device=xd.device)
        _bf16_2d(out, "out", N)
        if out.shape[0] != rows:
            raise ValueError("out: one row per row of x")
        dst = out
    return out, (xd.device, _dptr(xd), _dptr(w_gate.data), _dptr(w_up.data), _dptr(dst), rows, K, N,
                 xf | (BCTM_OUT_TILED if tiled else 0))


def bctm_swiglu(x, w_gate, w_up, out=None, tiled=False):
    """x: a [rows][K] tensor or a TiledRows; out: a [rows][N] tensor, or (tiled=True) a TiledRows."""
    out, args = _swiglu_args(x, w_gate, w_up, out, tiled)
    _ck(_launch(mlib().bctm_swiglu, *args), "bctm_swiglu")
    return out


class LoraWeights:
    """The low-rank adapters of one projection, packed (bctm_lora_pack): n of them, each rank x K per segment and N x rank."""

    def __init__(self, a, b, b_up, scale, n, segments, rank, K, N, used=0):
        self.a, self.b, self.b_up, self.scale = a, b, b_up, scale
        self.n, self.segments, self.rank, self.K, self.N = n, segments, rank, K, N
        self.used = used   # of rank: those the adapters had before they were filled up (0: all)
        self._sizes = {}   # rows -> bytes of workspace

    def workspace_bytes(self, rows):
        if rows not in self._sizes:
            v = ctypes.c_size_t(0)
            _ck(mlib().bctm_lora_workspace(rows, self.K, self.rank, self.segments, ctypes.byref(v)), "bctm_lora_workspace")
            if len(self._sizes) >= 64:   # of row counts that come and go
                self._sizes.clear()
            self._sizes[rows] = v.value
        return self._sizes[rows]


def bctm_lora_pack(a, b, scale=None):
    """n adapters of one projection -> LoraWeights.  a [n][rank][K], or [n][segments][rank][K] where every output of a split (or
    the gate and the up matrix of a SwiGLU) has its own; b [n][N][rank], or for a SwiGLU the pair (gate's, up's), bf16; a list
    of one tensor is that tensor.  scale float32 [n] or None = 1.  Any rank to 256: filled up with zeros to a multiple of 16."""
    torch = _torch()
    bs = list(b) if isinstance(b, (list, tuple)) else [b]
    if a.dim() == 3:
        a = a[:, None]
    if a.dim() != 4 or a.dtype != torch.bfloat16 or not a.is_cuda or len(bs) not in (1, 2):
        raise ValueError("a: expected bf16 [n][rank][K] or [n][segments][rank][K] on the GPU; b: one tensor or two")
    n, segments, rank, K = a.shape
    for t in bs:
        if t.dtype != torch.bfloat16 or t.dim() != 3 or t.device != a.device or t.shape != (n, bs[0].shape[1], rank):
            raise ValueError(f"b: expected bf16 [{n}][N][{rank}] on {a.device}, got {t.dtype} {tuple(t.shape)} on {t.device}")
    if len(bs) == 2 and segments != 2:
        raise ValueError("a: two segments for a SwiGLU, the gate's and the up matrix's")
    if scale is not None and (scale.dtype != torch.float32 or scale.shape != (n,) or not scale.is_contiguous() or
                              scale.device != a.device):
        raise ValueError(f"scale: expected a contiguous float32 vector of {n} on {a.device}")
    N, r = bs[0].shape[1], (rank + 15) // 16 * 16
    if max(n * segments * r, n * N, K) >> 32:
        raise ValueError("more adapters than one call packs")
    if r != rank:
        a = torch.nn.functional.pad(a, (0, 0, 0, r - rank))
        bs = [torch.nn.functional.pad(t, (0, r - rank)) for t in bs]
    pa = bctm_pack_weight(a.reshape(n * segments * r, K).contiguous()).data
    packed = []
    for t in bs:
        t = t.contiguous()
        p = torch.empty(n * N * r, dtype=torch.bfloat16, device=a.device)
        _ck(_launch(mlib().bctm_lora_pack, a.device, _dptr(t), _dptr(p), n * N, r), "bctm_lora_pack")
        packed.append(p)
    return LoraWeights(pa, packed[0], packed[1] if len(packed) == 2 else None, scale, n, segments, r, K, N, rank)


def _lora_arg(lora, ids, workspace, device, rows, K, N, segments, swiglu):
    torch = _torch()
    if not isinstance(lora, LoraWeights):
        raise ValueError("lora: expected LoraWeights (bctm_lora_pack)")
    if lora.K != K or lora.N != N or lora.segments != segments or (lora.b_up is not None) != swiglu or lora.a.device != device:
        raise ValueError(f"lora: packed for {lora.K} -> {lora.N} in {lora.segments} segments on {lora.a.device}, the projection is "
                         f"{K} -> {N} in {segments} on {device}")
    if ids.dtype is not torch.int32 or ids.shape != (rows,) or not ids.is_contiguous() or ids.device != device:
        raise ValueError(f"ids: expected a contiguous int32 vector of {rows} on {device}")
    if workspace is None:
        workspace = torch.empty(lora.workspace_bytes(rows), dtype=torch.uint8, device=device)
    elif workspace.dtype is not torch.uint8 or not workspace.is_contiguous() or workspace.device != device:
        raise ValueError(f"workspace: expected contiguous torch.uint8 on {device}")
    # read by the call, which the second value outlives
    return _bctm_lora(lora.a.data_ptr(), lora.b.data_ptr(), _dptr(lora.b_up), _dptr(lora.scale), ids.data_ptr(), lora.n, lora.rank,
                      workspace.data_ptr(), workspace.numel(), lora.used), workspace


def bctm_linear_lora(x, w, lora, ids, residual=None, out=None, workspace=None):
    """bctm_linear with the adapter ids[r] (int32, none where outside lora's) added to row r.  workspace: torch.uint8 of
    lora.workspace_bytes(rows), or None to take one from torch for this call."""
    out, args = _linear_args(x, w, residual, out)
    l, keep = _lora_arg(lora, ids, workspace, args[0], args[5], args[6], args[7], 1, False)
    _ck(_launch(mlib().bctm_linear_lora, *args, ctypes.byref(l)), "bctm_linear_lora")
    return out


def bctm_linear_split_lora(x, w, lora, ids, outs, workspace=None):
    """bctm_linear_split with adapters: lora has a segment for each output."""
    args = _split_args(x, w, outs)
    l, keep = _lora_arg(lora, ids, workspace, args[0], args[9], args[10], w.N, len(outs), False)
    _ck(_launch(mlib().bctm_linear_split_lora, *args, ctypes.byref(l)), "bctm_linear_split_lora")
    return outs


def bctm_swiglu_lora(x, w_gate, w_up, lora, ids, out=None, tiled=False, workspace=None):
    """bctm_swiglu with adapters of both matrices."""
    out, args = _swiglu_args(x, w_gate, w_up, out, tiled)
    l, keep = _lora_arg(lora, ids, workspace, args[0], args[5], args[6], args[7], 2, True)
    _ck(_launch(mlib().bctm_swiglu_lora, *args, ctypes.byref(l)), "bctm_swiglu_lora")
    return out


def bctm_linear_act(x, w, bias=None, act="none", residual=None, out=None, out_dtype=None, tiled=False):
    """residual + act(x W^T + bias).  x: a [rows][K] tensor or a TiledRows; bias bf16 [N]; act: a name of BCTM_ACTS; residual bf16
    [rows][N]; out [rows][N] of bf16 or float32 (out_dtype where it is made here), or (tiled=True) a TiledRows."""
    torch = _torch()
    xd, rows, K, xf = _x_arg(x)
    _packed(w, "w", K)
    N, device = w.N, xd.device
    if act not in BCTM_ACTS:
        raise ValueError(f"act: expected one of {tuple(BCTM_ACTS)}, got {act!r}")
    if w.data.device != device:
        raise ValueError(f"w: packed on {w.data.device}, x is on {device}")
    if bias is not None and (bias.dtype is not torch.bfloat16 or bias.shape != (N,) or not bias.is_contiguous() or bias.device != device):
        raise ValueError(f"bias: expected a contiguous bf16 vector of {N} on {device}")
    if residual is not None:
        _bf16_2d(residual, "residual", N)
        if residual.shape[0] != rows or residual.device != device:
            raise ValueError("residual: one row per row of x, on its device")
    if tiled:
        if out is None and out_dtype in (None, torch.bfloat16):
            out = TiledRows(rows, N, device)
        if not isinstance(out, TiledRows) or (out.rows, out.K) != (rows, N) or out.data.device != device:
            raise ValueError("out: a TiledRows [rows][N] on x's device")
        dst, of = out.data, BCTM_OUT_TILED
    else:
        if out is None:
            out = torch.empty((rows, N), dtype=out_dtype or torch.bfloat16, device=device)
        if not isinstance(out, torch.Tensor) or out.dtype not in (torch.bfloat16, torch.float32) or (out_dtype or out.dtype) != out.dtype \
                or out.shape != (rows, N) or not out.is_contiguous() or out.device != device:
            raise ValueError(f"out: expected contiguous bf16 or float32 [{rows}][{N}] on {device}")
        dst, of = out, BCTM_OUT_F32 if out.dtype is torch.float32 else 0
    _ck(_launch(mlib().bctm_linear_act, device, xd.data_ptr(), w.data.data_ptr(), _dptr(bias), _dptr(residual), dst.data_ptr(), rows, K, N,
                BCTM_ACTS[act], xf | of), "bctm_linear_act")
    return out


class ExpertPlan:
    """The pairs of rows tokens and their k slots (number token * k + slot) by expert: order int32 [rows * k], offsets int32
    [n_experts + 1], views of the plan; made by bctm_route or bctm_expert_plan."""

    def __init__(self, rows, k, n_experts, device):
        torch = _torch()
        size, order = ctypes.c_size_t(0), ctypes.c_size_t(0)
        if rows >> 32:
            raise ValueError("more tokens than one call takes")
        _ck(mlib().bctm_expert_plan_bytes(rows, k, n_experts, ctypes.byref(size), ctypes.byref(order)), "bctm_expert_plan_bytes")
        self.rows, self.k, self.n_experts, self.bytes = rows, k, n_experts, size.value
        # zeros, not empty: a plan that has not been made has no tokens
        self.data = torch.zeros(size.value // 4, dtype=torch.int32, device=device)
        self.offsets = self.data[:n_experts + 1]
        self.order = self.data[order.value:order.value + rows * k]


def _plan(plan, rows, k, n_experts, device):
    if not isinstance(plan, ExpertPlan) or (plan.rows, plan.k, plan.n_experts) != (rows, k, n_experts) or plan.data.device != device:
        raise ValueError(f"plan: expected an ExpertPlan of {rows} tokens, {k} slots and {n_experts} experts on {device}")


def bctm_route(logits, k, bias=None, sigmoid=False, normalise=True, scale=1.0, experts=None, weights=None, plan=None):
    """Each token's k experts from its logits [rows][n_experts] (float32 or bf16, rows at any distance): those with the largest
    logit, or with bias (float32 [n_experts]) the largest score + bias; scores are the logits' softmax or sigmoid.
    -> (experts int32 [rows][k], weights float32 [rows][k]: scale * score, normalised over the chosen ones, plan: an ExpertPlan,
    made here unless given).  Slots for which no expert is left have -1 and 0."""
    torch = _torch()
    if logits.dtype not in (torch.float32, torch.bfloat16) or logits.dim() != 2 or not logits.is_cuda or \
            (logits.stride(1) != 1 and logits.shape[1] > 1) or logits.shape[0] >> 32:
        raise ValueError(f"logits: expected [rows][n_experts] of float32 or bf16 on the GPU, each row contiguous, got {logits.dtype} "
                         f"{tuple(logits.shape)} strides {logits.stride()} on {logits.device}")
    (rows, E), device = logits.shape, logits.device
    if plan is None:
        plan = ExpertPlan(rows, k, E, device)
    _plan(plan, rows, k, E, device)
    if experts is None:
        experts = torch.empty((rows, k), dtype=torch.int32, device=device)
    if weights is None:
        weights = torch.empty((rows, k), dtype=torch.float32, device=device)
    for t, n, dtype, shape in ((experts, "experts", torch.int32, (rows, k)), (weights, "weights", torch.float32, (rows, k)),
                               (bias, "bias", torch.float32, (E,))):
        if t is not None and (t.dtype is not dtype or t.shape != shape or not t.is_contiguous() or t.device != device):
            raise ValueError(f"{n}: expected contiguous {dtype} {shape} on {device}")
    _ck(_launch(mlib().bctm_route, device, logits.data_ptr(), logits.stride(0) if rows > 1 else max(logits.stride(0), E), _dptr(bias),
                experts.data_ptr(), weights.data_ptr(), plan.data.data_ptr(), plan.bytes, rows, E, k, scale,
                binding.BCT_F32 if logits.dtype is torch.float32 else binding.BCT_BF16,
                (BCTM_ROUTE_SIGMOID if sigmoid else 0) | (BCTM_ROUTE_NORMALISE if normalise else 0)), "bctm_route")
    return experts, weights, plan


def bctm_expert_plan(experts, n_experts, plan=None):
    """The plan of experts int32 [rows][k] that the caller chose (outside [0, n_experts): none)."""
    torch = _torch()
    if experts.dtype is not torch.int32 or experts.dim() != 2 or not experts.is_contiguous() or not experts.is_cuda:
        raise ValueError(f"experts: expected contiguous int32 [rows][k] on the GPU, got {experts.dtype} {tuple(experts.shape)} on {experts.device}")
    rows, k = experts.shape
    if plan is None:
        plan = ExpertPlan(rows, k, n_experts, experts.device)
    _plan(plan, rows, k, n_experts, experts.device)
    _ck(_launch(mlib().bctm_expert_plan, experts.device, experts.data_ptr(), plan.data.data_ptr(), plan.bytes, rows, n_experts, k),
        "bctm_expert_plan")
    return plan


class ExpertWeights:
    """The matrices [n][N][K] of all experts, packed (bctm_pack_experts)."""

    def __init__(self, data, n, N, K):
        self.data, self.n, self.N, self.K = data, n, N, K


def bctm_pack_experts(w):
    """w bf16 [n_experts][N][K] -> ExpertWeights."""
    torch = _torch()
    if w.dtype is not torch.bfloat16 or w.dim() != 3 or not w.is_contiguous() or not w.is_cuda:
        raise ValueError(f"w: expected contiguous bf16 [n_experts][N][K] on the GPU, got {w.dtype} {tuple(w.shape)} on {w.device}")
    n, N, K = w.shape
    if N % 16 or K % 32:
        raise ValueError("N must be a multiple of 16 and K of 32")
    return ExpertWeights(bctm_pack_weight(w.view(n * N, K)).data, n, N, K)


def _expert_args(x, w, name, plan, rows):
    if not isinstance(plan, ExpertPlan):
        raise ValueError("plan: expected an ExpertPlan")
    _bf16_2d(x, "x")
    if not isinstance(w, ExpertWeights) or w.K != x.shape[1] or w.n != plan.n_experts or w.data.device != x.device:
        raise ValueError(f"{name}: expected ExpertWeights of {plan.n_experts} experts and {x.shape[1]} inputs on {x.device} (bctm_pack_experts)")
    if x.shape[0] != rows or plan.data.device != x.device:
        raise ValueError(f"x: expected {rows} rows for this plan, on its device")


def bctm_expert_swiglu(x, w_gate, w_up, plan, out=None):
    """x bf16 [rows][K] -> [rows * k][N]: the gated product of each token with each of its experts, row token * k + slot; rows of
    slots without an expert are left as they were (0 where out is made here)."""
    torch = _torch()
    _expert_args(x, w_gate, "w_gate", plan, plan.rows if isinstance(plan, ExpertPlan) else 0)
    _expert_args(x, w_up, "w_up", plan, plan.rows)
    if w_gate.N != w_up.N:
        raise ValueError("w_gate and w_up: same shape")
    if out is None:
        out = torch.zeros((plan.rows * plan.k, w_gate.N), dtype=torch.bfloat16, device=x.device)
    _bf16_2d(out, "out", w_gate.N)
    if out.shape[0] != plan.rows * plan.k or out.device != x.device:
        raise ValueError("out: one row per token and slot, on x's device")
    _ck(_launch(mlib().bctm_expert_swiglu, x.device, x.data_ptr(), w_gate.data.data_ptr(), w_up.data.data_ptr(), out.data_ptr(),
                plan.data.data_ptr(), plan.rows, plan.k, plan.n_experts, w_gate.K, w_gate.N), "bctm_expert_swiglu")
    return out


def bctm_expert_tile(rows, k, n_experts, K, N, swiglu):
    """(pairs, features) that the launch of this shape gives one workgroup."""
    v = [ctypes.c_uint32(0) for _ in range(2)]
    _ck(mlib().bctm_expert_tile(rows, k, n_experts, K, N, 1 if swiglu else 0, *(ctypes.byref(a) for a in v)), "bctm_expert_tile")
    return tuple(a.value for a in v)


def bctm_expert_workspace(rows, k, N):
    """Bytes of workspace that bctm_expert_linear takes."""
    v = ctypes.c_size_t(0)
    _ck(mlib().bctm_expert_workspace(rows, k, N, ctypes.byref(v)), "bctm_expert_workspace")
    return v.value


def bctm_expert_linear(h, w, plan, weights, residual=None, out=None, workspace=None):
    """h bf16 [rows * k][K], weights float32 [rows][k] -> [rows][N]: residual + the weighted sum of each token's products with its
    experts.  out may be the residual.  workspace: torch.uint8 of bctm_expert_workspace bytes, or None to take one from torch."""
    torch = _torch()
    _expert_args(h, w, "w", plan, plan.rows * plan.k if isinstance(plan, ExpertPlan) else 0)
    rows, k, N, device = plan.rows, plan.k, w.N, h.device
    if weights.dtype is not torch.float32 or weights.shape != (rows, k) or not weights.is_contiguous() or weights.device != device:
        raise ValueError(f"weights: expected contiguous float32 [{rows}][{k}] on {device}")
    if out is None:
        out = torch.empty((rows, N), dtype=torch.bfloat16, device=device)
    for t, n in ((out, "out"), (residual, "residual")):
        if t is not None:
            _bf16_2d(t, n, N)
            if t.shape[0] != rows or t.device != device:
                raise ValueError(f"{n}: one row per token, on h's device")
    if workspace is None:
        workspace = torch.empty(bctm_expert_workspace(rows, k, N), dtype=torch.uint8, device=device)
    elif workspace.dtype is not torch.uint8 or not workspace.is_contiguous() or workspace.device != device:
        raise ValueError(f"workspace: expected contiguous torch.uint8 on {device}")
    _ck(_launch(mlib().bctm_expert_linear, device, h.data_ptr(), w.data.data_ptr(), plan.data.data_ptr(), weights.data_ptr(), _dptr(residual),
                out.data_ptr(), workspace.data_ptr(), workspace.numel(), rows, k, plan.n_experts, w.K, N), "bctm_expert_linear")
    return out


def bctm_argmax(logits, out=None):
    torch = _torch()
    _bf16_2d(logits, "logits")
    if out is None:
        out = torch.empty(logits.shape[0], dtype=torch.int32, device=logits.device)
    if out.dtype != torch.int32 or tuple(out.shape) != (logits.shape[0],) or not out.is_contiguous():
        raise ValueError("out: a contiguous int32 vector, one entry per row")
    _ck(_launch(mlib().bctm_argmax, logits.device, _dptr(logits), _dptr(out), logits.shape[0], logits.shape[1]), "bctm_argmax")
    return out


def bctm_sample(logits, uniform, temperature=None, top_k=None, top_p=None, min_p=None, out=None, prob=None):
    """Draws a token from each row of logits [rows][N] (float32 or bf16, rows at any distance) with its uniform number, float32
    [rows] in [0, 1), and its settings: temperature, top_p, min_p float32 [rows], top_k int32 [rows], None = off.
    -> (ids int32 [rows], prob): prob the probability of each drawn token among those kept, into a float32 [rows] given or
    made (True), else None."""
    torch = _torch()
    if logits.dtype not in (torch.float32, torch.bfloat16) or logits.dim() != 2 or not logits.is_cuda or \
            (logits.stride(1) != 1 and logits.shape[1] > 1):
        raise ValueError(f"logits: expected [rows][N] of float32 or bf16 on the GPU, each row contiguous, got {logits.dtype} "
                         f"{tuple(logits.shape)} strides {logits.stride()} on {logits.device}")
    rows, N = logits.shape
    if rows >> 32 or N >> 32:
        raise ValueError("logits: more rows or tokens than one call takes")
    if out is None:
        out = torch.empty(rows, dtype=torch.int32, device=logits.device)
    if prob is True:
        prob = torch.empty(rows, dtype=torch.float32, device=logits.device)
    f32, i32 = torch.float32, torch.int32
    for t, n, want in ((uniform, "uniform", f32), (temperature, "temperature", f32), (top_k, "top_k", i32), (top_p, "top_p", f32),
                       (min_p, "min_p", f32), (out, "out", i32), (prob, "prob", f32)):
        if t is not None and (t.dtype is not want or t.shape != (rows,) or not t.is_contiguous() or t.device != logits.device):
            raise ValueError(f"{n}: expected a contiguous {want} vector of {rows} on {logits.device}")
    _ck(_launch(mlib().bctm_sample, logits.device, _dptr(logits), logits.stride(0) if rows > 1 else max(logits.stride(0), N),
                _dptr(temperature), _dptr(top_k), _dptr(top_p), _dptr(min_p), _dptr(uniform), _dptr(out), _dptr(prob), rows, N,
                binding.BCT_F32 if logits.dtype is f32 else binding.BCT_BF16), "bctm_sample")
    return out, prob


# ------------------------------------------------------------------ the stack


@dataclass(frozen=True)
class StackShape:
    """A Llama-shaped decoder whose attention layers are bounded caches (section 3.2)."""
    n_layers: int
    dim: int            # model width
    n_q_heads: int
    n_kv_heads: int
    head_dim: int
    ffn: int            # SwiGLU hidden width
    vocab: int
    capacity_M: int
    batch: int
    eps: float = 1e-5
    head_norm: bool = False       # queries and write queries normalised head by head (weights q_norm and wq_norm)
    rope_base: float = 0.0        # > 0: turned by their token's position, inv_freq[j] = rope_base ** (-2 j / rotary_dim)
    rotary_dim: int = 0           # how much of each head is turned (0: all of it)
    rope_interleaved: bool = False
    n_experts: int = 0            # > 0: experts of width ffn in place of the dense MLP, experts_per_token of them for each token
    experts_per_token: int = 0
    router_sigmoid: bool = False  # scores are the logits' sigmoids, not their softmax
    router_bias: bool = False     # a weight router_bias is added to the scores for the choice (not for the weights)
    router_normalise: bool = True
    router_scale: float = 1.0
    shared_ffn: int = 0           # > 0: beside its experts every token goes through a dense SwiGLU of that width

    def __post_init__(self):
        if self.n_experts and (not 1 <= self.experts_per_token <= min(16, self.n_experts) or self.n_experts > 512 or self.shared_ffn % 32):
            raise ValueError("experts_per_token must be 1 to 16 of at most 512 experts, shared_ffn a multiple of 32")
        if not math.isfinite(ctypes.c_float(self.router_scale).value):
            raise ValueError("router_scale must be finite in float32")
        if not self.n_experts and (self.experts_per_token or self.router_sigmoid or self.router_bias or self.shared_ffn):
            raise ValueError("experts_per_token, router_sigmoid, router_bias and shared_ffn go with n_experts")
        if (self.head_norm or self.rope_base) and (self.head_dim % 16 or self.rotary_dim % 16 or
                                                   not 0 <= self.rotary_dim <= self.head_dim or self.rope_base < 0):
            raise ValueError("head_dim and rotary_dim must be multiples of 16, rotary_dim at most head_dim, rope_base not negative")
        if self.dim % 32 or (self.n_q_heads * self.head_dim) % 32 or self.ffn % 32 or self.vocab % 16 or \
                (self.n_kv_heads * self.head_dim) % 16:
            raise ValueError("dim, n_q_heads * head_dim and ffn must be multiples of 32; vocab and "
                             "n_kv_heads * head_dim multiples of 16")

    @property
    def q_width(self):
        return self.n_q_heads * self.head_dim

    @property
    def kv_width(self):
        return self.n_kv_heads * self.head_dim

    def weight_shapes(self):
        """name -> shape of every per-layer weight, in the order load_layer expects."""
        E = (self.n_experts,) if self.n_experts else ()
        shapes = {"attn_norm": (self.dim,), "w_q": (self.q_width, self.dim), "w_wq": (self.kv_width, self.dim),
                  "w_wv": (self.kv_width, self.dim), "w_o": (self.dim, self.q_width), "mlp_norm": (self.dim,),
                  "w_gate": (*E, self.ffn, self.dim), "w_up": (*E, self.ffn, self.dim), "w_down": (*E, self.dim, self.ffn),
                  **({"q_norm": (self.head_dim,), "wq_norm": (self.head_dim,)} if self.head_norm else {})}
        if E:
            shapes["w_router"] = (self.n_experts, self.dim)
            if self.router_bias:
                shapes["router_bias"] = (self.n_experts,)
            if self.shared_ffn:
                shapes.update(w_shared_gate=(self.shared_ffn, self.dim), w_shared_up=(self.shared_ffn, self.dim),
                              w_shared_down=(self.dim, self.shared_ffn))
        return shapes

    def weight_bytes(self):
        per_layer = sum(math.prod(s) for s in self.weight_shapes().values())
        return 2 * (self.n_layers * per_layer + 2 * self.vocab * self.dim + self.dim)


@dataclass
class Sampling:
    """How each row of logits gets its next token (bctm_sample): device vectors of one entry a row, None = off.  They are read
    when the step runs, so a captured step takes what they hold at each replay."""
    uniform: object
    temperature: object = None
    top_k: object = None
    top_p: object = None
    min_p: object = None
    prob: object = None       # receives the drawn tokens' probabilities


class BctStack:
    """Token ids in, next ids out (greedy, or drawn): embedding, n_layers x (RMSNorm, W_q / W_wq / W_wv,
    bounded-cache attention, W_o + residual, RMSNorm, SwiGLU MLP + residual), RMSNorm, output head, arg-max.

    weights: {"embed": [vocab][dim], "final_norm": [dim], "head": [vocab][dim],
              "layers": [ {name: tensor} per layer, names of StackShape.weight_shapes() ],
              "keys": [ MK per layer, [Hkv][M][d] ]}  -- all bf16 device tensors, but router_bias may be float32 (its steps
              decide between scores closer than bf16 tells apart).
    With shape.head_norm and / or shape.rope_base, q and wq pass bctm_qk_norm_rope before the cache.
    With shape.n_experts each token's MLP is that of the experts a router chooses for it (bctm_linear_act, bctm_route,
    bctm_expert_swiglu, bctm_expert_linear), beside a shared one with shape.shared_ffn.
    """

    def __init__(self, shape: StackShape, weights, max_prefill_T=0, device="cuda:0"):
        torch = _torch()
        self.shape = shape
        self.device = torch.device(device)
        s = shape
        self.caches = []
        ws = None
        for l in range(s.n_layers):
            c = BctCache(s.capacity_M, s.batch, s.n_q_heads, s.n_kv_heads, s.head_dim, torch.bfloat16,
                         max_prefill_T=max_prefill_T, device=device, workspace=ws)
            ws = c._workspace          # one stream steps the layers in turn: they share the workspace
            c.set_keys(weights["keys"][l])
            c.set_values(None)
            self.caches.append(c)
        # matrices are repacked once into the streaming layout; the row-major copies are not kept
        self.layers = []
        for l, lw in enumerate(weights["layers"]):
            pl = {}
            for n, shp in s.weight_shapes().items():
                types = (torch.float32, torch.bfloat16) if n == "router_bias" else (torch.bfloat16,)
                if tuple(lw[n].shape) != shp or lw[n].dtype not in types:
                    raise ValueError(f"layer {l} {n}: expected {' or '.join(str(t) for t in types)} {shp}")
                if n == "router_bias":
                    pl[n] = lw[n].float().contiguous()
                elif len(shp) == 1:
                    pl[n] = lw[n]
                elif len(shp) == 3:
                    pl[n] = bctm_pack_experts(lw[n])
                elif n == "w_router":   # features are packed by 16, and a multiple of 64 has a kernel of its own
                    pl[n] = bctm_pack_weight(torch.nn.functional.pad(lw[n], (0, 0, 0, -shp[0] % 64)))
                elif n not in ("w_q", "w_wq", "w_wv"):
                    pl[n] = bctm_pack_weight(lw[n])
            # the three projections of the attention input run as one launch with three outputs
            pl["w_qkv"] = bctm_pack_weight(lw["w_q"], lw["w_wq"], lw["w_wv"])
            self.layers.append(pl)
        self.embed, self.final_norm = weights["embed"], weights["final_norm"]
        self.head = bctm_pack_weight(weights["head"])
        self.adapters = None
        self._lora_now = {}   # rows -> the workspace that the present adapters take
        self.inv_freq = None
        if s.rope_base:
            rot = s.rotary_dim or s.head_dim
            self.inv_freq = torch.tensor([s.rope_base ** (-2.0 * j / rot) for j in range(rot // 2)], dtype=torch.float64,
                                         device=self.device)
        self._bufs = {}

    def set_adapters(self, layers):
        """layers: per layer a dictionary of LoraWeights for any of "qkv" (three segments: q, wq, wv), "o", "gate_up" and "down";
        forward(adapters=) then says which adapter a row has.  None: no adapters.  A graph that was captured before goes on with
        the adapters of then, which the caller keeps as long as it is replayed; capture again for the new ones."""
        if layers is not None:
            if len(layers) != self.shape.n_layers:
                raise ValueError(f"adapters: expected {self.shape.n_layers} layers")
            s = self.shape
            want = {"qkv": (s.dim, s.q_width + 2 * s.kv_width, 3, False), "o": (s.q_width, s.dim, 1, False)}
            if not s.n_experts:   # experts have no adapters
                want.update(gate_up=(s.dim, s.ffn, 2, True), down=(s.ffn, s.dim, 1, False))
            for l, d in enumerate(layers):
                for n, a in d.items():
                    if n not in want or not isinstance(a, LoraWeights) or (a.K, a.N, a.segments, a.b_up is not None) != want[n] \
                            or a.a.device != self.embed.device:
                        raise ValueError(f"layer {l} {n}: expected LoraWeights of (K, N, segments) {want.get(n, tuple(want))[:3]} "
                                         f"on {self.embed.device}")
        # a dictionary that changes afterwards would go past the checks
        self.adapters = None if layers is None else [dict(d) for d in layers]
        self._lora_now.clear()

    def _lora_workspace(self, rows):
        torch = _torch()
        if rows not in self._lora_now:
            n = max([a.workspace_bytes(rows) for d in self.adapters for a in d.values()], default=16)
            # Other adapters' workspace of as many rows serves, if it is large enough.  One that is not stays all the same: a step on
            # another stream may be using it, and a captured one will.
            kept = self._bufs.setdefault(("lora", rows), [])
            if not kept or kept[-1].numel() < n:
                kept.append(torch.empty(n, dtype=torch.uint8, device=self.device))
            self._lora_now[rows] = kept[-1]
        return self._lora_now[rows]

    def _buf(self, name, rows, cols):
        torch = _torch()
        k = (name, rows, cols)
        if k not in self._bufs:
            self._bufs[k] = torch.empty((rows, cols), dtype=torch.bfloat16, device=self.device)
        return self._bufs[k]

    def _shared(self, name, n, dtype):
        """n values that calls of any number of rows share, so that prompts of many lengths do not keep a buffer each.  One that has become
        too small stays with the calls that have it, as a captured step has its address; each is twice the one before it at least, so all
        together are four times the largest call's at most."""
        kept = self._bufs.setdefault(("shared", name), [])
        if not kept or kept[-1].numel() < n:
            kept.append(_torch().empty(max(n, 2 * kept[-1].numel()) if kept else n, dtype=dtype, device=self.device))
        return kept[-1][:n]

    def _tiled(self, name, rows, cols):
        k = ("tiled", name, rows, cols)
        if k not in self._bufs:
            self._bufs[k] = TiledRows(rows, cols, self.device)
        return self._bufs[k]

    def _expert_bufs(self, rows):
        """(logits, experts, weights, plan, workspace, gated rows) of a step of that many rows."""
        torch = _torch()
        s = self.shape
        k = ("experts", rows)
        if k not in self._bufs:   # the layers run one after the other and share them
            dev = self.device
            self._bufs[k] = (torch.empty((rows, (s.n_experts + 63) // 64 * 64), dtype=torch.float32, device=dev),
                             torch.empty((rows, s.experts_per_token), dtype=torch.int32, device=dev),
                             torch.empty((rows, s.experts_per_token), dtype=torch.float32, device=dev),
                             ExpertPlan(rows, s.experts_per_token, s.n_experts, dev),
                             # each pair's products on the way back and its gated ones: far more than the rest
                             self._shared("workspace", bctm_expert_workspace(rows, s.experts_per_token, s.dim), torch.uint8),
                             self._shared("g", rows * s.experts_per_token * s.ffn, torch.bfloat16).view(rows * s.experts_per_token, s.ffn))
        return self._bufs[k]

    def _experts(self, x, lw, rows):
        """x += the experts' (and the shared) MLP of its norm."""
        s = self.shape
        logits, experts, weights, plan, workspace, g = self._expert_bufs(rows)
        h = bctm_rmsnorm(x, lw["mlp_norm"], s.eps, self._buf("h", rows, s.dim))
        bctm_linear_act(h, lw["w_router"], out=logits)
        bctm_route(logits[:, :s.n_experts], s.experts_per_token, lw.get("router_bias"), s.router_sigmoid, s.router_normalise, s.router_scale,
                   experts, weights, plan)
        if s.shared_ffn:
            f = bctm_swiglu(h, lw["w_shared_gate"], lw["w_shared_up"], self._tiled("shared", rows, s.shared_ffn), tiled=True)
            bctm_linear(f, lw["w_shared_down"], x, x)
        bctm_expert_swiglu(h, lw["w_gate"], lw["w_up"], plan, g)
        bctm_expert_linear(g, lw["w_down"], plan, weights, x, x, workspace)

    def forward(self, ids, T=1, next_ids=None, head="all", positions=None, adapters=None, sampling=None):
        """ids int32 [B*T] (sequence-major: row b*T + t) -> (next ids, logits).
        T = 1 is a decode step; T > 1 pushes a chunk of T tokens per sequence through bct_prefill.
        head = "all": logits [B*T][vocab] and next ids [B*T] for every row; head = "last": only for the last
        token of every sequence ([B][vocab], [B]) - what a prompt needs, without a [B*T][vocab] product.
        next_ids: where to write the next tokens (may be ids itself: it is read first, written last).
        positions: int32 [B*T], where each token stands; needed with shape.rope_base, else None.
        adapters: int32 [B*T], each row's adapter of those set_adapters has been given (outside them: none); None: no row has one.
        sampling: a Sampling with one entry per row of logits, or None: the most likely token.
        After the first call of a given (B, T, head), and the first one with adapters, no memory is allocated, so a call can be
        captured in a HIP graph."""
        torch = _torch()
        s = self.shape
        rows = s.batch * T
        if ids.numel() != rows:
            raise ValueError(f"ids: expected {rows} entries")
        if head not in ("all", "last"):
            raise ValueError('head: "all" or "last"')
        if (positions is not None) != bool(s.rope_base):
            raise ValueError("positions go with a shape that has a rope_base")
        if adapters is not None and self.adapters is None:
            raise ValueError("adapters: none have been set (set_adapters)")
        # here, as the caches take the step's tokens layer by layer: a call that is refused has changed nothing
        i32, f32, dev = torch.int32, torch.float32, self.embed.device
        checks = [(positions, "positions", i32, rows), (adapters, "adapters", i32, rows)]
        if sampling is not None:
            n = s.batch if head == "last" else rows
            if sampling.uniform is None or s.vocab > 1 << 22:
                raise ValueError("sampling needs uniform numbers, and a vocabulary of at most 4194304 tokens")
            checks += [(sampling.uniform, "uniform", f32, n), (sampling.temperature, "temperature", f32, n), (sampling.top_k, "top_k", i32, n),
                       (sampling.top_p, "top_p", f32, n), (sampling.min_p, "min_p", f32, n), (next_ids, "next_ids", i32, n),
                       (None if sampling.prob is True else sampling.prob, "prob", f32, n)]
        for t, name, dtype, n in checks:
            if t is not None and (t.dtype is not dtype or t.shape != (n,) or not t.is_contiguous() or t.device != dev):
                raise ValueError(f"{name}: expected a contiguous {dtype} vector of {n} on {dev}")
        lora_ws = self._lora_workspace(rows) if adapters is not None else None
        if s.n_experts:
            self._expert_bufs(rows)
        x = bctm_embed(ids, self.embed, self._buf("x", rows, s.dim))
        # every input of a projection is kept tiled, so that the projections read it in whole kilobytes
        h, f = self._tiled("h", rows, s.dim), None if s.n_experts else self._tiled("f", rows, s.ffn)
        q, wq, wv = self._buf("q", rows, s.q_width), self._buf("wq", rows, s.kv_width), self._buf("wv", rows, s.kv_width)
        a = self._buf("a", rows, s.q_width)
        # a chunk's attention output is re-tiled for W_o (the matrix-core kernel reads whole tiles); for the
        # few rows of a decode step re-tiling would cost more than it saves
        at = self._tiled("a", rows, s.q_width) if rows >= 128 else None
        for l, lw in enumerate(self.layers):
            bctm_rmsnorm(x, lw["attn_norm"], s.eps, h, tiled=True)
            lora = self.adapters[l] if adapters is not None else {}
            if "qkv" in lora:
                bctm_linear_split_lora(h, lw["w_qkv"], lora["qkv"], adapters, (q, wq, wv), lora_ws)
            else:
                bctm_linear_split(h, lw["w_qkv"], (q, wq, wv))
            if s.head_norm or s.rope_base:
                qh, kh = q.view(rows, s.n_q_heads, s.head_dim), wq.view(rows, s.n_kv_heads, s.head_dim)
                bctm_qk_norm_rope(qh, kh, lw.get("q_norm"), lw.get("wq_norm"), s.eps if s.head_norm else None, positions,
                                  self.inv_freq, s.rope_interleaved, qh, kh)
            c = self.caches[l]
            if T == 1:
                c.decode_step(q.view(s.batch, s.n_q_heads, s.head_dim), wq.view(s.batch, s.n_kv_heads, s.head_dim),
                              wv.view(s.batch, s.n_kv_heads, s.head_dim),
                              a.view(s.batch, s.n_q_heads, s.head_dim))
            else:
                c.prefill(q.view(s.batch, T, s.n_q_heads, s.head_dim), wq.view(s.batch, T, s.n_kv_heads, s.head_dim),
                          wv.view(s.batch, T, s.n_kv_heads, s.head_dim), T,
                          a.view(s.batch, T, s.n_q_heads, s.head_dim))
            ax = bctm_pack_rows(a, at) if at is not None else a
            if "o" in lora:
                bctm_linear_lora(ax, lw["w_o"], lora["o"], adapters, x, x, lora_ws)
            else:
                bctm_linear(ax, lw["w_o"], x, x)
            if s.n_experts:
                self._experts(x, lw, rows)
                continue
            bctm_rmsnorm(x, lw["mlp_norm"], s.eps, h, tiled=True)
            if "gate_up" in lora:
                bctm_swiglu_lora(h, lw["w_gate"], lw["w_up"], lora["gate_up"], adapters, f, True, lora_ws)
            else:
                bctm_swiglu(h, lw["w_gate"], lw["w_up"], f, tiled=True)
            if "down" in lora:
                bctm_linear_lora(f, lw["w_down"], lora["down"], adapters, x, x, lora_ws)
            else:
                bctm_linear(f, lw["w_down"], x, x)
        if head == "last" and T > 1:
            # rows b*T + T-1, gathered with the embedding kernel (a row lookup) from x as the table
            k = ("last_rows", s.batch, T)
            if k not in self._bufs:
                self._bufs[k] = (torch.arange(s.batch, dtype=torch.int32, device=self.device) * T + (T - 1)).contiguous()
            x = bctm_embed(self._bufs[k], x, self._buf("x_last", s.batch, s.dim))
            rows = s.batch
            h = self._tiled("h_last", rows, s.dim)
        bctm_rmsnorm(x, self.final_norm, s.eps, h, tiled=True)
        logits = bctm_linear(h, self.head, None, self._buf("logits", rows, s.vocab))
        if sampling is None:
            return bctm_argmax(logits, next_ids), logits
        nxt, _ = bctm_sample(logits, sampling.uniform, sampling.temperature, sampling.top_k, sampling.top_p, sampling.min_p, next_ids,
                             sampling.prob)
        return nxt, logits
