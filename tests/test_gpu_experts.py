"""Layers with experts: the projection with an epilogue, the router's choice and the experts' products, each against its definition
in 64 bits.

Tolerances.  A sum of n products of bf16 numbers in fp32 is off by at most about n 2^-24 of the sum of their magnitudes in any order; the
kernels add chains of up to K terms, whose errors average out, and are held to 2^-20 of that sum (K up to 4096: sqrt(4096) 2^-24 = 2^-18
would be the spread of errors that do not average within the matrix cores' own adders of 32 terms; 2^-20 is what the framework's other
projections are held to).  A bf16 output adds half a spacing, 2^-9 of the value, and where the sum's own error crosses the border between two
numbers a whole one: 2^-8 (bf16_ulp).  fp32 outputs add 2^-23 for bias, activation and residual each."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def M():
    from paper_2411_15785_amd import model
    model.mlib()
    return model


def normal(seed, shape, std=1.0, dtype=BF16):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * std).to(dtype).to(DEV)


def spacing(v):
    a = v.abs().clamp(min=2.0 ** -126)
    return torch.exp2(torch.floor(torch.log2(a)) - 7)


def close(got, want, slack, what):
    """got bf16 or fp32 against want in 64 bits; slack: what the fp32 arithmetic may be off."""
    want, slack = want.cpu(), slack.cpu()
    g = got.double().cpu()
    room = slack + (spacing(want) if got.dtype is BF16 else 2.0 ** -23 * 3 * want.abs())
    assert torch.isfinite(g).all(), what
    worst = ((g - want).abs() / room.clamp(min=1e-300)).max().item()
    assert worst <= 1.0, f"{what}: {worst} of the tolerance"


# ------------------------------------------------------------------ the projection with an epilogue

ACTS = {"none": lambda v: v, "relu": lambda v: v.clamp(min=0), "silu": lambda v: v * torch.sigmoid(v), "sigmoid": torch.sigmoid,
        "gelu": lambda v: 0.5 * v * torch.erfc(-v / 2.0 ** 0.5),
        "gelu_tanh": lambda v: 0.5 * v * (1 + torch.tanh((2.0 / np.pi) ** 0.5 * (v + 0.044715 * v ** 3)))}


def act_reference(x, w, bias, act, residual):
    x, w = x.double().cpu(), w.double().cpu()
    y, mass = x @ w.T, x.abs() @ w.abs().T
    if bias is not None:
        y, mass = y + bias.double().cpu(), mass + bias.double().cpu().abs()
    slack = 2.0 ** -20 * mass     # the activations' slopes are at most 1.13
    z = ACTS[act](y)
    # the fast exponential is off by 2^-22 + |y| 2^-24 relative: of the activation's value at most 2^-20 for |y| up to 48
    slack = 1.2 * slack + 2.0 ** -20 * z.abs() + (2.0 ** -21 if act in ("gelu", "gelu_tanh", "silu", "sigmoid") else 0)
    if residual is not None:
        z = z + residual.double().cpu()
        slack = slack + 2.0 ** -23 * residual.double().cpu().abs()
    return z, slack


@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("rows,K,N", [(1, 32, 16), (5, 1024, 208), (16, 2336, 48), (33, 64, 16400), (70, 512, 12288), (128, 96, 128),
                                      (200, 480, 1056), (300, 512, 640), (1100, 160, 512), (130, 64, 64), (17, 32, 64), (45, 4096, 64),
                                      (333, 2080, 192), (1030, 352, 256), (9000, 96, 64), (2100, 96, 320)])
def test_linear_act(M, rows, K, N, act):
    x, w, bias, res = normal(1, (rows, K)), normal(2, (N, K), K ** -0.5), normal(3, (N,)), normal(4, (rows, N))
    packed = M.bctm_pack_weight(w)
    if rows * N > 300000 and act not in ("gelu", "none"):
        pytest.skip("the large shapes run with two activations")
    for b, r, dtype in ((bias, res, BF16), (None, None, F32), (bias, None, BF16), (None, res, F32)):
        want, slack = act_reference(x, w, b, act, r)
        got = M.bctm_linear_act(x, packed, b, act, r, out_dtype=dtype)
        assert got.dtype is dtype
        close(got, want, slack, f"{act} bias {b is not None} residual {r is not None} {dtype}")
        tiled_in = M.bctm_linear_act(M.bctm_pack_rows(x), packed, b, act, r, out_dtype=dtype)
        assert torch.equal(got, tiled_in)
        if dtype is BF16 and N % 32 == 0:
            tiled = M.bctm_linear_act(x, packed, b, act, r, tiled=True)
            again = M.bctm_pack_rows(got)
            # rows behind the last one are not the call's
            whole = rows // 32 * 32 * N
            assert torch.equal(tiled.data[:whole], again.data[:whole])


@pytest.mark.parametrize("rows,N", [(4, 64), (16, 64), (40, 320), (300, 416), (600, 1024)])
def test_linear_act_without_anything_is_linear(M, rows, N):
    x, w, res = normal(5, (rows, 256)), M.bctm_pack_weight(normal(6, (N, 256), 1 / 16)), normal(7, (rows, N))
    assert torch.equal(M.bctm_linear_act(x, w), M.bctm_linear(x, w))
    assert torch.equal(M.bctm_linear_act(x, w, residual=res), M.bctm_linear(x, w, res))
    out = res.clone()
    assert M.bctm_linear_act(x, w, residual=out, out=out) is out
    assert torch.equal(out, M.bctm_linear(x, w, res))


def test_linear_act_ends_of_the_range(M):
    """Sums far from 0, infinities and NaN through every activation."""
    w = torch.zeros((16, 32), dtype=BF16, device=DEV)
    w[:, 0] = 1
    x = torch.zeros((9, 32), dtype=BF16, device=DEV)
    vals = torch.tensor([0.0, 1e-30, -1e-30, 120.0, -120.0, 3e4, -3e4, 60.0, -60.0])
    x[:, 0] = vals.to(BF16)
    p = M.bctm_pack_weight(w)
    for act, f in ACTS.items():
        got = M.bctm_linear_act(x, p, act=act, out_dtype=F32)[:, 3].double().cpu()
        want = f(x[:, 0].double().cpu())
        assert torch.isfinite(got).all(), act
        assert ((got - want).abs() <= 2.0 ** -20 * want.abs() + 2.0 ** -21 * (want.abs() < 1)).all(), (act, got, want)
    bias = torch.full((16,), float("nan"), dtype=BF16, device=DEV)
    for act in ACTS:
        assert torch.isnan(M.bctm_linear_act(x, p, bias, act)).all(), act
    bias.fill_(float("inf"))
    for act in ACTS:
        got = M.bctm_linear_act(x, p, bias, act)
        assert (got == (1.0 if act == "sigmoid" else float("inf"))).all(), act


# ------------------------------------------------------------------ the router


def route_reference(logits, k, bias, sigmoid, normalise, scale):
    x = logits.double().cpu().numpy()
    E = x.shape[1]
    ids = np.full((x.shape[0], k), -1, np.int32)
    w = np.zeros((x.shape[0], k))
    for r in range(x.shape[0]):
        may = np.flatnonzero(x[r] > -np.inf)
        if may.size == 0:
            continue
        l = x[r, may]
        with np.errstate(all="ignore"):
            # logarithms of the scores: their ratios do not underflow
            logp = -np.logaddexp(0.0, -l) if sigmoid else np.where(l == l.max(), 0.0, l - l.max())
            if not sigmoid:
                logp = logp - np.log(np.exp(logp).sum())
        rank = l if bias is None else np.exp(logp) + bias[may]
        ok = rank > -np.inf
        if normalise and not sigmoid:
            logp = l   # a softmax' ratios are those of exp(l), also where another logit is infinite
        may, logp, rank = may[ok], logp[ok], rank[ok]
        first = np.argsort(-rank, kind="stable")[:k]
        ids[r, :first.size] = may[first]
        with np.errstate(invalid="ignore"):
            if first.size == 0:
                continue
            top = logp[first].max() if normalise else 0.0
            p = np.where(logp[first] == top, 1.0, np.exp(logp[first] - top)) if normalise else np.exp(logp[first])
            w[r, :first.size] = scale * p / (p.sum() if normalise else 1.0)
    return ids, w


def plan_reference(ids, E):
    flat = ids.reshape(-1)
    key = np.where((flat >= 0) & (flat < E), flat, E)
    order = np.argsort(key, kind="stable")
    return order, np.searchsorted(key[order], np.arange(E + 1))


def check_plan(plan, ids, E):
    order, offsets = plan_reference(ids, E)
    assert np.array_equal(plan.offsets.cpu().numpy(), offsets)
    assert np.array_equal(plan.order.cpu().numpy(), order)


def check_route(M, logits, k, bias=None, sigmoid=False, normalise=True, scale=1.0):
    E = logits.shape[1]
    ids, w, plan = M.bctm_route(logits, k, bias, sigmoid, normalise, scale)
    want, ww = route_reference(logits, k, None if bias is None else bias.double().cpu().numpy(), sigmoid, normalise, scale)
    got = ids.cpu().numpy()
    assert np.array_equal(got, want)
    # exponentials and their sum over E experts, errors of 2^-23 each, the sum's average out; a far exponent's own rounding: |x| 2^-24
    span = 80.0
    off = np.abs(w.double().cpu().numpy() - ww) - (np.abs(ww) * (2.0 ** -24 * (8 + span)) + 2.0 ** -126)
    assert off.max() <= 0
    check_plan(plan, want, E)
    return ids, w, plan


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("biased", [False, True])
@pytest.mark.parametrize("rows,E,k", [(1, 1, 1), (1, 64, 8), (3, 16, 16), (17, 5, 2), (64, 65, 4), (65, 128, 8), (129, 300, 6), (700, 512, 16),
                                      (2049, 60, 4)])
def test_route(M, rows, E, k, biased, sigmoid):
    for dtype in (F32, BF16):   # bf16 logits have equal ones
        logits = normal(rows + E, (rows, E), 2.0, dtype)
        bias = normal(9, (E,), 0.1, F32) if biased else None
        check_route(M, logits, k, bias, sigmoid)
        check_route(M, logits, k, bias, sigmoid, normalise=False, scale=2.5)


def test_route_masks(M):
    """Rows with fewer experts than slots, with none, with NaN and infinities; rows at a distance."""
    wide = normal(11, (100, 40), 2.0, F32)
    x = wide[:, 3:33]
    x[::7] = float("-inf")
    x[1::7, 2:] = float("-inf")
    x[2::7, ::2] = float("nan")
    x[3::7, 5] = float("inf")
    x[4::7, 5:8] = float("inf")
    x[5::7] = torch.finfo(F32).min
    x[6::7, 4] = torch.finfo(F32).min
    for sigmoid in (False, True):
        for normalise in (False, True):
            check_route(M, x, 4, None, sigmoid, normalise)
    bias = torch.zeros(30, device=DEV)
    bias[::3] = float("-inf")
    bias[1] = float("nan")
    y = wide[:, 10:40].clone()
    y[::7] = float("-inf")
    for sigmoid in (False, True):
        check_route(M, y, 4, bias, sigmoid)


def test_route_equal_and_far_logits(M):
    x = torch.zeros((70, 100), device=DEV)
    check_route(M, x, 7)
    x[:, 50] = -0.0
    check_route(M, x, 7, sigmoid=True)
    # sigmoids that underflow in fp32 are still told apart and normalised
    x = normal(12, (70, 100), 3.0, F32) - 85.0
    check_route(M, x, 7, sigmoid=True)
    x = normal(12, (70, 100), 200.0, F32)
    check_route(M, x, 7)
    # a bias that decides between scores closer than fp32 tells apart
    x = torch.full((3, 8), 20.0, device=DEV) + torch.arange(8, device=DEV) * 2.0 ** -19
    bias = torch.full((8,), 0.5, device=DEV)
    ids, _, _ = check_route(M, x, 3, bias, sigmoid=True)
    assert ids[0].tolist() == [7, 6, 5]


@pytest.mark.parametrize("E,k", [(40, 8), (40, 16), (100, 6), (200, 16), (512, 16)])
def test_route_crowds_at_the_border(M, E, k):
    """Biased sigmoids of which many lie within the roundings of fp32 of the kth, more than there are lanes for a token, beside tokens
    without such crowds; equal sums among them."""
    g = torch.Generator().manual_seed(E)
    x = torch.randn((50, E), generator=g)
    x[::3] = 1.0 + torch.randint(0, 40, (17, E), generator=g) * 2.0 ** -22
    x[1::6, : E // 2] = 3.0
    x[7] = 0.0
    x[8] = 12.0 + torch.arange(E) * 2.0 ** -20     # sigmoids that differ by 6e-12, far above 2^-53, far below 2^-24
    x[9, ::2] = float("-inf")
    for bias in (torch.zeros(E), torch.full((E,), 1000.0), torch.randn(E, generator=g) * 1e-7):
        for sigmoid in (True, False):
            check_route(M, x.to(DEV), k, bias.to(DEV), sigmoid)


@pytest.mark.parametrize("rows,k,E", [(1, 1, 1), (1, 16, 16), (64, 16, 512), (65, 3, 7), (4096, 8, 64), (20001, 2, 512), (33000, 16, 33)])
def test_plan_of_given_experts(M, rows, k, E):
    """Any ids: the same expert twice in a row of slots, one expert for all, none for some or all."""
    g = torch.Generator().manual_seed(rows)
    ids = torch.randint(-2, E + 2, (rows, k), generator=g, dtype=torch.int32)
    for i in (ids, torch.full_like(ids, E - 1), torch.full_like(ids, -1), torch.full_like(ids, 2 ** 31 - 1)):
        check_plan(M.bctm_expert_plan(i.to(DEV), E), i.numpy(), E)


# ------------------------------------------------------------------ the experts' products


def choose(seed, rows, k, E, none=0.1, only=None):
    """Experts of each token's own (now and then the same one twice), none for some slots and some tokens."""
    g = torch.Generator().manual_seed(seed)
    ids = torch.randint(0, E, (rows, k), generator=g, dtype=torch.int32)
    ids[torch.rand((rows, k), generator=g) < none] = -1
    ids[torch.rand(rows, generator=g) < none] = E + 3
    if only is not None:
        ids[:] = only
    return ids, torch.rand((rows, k), generator=g) * 2 - 0.5


def swiglu_reference(x, wg, wu, ids):
    rows, k = ids.shape
    x, wg, wu = x.double().cpu(), wg.double().cpu(), wu.double().cpu()
    out, slack = torch.zeros((rows * k, wg.shape[1]), dtype=torch.float64), torch.zeros((rows * k, wg.shape[1]), dtype=torch.float64)
    for e in range(wg.shape[0]):
        p = torch.nonzero(ids.reshape(-1) == e)[:, 0]
        v = x[p // k]
        g, u, mg, mu = v @ wg[e].T, v @ wu[e].T, v.abs() @ wg[e].abs().T, v.abs() @ wu[e].abs().T
        s = g * torch.sigmoid(g)
        out[p] = s * u
        slack[p] = 2.0 ** -20 * (1.1 * mg * u.abs() + s.abs() * mu + out[p].abs())
    return out, slack


SHAPES = [  # rows, k, E, K, N
    (1, 1, 1, 32, 16), (1, 2, 16, 1024, 512), (7, 3, 5, 96, 48), (32, 8, 64, 256, 176), (50, 2, 3, 2080, 32), (129, 2, 8, 128, 80),
    (300, 4, 16, 160, 96), (400, 2, 4, 64, 272), (1300, 4, 9, 96, 144), (2000, 2, 4, 64, 528), (1, 16, 512, 32, 16), (260, 1, 2, 1376, 64),
    (900, 4, 4, 640, 1040), (2500, 8, 16, 192, 1040), (2600, 4, 4, 640, 2064), (3000, 2, 2, 1056, 4112)]


def test_the_shapes_reach_every_tile(M):
    assert {M.bctm_expert_tile(*s, True) for s in SHAPES} == {(16, 16), (64, 64), (128, 128), (256, 128)}
    assert {M.bctm_expert_tile(*s, False) for s in SHAPES} == {(16, 32), (64, 128), (128, 256), (256, 256)}


@pytest.mark.parametrize("rows,k,E,K,N", SHAPES)
def test_expert_swiglu(M, rows, k, E, K, N):
    x, wg, wu = normal(1, (rows, K)), normal(2, (E, N, K), K ** -0.5), normal(3, (E, N, K), K ** -0.5)
    pg, pu = M.bctm_pack_experts(wg), M.bctm_pack_experts(wu)
    for ids, _ in (choose(5, rows, k, E), choose(6, rows, k, E, only=E - 1), choose(7, rows, k, E, only=-1)):
        plan = M.bctm_expert_plan(ids.to(DEV), E)
        out = torch.full((rows * k, N), 7.0, dtype=BF16, device=DEV)
        assert M.bctm_expert_swiglu(x, pg, pu, plan, out) is out
        has = ((ids >= 0) & (ids < E)).reshape(-1)
        want, slack = swiglu_reference(x, wg, wu, ids)
        close(out[has.to(DEV)], want[has], slack[has], "with an expert") if has.any() else None
        assert (out[~has.to(DEV)] == 7.0).all()   # left as they were
        assert torch.equal(M.bctm_expert_swiglu(x, pg, pu, plan)[has.to(DEV)], out[has.to(DEV)])


@pytest.mark.parametrize("rows,k,E,K,N", SHAPES)
def test_expert_linear(M, rows, k, E, K, N):
    h, w, res = normal(1, (rows * k, K)), normal(2, (E, N, K), K ** -0.5), normal(3, (rows, N))
    packed = M.bctm_pack_experts(w)
    for ids, weights in (choose(5, rows, k, E), choose(6, rows, k, E, only=0), choose(7, rows, k, E, only=-1)):
        plan = M.bctm_expert_plan(ids.to(DEV), E)
        flat = ids.reshape(-1)
        hd, wd = h.double().cpu(), w.double().cpu()
        y, mass = torch.zeros((rows * k, N), dtype=torch.float64), torch.zeros((rows * k, N), dtype=torch.float64)
        for e in range(E):
            p = torch.nonzero(flat == e)[:, 0]
            y[p], mass[p] = hd[p] @ wd[e].T, hd[p].abs() @ wd[e].abs().T
        wt = weights.double()[..., None]
        # Products that wait for their sum in blocks of eight: multiples of 2^(e - 140), with the largest of the eight at least 2^(e - 127)
        # (1 - 2^-12) in magnitude, so off by at most 2^(e - 141) = 2^-14 / (1 - 2^-12) of it.
        block = y.abs().view(rows * k, N // 8, 8).max(-1, keepdim=True).values.expand(-1, -1, 8).reshape(rows, k, N)
        blocks = (2.0 ** -14 * 1.01 * block * wt.abs()).sum(1) if M.bctm_expert_tile(rows, k, E, K, N, False)[0] > 16 else 0.0
        out, mass = (y.view(rows, k, N) * wt).sum(1), (mass.view(rows, k, N) * wt.abs()).sum(1)
        # rows without an expert may hold anything
        hp = torch.where(((flat >= 0) & (flat < E)).to(DEV)[:, None], h, torch.full_like(h, float("nan")))
        wts = weights.to(DEV)
        close(M.bctm_expert_linear(hp, packed, plan, wts), out, 2.0 ** -20 * mass + blocks, "plain")
        close(M.bctm_expert_linear(hp, packed, plan, wts, res), out + res.double().cpu(),
              2.0 ** -20 * (mass + res.double().cpu().abs()) + blocks, "residual")
        inplace = res.clone()
        M.bctm_expert_linear(hp, packed, plan, wts, inplace, inplace)
        assert torch.equal(inplace, M.bctm_expert_linear(hp, packed, plan, wts, res))


def test_expert_linear_of_more_tiles_than_a_grid_is_high(M):
    """Tiny matrices have tiles of 16 rows at any number of tokens: more than 65535 of them."""
    rows, k, E, K, N = 140000, 8, 8, 32, 16
    assert M.bctm_expert_tile(rows, k, E, K, N, False) == (16, 32) and rows * k / 16 > 65535
    h, w = normal(1, (rows * k, K)), normal(2, (E, N, K), K ** -0.5)
    ids, weights = choose(5, rows, k, E)
    plan = M.bctm_expert_plan(ids.to(DEV), E)
    flat, y, mass = ids.reshape(-1).to(DEV), torch.zeros((rows * k, N), dtype=torch.float64, device=DEV), torch.zeros((rows * k, N), dtype=torch.float64, device=DEV)
    for e in range(E):
        p = torch.nonzero(flat == e)[:, 0]
        hd, wd = h[p].double(), w[e].double()
        y[p], mass[p] = (hd[:, None] * wd).sum(-1), (hd[:, None] * wd).abs().sum(-1)
    wt = weights.to(DEV).double()[..., None]
    out, slack = (y.view(rows, k, N) * wt).sum(1), 2.0 ** -20 * (mass.view(rows, k, N) * wt.abs()).sum(1)
    close(M.bctm_expert_linear(h, M.bctm_pack_experts(w), plan, weights.to(DEV)), out.cpu(), slack.cpu(), "many tiles")


@pytest.mark.parametrize("rows,E", [(40, 8), (400, 8), (2500, 8)])
def test_a_tokens_bits_do_not_depend_on_the_others(M, rows, E):
    """The same tokens with other companions, another order and the experts' other tokens gone."""
    K, N, k = 160, 96, 2
    x, wg, wu = normal(1, (rows, K)), M.bctm_pack_experts(normal(2, (E, N, K), 0.1)), M.bctm_pack_experts(normal(3, (E, N, K), 0.1))
    ids, _ = choose(4, rows, k, E, none=0)
    base = M.bctm_expert_swiglu(x, wg, wu, M.bctm_expert_plan(ids.to(DEV), E)).view(rows, k, N)
    perm = torch.randperm(rows, generator=torch.Generator().manual_seed(1))
    moved = M.bctm_expert_swiglu(x[perm.to(DEV)].contiguous(), wg, wu, M.bctm_expert_plan(ids[perm].contiguous().to(DEV), E)).view(rows, k, N)
    assert torch.equal(moved, base[perm.to(DEV)])
    fewer = ids.clone()
    fewer[::2] = -1
    assert torch.equal(M.bctm_expert_swiglu(x, wg, wu, M.bctm_expert_plan(fewer.to(DEV), E)).view(rows, k, N)[1::2], base[1::2])


def test_nan_and_infinity_stay_with_their_token_and_expert(M):
    rows, k, E, K, N = 60, 2, 6, 64, 32
    for rows in (60, 600):
        x, wg, wu = normal(1, (rows, K)), normal(2, (E, N, K), 0.1), normal(3, (E, N, K), 0.1)
        x[5] = float("nan")
        wu[2] = float("nan")
        ids, _ = choose(4, rows, k, E, none=0)
        out = M.bctm_expert_swiglu(x, M.bctm_pack_experts(wg), M.bctm_pack_experts(wu), M.bctm_expert_plan(ids.to(DEV), E))
        bad = torch.isnan(out).all(1).cpu()
        want = (ids.reshape(-1) == 2) | (torch.arange(rows * k) // k == 5)
        assert torch.equal(bad, want)
        assert torch.isfinite(out[(~want).to(DEV)]).all()


@pytest.mark.parametrize("rows,k,E,K,N", [(40, 2, 4, 64, 528), (2000, 2, 4, 64, 528), (2600, 4, 4, 640, 2064)])
def test_products_without_a_number_leave_their_neighbours_alone(M, rows, k, E, K, N):
    """NaN and infinities among the features of a block of eight, and numbers of very different size in one."""
    h, w = normal(1, (rows * k, K)).abs(), normal(2, (E, N, K), K ** -0.5)
    ids, _ = choose(4, rows, k, E, none=0)
    weights = torch.ones((rows, k), device=DEV)
    plan = M.bctm_expert_plan(ids.to(DEV), E)
    base = M.bctm_expert_linear(h, M.bctm_pack_experts(w), plan, weights)
    w2 = w.clone()
    w2[:, 3] = float("nan")
    w2[:, 12] = float("inf")
    w2[:, 13] = float("-inf")
    w2[:, 40:48] = 0
    w2[:, 65:72] *= 2.0 ** -40   # feature 64 has the block's numbers to itself
    w2[:, 72:80] *= 2.0 ** -100
    w2[:, 80:88] *= 2.0 ** 100
    got = M.bctm_expert_linear(h, M.bctm_pack_experts(w2), plan, weights)
    zero = (h == 0).view(rows, -1).any(1)   # 0 times infinity
    assert torch.isnan(got[:, 3]).all() and torch.isnan(got[zero][:, 12:14]).all()
    assert (got[~zero][:, 12] == float("inf")).all() and (got[~zero][:, 13] == float("-inf")).all()
    assert (got[:, 40:48] == 0).all()
    same = torch.ones(N, dtype=torch.bool, device=DEV)
    same[[3, 12, 13]] = False
    same[40:48] = same[64:88] = False
    same[0:16] = False
    assert torch.equal(got[:, same], base[:, same])
    # the neighbours of what is no number: a smaller largest one only makes them more exact
    near = [i for i in range(16) if i not in (3, 12, 13)] + [64]
    scale = base[:, :80].float().abs().max().item() + h.float().max().item() * K ** 0.5
    # two roundings of sums that far apart: one spacing of the larger, which is up to 2^-7 of it, and the sums' own distance
    g, f = got[:, near].double(), base[:, near].double()
    off = (g - f).abs() / (spacing(torch.maximum(g.abs(), f.abs())) + k * 2.0 ** -14 * scale)
    assert off.max().item() <= 1.0
    assert torch.equal(got[:, 72:80].float(), base[:, 72:80].float() * 2.0 ** -100)
    assert torch.equal(got[:, 80:88].float(), base[:, 80:88].float() * 2.0 ** 100)


# ------------------------------------------------------------------ together, as a layer uses them


class Layer:
    """Router, experts and their way back on buffers of their own."""

    def __init__(self, M, rows, E, k, dim, ffn, seed=1):
        self.M, self.k, self.E = M, k, E
        self.x = normal(seed, (rows, dim))
        self.router = M.bctm_pack_weight(normal(seed + 1, (64 * ((E + 63) // 64), dim), dim ** -0.5))
        self.gate, self.up = (M.bctm_pack_experts(normal(seed + i, (E, ffn, dim), dim ** -0.5)) for i in (2, 3))
        self.down = M.bctm_pack_experts(normal(seed + 4, (E, dim, ffn), ffn ** -0.5))
        self.bias = normal(seed + 5, (E,), 0.05, F32)
        self.logits = torch.empty((rows, 64 * ((E + 63) // 64)), device=DEV)
        self.experts, self.weights = torch.empty((rows, k), dtype=torch.int32, device=DEV), torch.empty((rows, k), device=DEV)
        self.plan = M.ExpertPlan(rows, k, E, DEV)
        self.h = torch.zeros((rows * k, ffn), dtype=BF16, device=DEV)
        self.out = torch.empty((rows, dim), dtype=BF16, device=DEV)
        self.workspace = torch.empty(M.bctm_expert_workspace(rows, k, dim), dtype=torch.uint8, device=DEV)

    def __call__(self):
        M = self.M
        M.bctm_linear_act(self.x, self.router, out=self.logits)
        M.bctm_route(self.logits[:, :self.E], self.k, self.bias, True, experts=self.experts, weights=self.weights, plan=self.plan)
        M.bctm_expert_swiglu(self.x, self.gate, self.up, self.plan, self.h)
        return M.bctm_expert_linear(self.h, self.down, self.plan, self.weights, self.x, self.out, self.workspace)


@pytest.mark.parametrize("rows,E,k,dim,ffn", [(1, 8, 2, 256, 96), (40, 12, 3, 128, 64), (700, 70, 6, 512, 160), (3000, 4, 2, 1056, 2080)])
def test_captured_layers_follow_their_inputs(M, rows, E, k, dim, ffn):
    """Replays with other tokens, and so other experts and another plan, eager work of a second layer in between."""
    a, b = Layer(M, rows, E, k, dim, ffn), Layer(M, rows, E, k, dim, ffn)
    a()
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        a()
    for step in range(4):
        x = normal(100 + step, (rows, dim))
        if step == 2:
            x[rows // 2:] = x[0]   # many tokens for the same experts
        a.x.copy_(x)
        b.x.copy_(x)
        g.replay()
        b()
        torch.cuda.synchronize()
        assert torch.equal(a.experts, b.experts) and torch.equal(a.plan.order, b.plan.order) and torch.equal(a.plan.offsets, b.plan.offsets)
        assert torch.equal(a.weights, b.weights) and torch.equal(a.out.view(torch.int16), b.out.view(torch.int16)), step
        check_plan(b.plan, b.experts.cpu().numpy(), E)


def test_two_streams_at_once(M):
    """Two layers that share weights and nothing else, each on a stream of its own, many times: the bits of the same calls one after the other."""
    a, b = Layer(M, 300, 16, 4, 512, 160), Layer(M, 300, 16, 4, 512, 160)
    for n in ("router", "gate", "up", "down", "bias"):
        setattr(b, n, getattr(a, n))
    b.x = normal(77, (300, 512))
    want = [a().clone(), b().clone()]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[], []]
    for _ in range(20):
        for i, layer in enumerate((a, b)):
            with torch.cuda.stream(streams[i]):
                layer()
                got[i].append(layer.out.clone())
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(o.view(torch.int16), want[i].view(torch.int16)) for o in got[i])


def test_a_plan_that_was_not_made_has_no_tokens(M):
    """Products by a plan of zeros write nothing; the weighted sum of nothing is the residual."""
    x, w = normal(1, (20, 64)), M.bctm_pack_experts(normal(2, (4, 32, 64)))
    plan = M.ExpertPlan(20, 2, 4, DEV)
    out = torch.full((40, 32), 3.0, dtype=BF16, device=DEV)
    assert (M.bctm_expert_swiglu(x, w, w, plan, out) == 3.0).all()
    res, workspace = normal(3, (20, 32)), torch.full((M.bctm_expert_workspace(20, 2, 32),), 255, dtype=torch.uint8, device=DEV)
    got = M.bctm_expert_linear(normal(4, (40, 64)), w, plan, torch.ones((20, 2), device=DEV), res, workspace=workspace)
    assert torch.equal(got, res)


def test_refusals_of_the_wrappers(M):
    x, w = normal(1, (20, 64)), M.bctm_pack_experts(normal(2, (4, 32, 64)))
    ids = torch.zeros((20, 2), dtype=torch.int32, device=DEV)
    plan, weights = M.bctm_expert_plan(ids, 4), torch.ones((20, 2), device=DEV)
    logits, h = torch.zeros((20, 4), device=DEV), normal(3, (40, 64))
    p = M.bctm_pack_weight(normal(4, (32, 64)))
    bad = [
        lambda: M.bctm_route(logits.double(), 2), lambda: M.bctm_route(logits.t(), 2), lambda: M.bctm_route(logits[0], 2),
        lambda: M.bctm_route(logits, 2, bias=torch.zeros(3, device=DEV)), lambda: M.bctm_route(logits, 2, bias=torch.zeros(4, device=DEV).half()),
        lambda: M.bctm_route(logits, 3, plan=plan), lambda: M.bctm_route(logits[:10], 2, plan=plan),
        lambda: M.bctm_route(logits, 2, experts=ids[:, :1]), lambda: M.bctm_route(logits, 2, weights=weights.double()),
        lambda: M.bctm_route(logits, 2, experts=ids.long()),
        lambda: M.bctm_expert_plan(ids.long(), 4), lambda: M.bctm_expert_plan(ids.t(), 4), lambda: M.bctm_expert_plan(ids[0], 4),
        lambda: M.bctm_expert_plan(ids, 5, plan), lambda: M.bctm_pack_experts(normal(5, (2, 24, 64))), lambda: M.bctm_pack_experts(normal(5, (32, 64))),
        lambda: M.bctm_expert_swiglu(x[:10], w, w, plan), lambda: M.bctm_expert_swiglu(x[:, :32].contiguous(), w, w, plan),
        lambda: M.bctm_expert_swiglu(x, w, p, plan), lambda: M.bctm_expert_swiglu(x, w, M.bctm_pack_experts(normal(6, (4, 48, 64))), plan),
        lambda: M.bctm_expert_swiglu(x, w, w, plan, out=normal(7, (20, 32))), lambda: M.bctm_expert_swiglu(x, w, w, plan.data),
        lambda: M.bctm_expert_linear(x, w, plan, weights), lambda: M.bctm_expert_linear(h, w, plan, weights.double()),
        lambda: M.bctm_expert_linear(h, w, plan, weights[:10]), lambda: M.bctm_expert_linear(h, w, plan, weights, residual=normal(8, (20, 64))),
        lambda: M.bctm_expert_linear(h, w, plan, weights, out=normal(8, (40, 32))),
        lambda: M.bctm_expert_linear(h, w, plan, weights, workspace=torch.empty(9999, device=DEV)),
        lambda: M.bctm_linear_act(x, p, act="tanh"), lambda: M.bctm_linear_act(x, p, bias=torch.zeros(32, device=DEV)),
        lambda: M.bctm_linear_act(x, p, residual=normal(9, (19, 32))), lambda: M.bctm_linear_act(x, p, out=torch.empty((20, 32), device=DEV).half()),
        lambda: M.bctm_linear_act(x, p, out=torch.empty((20, 32), device=DEV), out_dtype=BF16),
        lambda: M.bctm_linear_act(x, p, out=torch.empty((20, 32), device=DEV), tiled=True), lambda: M.bctm_linear_act(x, p, out_dtype=F32, tiled=True),
        lambda: M.bctm_linear_act(x, p, out=M.TiledRows(20, 32, DEV)), lambda: M.bctm_linear_act(x, w),
    ]
    for i, f in enumerate(bad):
        with pytest.raises(ValueError):
            f()
            pytest.fail(f"call {i} was taken")
    for f in (lambda: M.bctm_route(logits, 5), lambda: M.bctm_route(logits, 0), lambda: M.bctm_route(logits, 2, scale=float("nan")),
              lambda: M.bctm_expert_linear(h, w, plan, weights, workspace=torch.empty(64, dtype=torch.uint8, device=DEV)),
              lambda: M.bctm_route(torch.zeros((0, 4), device=DEV), 2)):
        with pytest.raises(M.BctModelError):
            f()
