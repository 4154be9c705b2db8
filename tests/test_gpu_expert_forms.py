"""The tiled forms of the experts' products: shapes that reach each tile (16 x .. is the streaming kernel, which test_gpu_experts.py
reaches with most of its shapes), held value by value to the formula in 64 bits.

Tolerances as in test_gpu_experts.py: a product's fp32 sum is off by at most 2^-20 of the sum of its terms' magnitudes, and the weighted
sum of products likewise; a bf16 output adds one spacing (a rounding is half of one, and the sum's own error may carry it over the
border between two numbers, which costs the other half).  Nothing is taken from a value's neighbours."""
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
BF16 = torch.bfloat16


@pytest.fixture(scope="module")
def M():
    from paper_2411_15785_amd import model
    model.mlib()
    return model


def normal(seed, shape, std=1.0, dtype=BF16):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (torch.randn(shape, generator=g, device=DEV) * std).to(dtype)


def choose(seed, rows, k, E, none=0.1):
    """Any experts, none for some slots and some tokens; int32 [rows][k] and weights float32 [rows][k]."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    ids = torch.randint(0, E, (rows, k), generator=g, device=DEV, dtype=torch.int32)
    ids[torch.rand((rows, k), generator=g, device=DEV) < none] = -1
    ids[torch.rand(rows, generator=g, device=DEV) < none] = E + 3
    return ids, torch.rand((rows, k), generator=g, device=DEV) * 2 - 0.5


def close(got, want, slack, what):
    """bf16 against 64 bits; slack: what the fp32 arithmetic may be off."""
    spacing = torch.exp2(torch.floor(torch.log2(want.abs().clamp(min=2.0 ** -126))) - 7)
    assert torch.isfinite(got).all(), what
    worst = ((got.double() - want).abs() / (slack + spacing)).max().item()
    assert worst <= 1.0, f"{what}: {worst} of the tolerance"


def back_reference(h, w, ids, weights, residual=None):
    """The way back in 64 bits and what fp32 may be off."""
    rows, k = ids.shape
    out = torch.zeros((rows * k, w.shape[1]), dtype=torch.float64, device=DEV)
    mass = torch.zeros_like(out)
    for e in range(w.shape[0]):
        p = torch.nonzero(ids.reshape(-1) == e)[:, 0]
        out[p], mass[p] = h[p].double() @ w[e].double().t(), h[p].double().abs() @ w[e].double().abs().t()
    wt = weights.double()[..., None]
    out, mass = (out.view(rows, k, -1) * wt).sum(1), (mass.view(rows, k, -1) * wt.abs()).sum(1)
    if residual is not None:
        out, mass = out + residual.double(), mass + residual.double().abs()
    return out, 2.0 ** -20 * mass


# the way back: tile rows, rows, k, E, N, K steps of 32
BACK = {64: (600, 2, 2, 1040, 20), 128: (1500, 4, 4, 2064, 13), 256: (6000, 4, 4, 1040, 22)}


@pytest.mark.parametrize("larger", [0, 7, 10, 14])
@pytest.mark.parametrize("tile", BACK)
def test_products_are_as_exact_beside_larger_features(M, tile, larger):
    """One feature of every eight is 2^larger times the others, as the outputs of a few features of down projections are."""
    rows, k, E, N, steps = BACK[tile]
    K = 32 * steps
    assert M.bctm_expert_tile(rows, k, E, K, N, False)[0] == tile
    h, w, res = normal(1, (rows * k, K)), normal(2, (E, N, K), K ** -0.5), normal(3, (rows, N))
    w[:, 5::8] *= 2.0 ** larger
    res[:, 5::8] *= 2.0 ** larger
    ids, weights = choose(4, rows, k, E)
    plan, packed = M.bctm_expert_plan(ids, E), M.bctm_pack_experts(w)
    for r in (None, res):
        close(M.bctm_expert_linear(h, packed, plan, weights, r), *back_reference(h, w, ids, weights, r), f"2^{larger}, residual {r is not None}")


def test_a_weighted_sum_of_products_that_cancel(M):
    """Two slots with the same expert and opposite weights, a third with a small one: what is left is the third's product, to fp32."""
    for tile, (rows, _, E, N, steps) in BACK.items():
        K, k = 32 * steps, 4 if tile != 64 else 2
        rows = rows if tile != 64 else 600
        h, w = normal(1, (rows * k, K)), normal(2, (E, N, K), K ** -0.5)
        h.view(rows, k, K)[:, 1] = h.view(rows, k, K)[:, 0]
        ids = torch.zeros((rows, k), dtype=torch.int32, device=DEV)
        weights = torch.full((rows, k), 2.0 ** -6, device=DEV)
        weights[:, 0], weights[:, 1] = 1.0, -1.0
        ids[:, 2:] = E - 1
        assert M.bctm_expert_tile(rows, k, E, K, N, False)[0] == tile
        got = M.bctm_expert_linear(h, M.bctm_pack_experts(w), M.bctm_expert_plan(ids, E), weights)
        close(got, *back_reference(h, w, ids, weights), tile)
        if k == 2:
            assert (got == 0).all()   # the same bits, one less the other


def gated_reference(x, wg, wu, ids):
    """silu(g) u in 64 bits and what fp32 may be off: silu's slope is at most 1.1."""
    rows, k = ids.shape
    out = torch.zeros((rows * k, wg.shape[1]), dtype=torch.float64, device=DEV)
    slack = torch.zeros_like(out)
    for e in range(wg.shape[0]):
        p = torch.nonzero(ids.reshape(-1) == e)[:, 0]
        v, a, b = x[p // k].double(), wg[e].double().t(), wu[e].double().t()
        g, u, mg, mu = v @ a, v @ b, v.abs() @ a.abs(), v.abs() @ b.abs()
        s = g * torch.sigmoid(g)
        out[p] = s * u
        slack[p] = 2.0 ** -20 * (1.1 * mg * u.abs() + s.abs() * mu + out[p].abs())
    return out, slack


def uneven(ids, E):
    """The last expert has one pair, the tokens that it had go to the first."""
    ids = torch.where(ids == E - 1, torch.zeros_like(ids), ids)
    ids[1, 0] = E - 1
    return ids


# tile rows: (rows, k, E, N), K steps of 32.  Stages are four, of 128 rows three: every remainder of the steps by the stages, and
# fewer steps than stages (256 rows take no fewer than seventeen here).
GATED_STEPS = {64: [((900, 4, 4, 1040), (1, 2)), ((600, 2, 2, 1040), (3, 4, 5, 6, 7, 8))],
               128: [((2000, 2, 2, 2064), (1, 2)), ((900, 4, 4, 1040), (3, 4, 5, 6, 7, 8))],
               256: [((4000, 2, 2, 2064), (20, 21, 22, 23))]}
BACK_STEPS = {64: [((2500, 8, 16, 1040), (1,)), ((900, 4, 4, 1040), (2, 3, 4, 5)), ((600, 2, 2, 1040), (6, 7, 8, 9))],
              128: [((1500, 8, 40, 1040), (1, 2, 3, 4)), ((1500, 4, 4, 2064), (5, 6, 7, 8))],
              256: [((6000, 4, 4, 1040), (21, 22, 23, 24))]}


def flat(table):
    return [(tile, *sizes, steps) for tile, v in table.items() for sizes, all_steps in v for steps in all_steps]


@pytest.mark.parametrize("tile,rows,k,E,N,steps", flat(GATED_STEPS))
def test_gated_products_of_every_remainder_of_steps(M, tile, rows, k, E, N, steps):
    K = 32 * steps
    assert M.bctm_expert_tile(rows, k, E, K, N, True)[0] == tile
    x, wg, wu = normal(1, (rows, K)), normal(2, (E, N, K), K ** -0.5), normal(3, (E, N, K), K ** -0.5)
    pg, pu = M.bctm_pack_experts(wg), M.bctm_pack_experts(wu)
    ids, _ = choose(4, rows, k, E)
    for i in (ids, uneven(ids, E)):
        out = torch.full((rows * k, N), 7.0, dtype=BF16, device=DEV)
        M.bctm_expert_swiglu(x, pg, pu, M.bctm_expert_plan(i, E), out)
        has = ((i >= 0) & (i < E)).reshape(-1)
        want, slack = gated_reference(x, wg, wu, i)
        close(out[has], want[has], slack[has], f"{steps} steps")
        assert (out[~has] == 7.0).all()


@pytest.mark.parametrize("tile,rows,k,E,N,steps", flat(BACK_STEPS))
def test_the_way_back_of_every_remainder_of_steps(M, tile, rows, k, E, N, steps):
    K = 32 * steps
    assert M.bctm_expert_tile(rows, k, E, K, N, False)[0] == tile
    h, w, res = normal(1, (rows * k, K)), normal(2, (E, N, K), K ** -0.5), normal(3, (rows, N))
    packed = M.bctm_pack_experts(w)
    ids, weights = choose(4, rows, k, E)
    for i in (ids, uneven(ids, E)):
        has = ((i >= 0) & (i < E)).reshape(-1)
        hp = torch.where(has[:, None], h, torch.full_like(h, float("nan")))   # rows without an expert may hold anything
        workspace = torch.full((M.bctm_expert_workspace(rows, k, N),), 255, dtype=torch.uint8, device=DEV)   # NaN
        got = M.bctm_expert_linear(hp, packed, M.bctm_expert_plan(i, E), weights, res, workspace=workspace)
        close(got, *back_reference(h, w, i, weights, res), f"{steps} steps")


def test_the_tables_have_every_remainder():
    for table in (GATED_STEPS, BACK_STEPS):
        for tile, stages in ((64, 4), (128, 3), (256, 4)):
            assert {s % stages for t, *_, s in flat(table) if t == tile} == set(range(stages))


# tile rows of both products: rows, k, E, dim, ffn (gated dim -> ffn, back ffn -> dim)
LAYERS = {16: (40, 2, 8, 160, 96), 64: (600, 2, 4, 512, 512), 128: (1500, 4, 8, 1056, 1056), 256: (6000, 4, 4, 1056, 800)}


class Products:
    """Both products of the experts, weights shared by what is made `like` another, buffers of its own."""

    def __init__(self, M, tile, seed=1, like=None):
        self.M, (self.rows, self.k, self.E, self.dim, self.ffn) = M, LAYERS[tile]
        rows, k, E, dim, ffn = LAYERS[tile]
        assert M.bctm_expert_tile(rows, k, E, dim, ffn, True)[0] == M.bctm_expert_tile(rows, k, E, ffn, dim, False)[0] == tile
        self.raw = like.raw if like else [normal(2 + i, s, s[-1] ** -0.5) for i, s in enumerate(((E, ffn, dim), (E, ffn, dim), (E, dim, ffn)))]
        self.packed = like.packed if like else [M.bctm_pack_experts(w) for w in self.raw]
        self.x, self.res = normal(seed, (rows, dim)), normal(seed + 10, (rows, dim))
        self.ids, self.weights = choose(seed + 20, rows, k, E, none=0.0)
        self.plan = M.ExpertPlan(rows, k, E, DEV)
        self.h = torch.zeros((rows * k, ffn), dtype=BF16, device=DEV)
        self.out = torch.empty((rows, dim), dtype=BF16, device=DEV)
        self.workspace = torch.empty(M.bctm_expert_workspace(rows, k, dim), dtype=torch.uint8, device=DEV)

    def __call__(self):
        M = self.M
        M.bctm_expert_plan(self.ids, self.E, self.plan)
        M.bctm_expert_swiglu(self.x, self.packed[0], self.packed[1], self.plan, self.h)
        return M.bctm_expert_linear(self.h, self.packed[2], self.plan, self.weights, self.res, self.out, self.workspace)


def same(a, b):
    return torch.equal(a.view(torch.int16), b.view(torch.int16))


@pytest.mark.parametrize("tile", LAYERS)
def test_bits_of_a_token_are_its_own(M, tile):
    """The same tokens in another order, and with half of their companions gone."""
    p = Products(M, tile)
    out, h = p().clone(), p.h.clone().view(p.rows, p.k, -1)
    perm = torch.randperm(p.rows, generator=torch.Generator().manual_seed(1)).to(DEV)
    kept = [t.clone() for t in (p.x, p.res, p.ids, p.weights)]
    p.x, p.res, p.ids, p.weights = (t[perm].contiguous() for t in kept)
    moved = p()
    assert same(p.h.view(p.rows, p.k, -1), h[perm]) and same(moved, out[perm])
    p.x, p.res, p.ids, p.weights = kept
    p.ids = p.ids.clone()
    p.ids[::2] = -1
    fewer = p()
    assert same(p.h.view(p.rows, p.k, -1)[1::2], h[1::2]) and same(fewer[1::2], out[1::2])
    assert same(fewer[::2], p.res[::2])   # no expert: the residual


@pytest.mark.parametrize("tile", LAYERS)
def test_what_is_no_number_stays_with_its_token_expert_and_feature(M, tile):
    p = Products(M, tile)
    good, h = p().clone(), p.h.clone()
    p.x[5], p.x[p.rows - 1, 3] = float("nan"), float("nan")
    p()
    token = torch.zeros(p.rows, dtype=torch.bool, device=DEV)
    token[[5, p.rows - 1]] = True
    pair = token.repeat_interleave(p.k)
    assert torch.isnan(p.h[pair]).all() and same(p.h[~pair], h[~pair])
    assert torch.isnan(p.out[token]).all() and same(p.out[~token], good[~token])
    # an expert of NaN, and features of infinities and NaN in the way back: a block of eight has a few of each
    p = Products(M, tile, like=p)
    w = [t.clone() for t in p.raw]
    w[1][2 % p.E] = float("nan")
    p.packed = [M.bctm_pack_experts(t) for t in w]
    p()
    hit = (p.ids.reshape(-1) == 2 % p.E)
    assert torch.isnan(p.h[hit]).all() and same(p.h[~hit], h[~hit])
    w = [t.clone() for t in p.raw]
    w[2][:, 3], w[2][:, 12], w[2][:, 13] = float("nan"), float("inf"), float("-inf")
    p.packed = [M.bctm_pack_experts(t) for t in w]
    got = p()
    odd = torch.zeros(p.dim, dtype=torch.bool, device=DEV)
    odd[[3, 12, 13]] = True
    # sums of infinities of either sign or times 0 are NaN, others an infinity: no number in any case
    some = (p.ids < p.E).any(1)
    assert not torch.isfinite(got[some][:, odd]).any() and torch.isnan(got[some][:, 3]).all()
    assert same(got[:, ~odd], good[:, ~odd])


@pytest.mark.parametrize("tile", [64, 128, 256])
def test_two_streams_of_tiled_products(M, tile):
    """Two sets of tokens with the same weights, each on a stream of its own: the bits of one after the other."""
    a = Products(M, tile)
    b = Products(M, tile, seed=50, like=a)
    want = [a().clone(), b().clone()]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], [[], []]
    for _ in range(8):
        for i, p in enumerate((a, b)):
            with torch.cuda.stream(streams[i]):
                got[i].append(p().clone())
    torch.cuda.synchronize()
    assert all(same(o, want[i]) for i in range(2) for o in got[i])


@pytest.mark.parametrize("tile", [64, 128, 256])
def test_captured_tiled_products(M, tile):
    """Replays with other tokens, experts and weights; eager calls on other buffers between them."""
    a = Products(M, tile)
    b = Products(M, tile, like=a)
    a()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        a()
    for step in range(4):
        ids, weights = choose(60 + step, a.rows, a.k, a.E, none=0.1 * step)
        x = normal(70 + step, (a.rows, a.dim))
        for p in (a, b):
            p.x.copy_(x), p.ids.copy_(uneven(ids, a.E) if step == 2 else ids), p.weights.copy_(weights)
        g.replay()
        b()
        torch.cuda.synchronize()
        assert same(a.out, b.out), step


def test_weights_past_32_bits(M):
    """512 experts of 1024 x 4096: 2^31 values, 4 GB.  Tokens of the first, the last and one between, of few and of many a call."""
    E, N, K = 512, 1024, 4096
    used = torch.tensor([0, 300, 511], dtype=torch.int32, device=DEV)
    w = torch.zeros((E, N, K), dtype=BF16, device=DEV)
    some = normal(1, (3, N, K), K ** -0.5)
    w[used.long()] = some
    packed = M.bctm_pack_experts(w)
    del w
    for rows, k, tiles in ((64, 4, (16, 16)), (4096, 8, (256, 256))):
        assert (M.bctm_expert_tile(rows, k, E, K, N, True)[0], M.bctm_expert_tile(rows, k, E, K, N, False)[0]) == tiles
        g = torch.Generator(device=DEV).manual_seed(rows)
        which = torch.randint(0, 3, (rows, k), generator=g, device=DEV)
        plan, x = M.bctm_expert_plan(used[which], E), normal(2, (rows, K))
        want, slack = gated_reference(x, some, some, which)
        close(M.bctm_expert_swiglu(x, packed, packed, plan), want, slack, "gated")
        h, weights = normal(3, (rows * k, K)), torch.rand((rows, k), generator=g, device=DEV)
        close(M.bctm_expert_linear(h, packed, plan, weights), *back_reference(h, some, which, weights), "back")


def test_rows_past_32_bits(M):
    """More than 2^32 values of h: 1052672 rows of 4096, the same 4096 over and over."""
    E, N, K, rows = 2, 32, 4096, (1 << 20) + 4096
    base, w = normal(1, (4096, K)), normal(2, (E, N, K), K ** -0.5)
    h = base.repeat(rows // 4096, 1)
    assert h.numel() > 1 << 32
    g = torch.Generator(device=DEV).manual_seed(3)
    ids = torch.randint(0, E, (rows, 1), generator=g, device=DEV, dtype=torch.int32)
    plan, packed, one = M.bctm_expert_plan(ids, E), M.bctm_pack_experts(w), torch.ones((rows, 1), device=DEV)
    got = M.bctm_expert_linear(h, packed, plan, one)
    gated = M.bctm_expert_swiglu(h, packed, packed, plan)
    both = [back_reference(base, w, torch.full((4096, 1), e, dtype=torch.int32, device=DEV), one[:4096]) for e in range(E)]
    pick = (ids[:, 0].long(), torch.arange(rows, device=DEV) % 4096)
    close(got, torch.stack([b[0] for b in both])[pick], torch.stack([b[1] for b in both])[pick], "back")
    both = [gated_reference(base, w, w, torch.full((4096, 1), e, dtype=torch.int32, device=DEV)) for e in range(E)]
    close(gated, torch.stack([b[0] for b in both])[pick], torch.stack([b[1] for b in both])[pick], "gated")
