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
