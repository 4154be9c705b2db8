"""bctm_sample against its definition in numpy's longdouble: sort, cumulate, compare.  Tokens have to be equal.  prob: one
rounding to fp32, 2^-24; N roundings of weights to half of 2^-S (S at least 40, N * 2^-S at most 2^-22 * 2^4 for the largest N
here, 2^-29 for N up to 2^17) and the series' 2e-13."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def M():
    from paper_2411_15785_amd import model
    model.mlib()
    return model


def reference(x, u, t, k, p, m):
    """One row, float64 logits -> (token, its probability)."""
    at = np.flatnonzero(x > -np.inf)
    if at.size == 0:
        return -1, 0.0
    order = at[np.argsort(-x[at], kind="stable")]
    l = x[order].astype(np.longdouble)
    if not t > 0:
        return int(order[0]), 1.0
    with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
        w = np.where(l == l[0], np.longdouble(1), np.exp((l - l[0]) / np.longdouble(t)))
    cum = np.cumsum(w)
    n = len(w)
    if 0 < k < n:
        n = int(k)
    base, keep = cum[n - 1], n
    if p < 1:
        keep = min(keep, int(np.searchsorted(cum[:n], np.longdouble(p) * base, side="left")) + 1)
    if m > 0:
        keep = min(keep, int(np.count_nonzero(w >= np.longdouble(m))))
    keep = max(keep, 1)
    u = min(max(u, 0.0), 1.0 - 2.0 ** -24) if u == u else 0.0
    j = min(int(np.searchsorted(cum[:keep], np.longdouble(u) * cum[keep - 1], side="right")), keep - 1)
    return int(order[j]), float(w[j] / cum[keep - 1])


def check(M, x, u, t=None, k=None, p=None, m=None, what=""):
    rows = x.shape[0]
    f = lambda v, dt: None if v is None else torch.tensor(np.broadcast_to(np.asarray(v, dt), (rows,)).copy()).cuda()
    tu, tt, tk, tp, tm = f(u, np.float32), f(t, np.float32), f(k, np.int32), f(p, np.float32), f(m, np.float32)
    ids, prob = M.bctm_sample(x, tu, tt, tk, tp, tm, prob=True)
    h = lambda v, d: np.full(rows, d) if v is None else v.cpu().numpy().astype(np.float64)
    xs, hu, ht, hk, hp, hm = x.double().cpu().numpy(), h(tu, 0), h(tt, 1), h(tk, 0), h(tp, 1), h(tm, 0)
    want = [reference(xs[r], hu[r], ht[r], hk[r], hp[r], hm[r]) for r in range(rows)]
    ids, prob = ids.cpu().numpy(), prob.cpu().numpy().astype(np.float64)
    wid, wpr = np.array([a for a, _ in want]), np.array([b for _, b in want])
    bad = np.flatnonzero(ids != wid)
    assert bad.size == 0, f"{what}: rows {bad[:5]}: {ids[bad[:5]]} for {wid[bad[:5]]}"
    assert np.all(np.abs(prob - wpr) <= wpr * (2.0 ** -24 * 1.001 + 2.0 ** -28) + 2.0 ** -149), what
    return ids


def logits(rows, N, dtype, seed, spread=2.5, ld=None):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((rows, ld or N), generator=g) * spread
    x[:, : min(N, 8)] += 5.0 * torch.rand((rows, min(N, 8)), generator=g)
    return x.to(DT[dtype]).cuda()[:, :N]


def uniform(rows, seed):
    return torch.rand(rows, generator=torch.Generator().manual_seed(seed)).numpy()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N", [1, 2, 7, 63, 64, 65, 1000, 1024, 8191, 32000, 50001, 131072])
def test_every_setting_alone_and_together(M, N, dtype):
    rows = 12
    x = logits(rows, N, dtype, N)
    u = uniform(rows, N + 1)
    rng = np.random.RandomState(N)
    t = rng.choice([0.3, 0.7, 1.0, 1.5, 4.0], rows)
    k = rng.choice([0, 1, 2, 5, 50, 500, N - 1, N, N + 7], rows)
    p = rng.choice([0.0, 0.01, 0.5, 0.9, 0.95, 0.999, 0.99999994, 1.0, 2.0], rows)
    m = rng.choice([0.0, 1e-30, 1e-6, 0.01, 0.1, 0.5, 1.0, 1.5], rows)
    check(M, x, u, what="nothing set")
    check(M, x, u, t=t, what="temperature")
    check(M, x, u, t=t, k=k, what="top-k")
    check(M, x, u, t=t, p=p, what="top-p")
    check(M, x, u, t=t, m=m, what="min-p")
    check(M, x, u, t=t, k=k, p=p, m=m, what="all")
    check(M, x, u, t=np.zeros(rows), k=k, p=p, m=m, what="greedy")


def test_greedy_is_the_argmax(M):
    x = logits(40, 32000, "bf16", 3)
    ids, _ = M.bctm_sample(x, torch.zeros(40, device="cuda"), temperature=torch.zeros(40, device="cuda"))
    assert torch.equal(ids, M.bctm_argmax(x.contiguous()))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_equal_logits(M, dtype):
    """Rows of one value, of two, of few: ties go to the lowest index, and the border between two tokens is exact."""
    rows, N = 16, 4096
    u = np.arange(rows) / rows
    for v in (0.0, -0.0, 3.5, -1e30):
        ids = check(M, torch.full((rows, N), v, dtype=DT[dtype], device="cuda"), u, what=f"all {v}")
        assert np.array_equal(ids, np.arange(rows) * (N // rows))     # u * N exactly: the token after those below it
    x = torch.zeros((rows, N), dtype=DT[dtype], device="cuda")
    x[:, ::2] = -0.0                                                  # zeros of both signs are one value
    check(M, x, u, what="zeros of both signs")
    check(M, x, u, k=100, p=0.5, what="ties cut by top-k and top-p")
    x = (torch.randint(0, 3, (rows, N), generator=torch.Generator().manual_seed(1)) * 0.75).to(DT[dtype]).cuda()
    for k in (0, 1, 700, 1400, 2000, 4000):
        check(M, x, u, k=k, p=0.8, m=0.3, what=f"three values, k={k}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_masks_infinities_and_nan(M, dtype):
    rows, N = 12, 5003
    x = logits(rows, N, dtype, 5).contiguous()
    inf, nan = float("inf"), float("nan")
    x[0] = -inf                      # nothing left
    x[1] = nan
    x[2] = -inf
    x[2, 4711] = -7.0                # one left
    x[3, ::2] = -inf
    x[4, 5::3] = nan
    x[5, 17] = inf                   # an infinity takes all
    x[6, [5, 900, 5002]] = inf       # three of them share
    x[7] = torch.finfo(DT[dtype]).min   # the type's lowest value as a mask
    x[7, 100:110] = 1.0
    x[8] = torch.finfo(DT[dtype]).min   # the lowest value everywhere is a row like any other
    x[9] = -inf
    x[9, 1::2] = nan
    x[10, 0] = torch.finfo(DT[dtype]).max
    x[11] *= 1e-38
    for t in (1.0, 0.0, 0.01, 100.0):
        for kw in ({}, dict(k=3), dict(p=0.6), dict(m=0.2), dict(k=40, p=0.9, m=0.01)):
            ids = check(M, x, uniform(rows, 6), t=t, what=f"t={t} {kw}", **kw)
            assert ids[0] == ids[1] == ids[9] == -1 and ids[2] == 4711 and ids[5] == 17


def test_settings_out_of_range(M):
    """u outside [0, 1), NaN settings: as documented, never another token than one that is kept."""
    nan, inf = float("nan"), float("inf")
    x = logits(8, 1000, "bf16", 9)
    check(M, x, [0.0, -1.0, nan, 1.0, 2.0, inf, -inf, 1 - 2.0 ** -24], k=10, what="u")
    u = uniform(8, 10)
    check(M, x, u, t=[nan, -1.0, 0.0, 1e-40, 1e-20, 1e20, 3e38, inf], what="temperature")
    check(M, x, u, k=[-5, -2 ** 31, 2 ** 31 - 1, 0, 1, 999, 1000, 1001], what="top_k")
    check(M, x, u, p=[nan, -1.0, 0.0, 1e-40, 1e-20, 1.0, inf, 1 - 2.0 ** -24], what="top_p")
    check(M, x, u, m=[nan, -1.0, 0.0, 1e-40, 1e-20, 1.0, inf, 1.0000001], what="min_p")


def test_wide_ranges_of_logits(M):
    """Values whose keys are far apart within one bin of weights (a high temperature, values around zero)."""
    g = torch.Generator().manual_seed(11)
    e = torch.randint(-30, 5, (16, 20000), generator=g).float()
    x = (torch.randn((16, 20000), generator=g) * torch.exp2(e)).cuda()
    for t in (0.5, 1.0, 50.0, 1e4):
        check(M, x, uniform(16, 12), t=t, p=0.7, what=f"fp32, t={t}")
        check(M, x.bfloat16(), uniform(16, 12), t=t, k=5000, p=0.7, what=f"bf16, t={t}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,ld,at", [(32000, 32016, 0), (32000, 32001, 0), (999, 1003, 0), (1000, 1024, 3), (4097, 4104, 1)])
def test_padded_and_unaligned_rows(M, N, ld, at, dtype):
    """Rows at a distance, rows that start anywhere: what lies between is not read as a logit."""
    x = torch.full((9, ld + at), 1e4, dtype=DT[dtype], device="cuda")
    x[:, at:at + N] = logits(9, N, dtype, ld)
    check(M, x[:, at:at + N], uniform(9, 1), k=1000, p=0.97, m=1e-4, what=f"{N} of {ld} from {at}")


def test_many_rows_and_repeats(M):
    """A row's token does not depend on the other rows or on the call."""
    x, u = logits(700, 2000, "bf16", 13), torch.tensor(uniform(700, 14)).cuda()
    p = torch.full((700,), 0.9, device="cuda")
    ids, prob = M.bctm_sample(x, u, top_p=p, prob=True)
    check(M, x, u.cpu().numpy(), p=0.9, what="700 rows")
    for at, n in ((0, 1), (13, 7), (699, 1), (100, 300)):
        s = slice(at, at + n)
        a, b = M.bctm_sample(x[s], u[s].contiguous(), top_p=p[s].contiguous(), prob=True)
        assert torch.equal(a, ids[s]) and torch.equal(b, prob[s])


@pytest.mark.parametrize("N", [(1 << 18) + 5, (1 << 22) - 3])
def test_very_wide_vocabularies(M, N):
    x = logits(2, N, "f32", 15)
    check(M, x, [0.3, 0.999], t=1.3, p=0.99, what="top-p")
    check(M, torch.zeros((2, N), device="cuda"), [0.25, 0.75], what="equal")


def test_distribution(M):
    """Evenly spaced numbers draw every kept token as often as its probability says (to one of the spacing)."""
    n = 4096
    x = logits(1, 50, "f32", 16).expand(n, 50).contiguous()
    u = (torch.arange(n, device="cuda", dtype=torch.float32) + 0.5) / n
    ids, _ = M.bctm_sample(x, u, top_k=torch.full((n,), 10, dtype=torch.int32, device="cuda"))
    w = torch.exp(x[0].double() - x[0].double().max())
    w[w < torch.sort(w, descending=True)[0][9]] = 0
    got = torch.bincount(ids.long(), minlength=50).double()
    assert torch.all((got - n * w / w.sum()).abs() <= 1.001)


def test_another_stream_and_a_captured_graph(M):
    x, u = logits(32, 32000, "bf16", 17).contiguous(), torch.tensor(uniform(32, 18)).cuda()
    t = torch.full((32,), 0.8, device="cuda")
    p = torch.full((32,), 0.95, device="cuda")
    want, _ = M.bctm_sample(x, u, t, top_p=p)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got, _ = M.bctm_sample(x, u, t, top_p=p)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)
    out, g = torch.empty_like(want), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        M.bctm_sample(x, u, t, top_p=p, out=out)
    for step in range(4):
        u.copy_(torch.tensor(uniform(32, 19 + step)))
        x.add_(torch.tensor(0.01 * step).bfloat16().cuda())
        want, _ = M.bctm_sample(x, u, t, top_p=p)
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want), step


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N", [65535, 65536, 65537, 131071, 131080, 200003])
def test_one_value_of_many_tokens(M, N, dtype):
    """A value that occurs in nearly all of a long row, beside others: counts around 65536, of the even and the odd of two
    values next to each other, and both."""
    rows = 6
    x = torch.full((rows, N), 1.0, dtype=DT[dtype], device="cuda")
    nxt = 1.0 + torch.finfo(DT[dtype]).eps
    x[1] = nxt
    x[2, : N // 2] = nxt
    x[3, ::7] = 4.0
    x[4] = -2.0
    x[4, N - 1] = 3.0
    x[5] = logits(1, N, dtype, N)[0]
    x[5, ::2] = 0.0
    u = np.array([0.9999, 0.5, 0.7, 0.99, 0.999, 0.6])
    check(M, x, u, what="plain")
    check(M, x, u, k=N // 3, p=0.9, m=1e-3, what="all settings")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N", [4095, 4096, 4097, 8192, 8200, 16383, 16384, 16391, 24577, 32767, 32768, 32769, 32776, 40001, 49152, 49153])
def test_rows_that_fill_their_registers_or_do_not(M, N, dtype):
    """Rows around the numbers of vectors a thread can hold: the last vector there, missing, or one token of it."""
    rows = 6
    x, u = logits(rows, N, dtype, N + 3), uniform(rows, N + 4)
    x[:, -1] = x[:, 0]                       # a likely token at the end
    check(M, x, u, t=0.9, what="temperature")
    check(M, x, u, t=0.9, k=N // 2, p=0.97, m=1e-7, what="all")
    check(M, x, np.full(rows, 0.99999994), t=3.0, what="the far end")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N", [1000, 20011, 131072, 131085])
def test_weights_over_the_whole_range_of_the_type(M, N, dtype):
    """Temperatures at which logits of both signs and of magnitudes from 1 to 1e38 all have weights: more values than are counted
    at a time (36864 of bf16), thresholds on either side of that border, ties there, and masked tokens beside them."""
    rows = 12
    g = torch.Generator().manual_seed(N)
    near = torch.tensor([1.0, -1.0, 0.0, 1e5, -1e5, -3e9, -3e10, -1e11, -2e11, -1e20])
    far = torch.tensor([3e38, 1e38, -1e38, -2e38, 1e30, -1e30, 1e-3, -1e-3, -3e38, 1e38])
    pick = torch.randint(0, 10, (rows, N), generator=g)
    x = torch.where(torch.arange(rows)[:, None] % 2 == 0, near[pick] * (0.5 + torch.rand((rows, N), generator=g)),
                    far[pick] * (0.25 + 0.75 * torch.rand((rows, N), generator=g)))
    x[2, x[2] > 0] *= 1e-5                     # the largest value next to 1
    x[4] = near[pick[4]]                       # few values, each of many tokens
    x[5] = far[pick[5]]
    x[6:9, ::3] = -float("inf")
    x[7, 1::5] = float("nan")
    x = x.to(DT[dtype]).cuda()
    t = np.array([1e10, 1e37, 3e10, 1e38, 1e11, 3e38, 1e20, 5e37, 1e12, 2e37, 1e21, np.inf], np.float32)
    k = np.array([N // 2, 1, 7 * N // 10, 9 * N // 10, N // 3, N // 4, N // 2, N // 3, 5, N - 3, 8 * N // 10, N // 2])
    p = np.array([0.3, 0.7, 0.9, 0.95, 0.6, 0.8, 0.99, 0.4, 0.85, 0.999, 0.2, 0.65])
    m = np.array([0.9, 0.2, 0.5, 0.01, 1e-6, 0.3, 0.99, 0.05, 1e-9, 0.7, 0.999, 0.1])
    for s, u in enumerate((uniform(rows, N + 1), uniform(rows, N + 2) * 0.05, 1.0 - 0.05 * uniform(rows, N + 3))):
        check(M, x, u, t=t, what=f"temperature {s}")
        check(M, x, u, t=t, k=k, what=f"top-k {s}")
        check(M, x, u, t=t, p=p, what=f"top-p {s}")
        check(M, x, u, t=t, m=m, what=f"min-p {s}")
        check(M, x, u, t=t, k=k, p=p, m=m, what=f"all {s}")
        check(M, x, u, t=np.roll(t, 2), k=np.roll(k, 1), p=np.roll(p, 3), m=np.roll(m, 4), what=f"all, others {s}")
