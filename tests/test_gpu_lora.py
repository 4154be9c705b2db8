"""bctm_linear_lora, bctm_linear_split_lora, bctm_swiglu_lora against their formula in 64 bits.

Tolerance of a projection's output y: one rounding to bf16, 2^-8 |y|; fp32 sums, 2^-20 of the sum of the products' absolute
values (as for the projections without adapters); t = scale x A^T enters the second product with what two bf16 roundings
leave, 2^-16 of it at most, and its own fp32 sum: (2^-16 + 2^-20) * scale * (|x| |A|^T) |B|^T.  SwiGLU: the slacks of gate and
up through silu(g) u, whose derivatives are at most 1.1 |u| and |g| + 1."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def M():
    from paper_2411_15785_amd import model
    model.mlib()
    return model


class Case:
    def __init__(self, rows, K, N, rank, n, segments=1, mats=1, scale=True, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed + 7 * rows + K + N + rank)
        r = lambda *s, std=1.0: (torch.randn(s, generator=g, device="cuda") * std).bfloat16()
        self.rows, self.K, self.N, self.rank, self.n = rows, K, N, rank, n
        self.x = r(rows, K)
        self.w = [r(N, K, std=K ** -0.5) for _ in range(mats)]
        self.a, self.b = r(n, segments, rank, K, std=K ** -0.5), [r(n, N, rank, std=rank ** -0.5) for _ in range(mats)]
        self.scale = 0.25 + torch.rand(n, generator=g, device="cuda") if scale else None
        self.res = r(rows, N)

    def pack(self, M):
        return [M.bctm_pack_weight(w) for w in self.w], M.bctm_lora_pack(self.a, self.b, self.scale)

    def product(self, ids, mat, segment_of, cols):
        """The projection of these features in float64, and its slack.  segment_of: feature -> segment of A."""
        x, w = self.x.double(), self.w[mat][cols].double()
        y, mass = x @ w.T, x.abs() @ w.abs().T
        for i in range(self.n):
            at = torch.nonzero(ids == i)[:, 0]
            if at.numel() == 0:
                continue
            s = float(self.scale[i]) if self.scale is not None else 1.0
            for seg in range(self.a.shape[1]):
                f = torch.nonzero(segment_of[cols] == seg)[:, 0]
                if f.numel() == 0:
                    continue
                a, b = self.a[i, seg].double(), self.b[mat][i][cols][f].double()
                y[at[:, None], f] += s * ((x[at] @ a.T) @ b.T)
                # 17 times: 2^-16 + 2^-20 in units of 2^-20
                mass[at[:, None], f] += 18 * s * ((x[at].abs() @ a.abs().T) @ b.abs().T)
        return y, mass * 2.0 ** -20


def close(got, want, slack, what):
    err, tol = (got.double() - want).abs(), 2.0 ** -8 * want.abs() + slack
    assert bool((err <= tol).all()), f"{what}: worst {(err / tol).max().item():.2f} of the tolerance, " \
                                     f"{int((err > tol).sum())} of {err.numel()} beyond"


def some(N, width=320):
    """All features, or the first, middle and last ones of a wide projection."""
    if N <= 3 * width:
        return torch.arange(N, device="cuda")
    at = [0, (N // 2 - width // 2) // 16 * 16 + 5, N - width]
    return torch.cat([torch.arange(s, s + width, device="cuda") for s in at])


def adapters(rows, n, seed, run=1):
    """Ids with some below and some beyond the adapters."""
    g = torch.Generator().manual_seed(seed)
    ids = torch.randint(-1, n + 1, ((rows + run - 1) // run,), generator=g).repeat_interleave(run)[:rows]
    ids[ids == n] = torch.where(torch.rand(int((ids == n).sum()), generator=g) < 0.5, n, 2 ** 31 - 1)
    return ids.to(torch.int32).cuda().contiguous()


def same(a, b):
    return torch.equal(a.view(torch.int16), b.view(torch.int16))


# rows, K, N, rank, adapters, consecutive rows of one request
SHAPES = [
    # streaming: one and two row tiles, one to three feature tiles a workgroup, few K steps and uneven shares of them
    (1, 32, 16, 16, 1, 1), (3, 64, 96, 8, 2, 1), (16, 320, 48, 16, 40, 1), (17, 2336, 160, 33, 5, 1), (32, 4096, 256, 16, 32, 1),
    (33, 96, 16416, 64, 3, 1), (9, 96, 12288, 32, 9, 1), (70, 1024, 12336, 16, 100, 1), (127, 512, 64, 256, 7, 1), (100, 64, 128, 1, 3, 40),
    # the matrix-core kernel's tiles: 64 x 64, 128 x 64 and 128 x 128 with K in two, 128 x 128, 128 x 256, 256 x 256, 128 x 512
    (128, 32, 128, 16, 2, 1), (130, 320, 256, 48, 60, 1), (257, 160, 400, 16, 9, 30), (320, 512, 4096, 32, 12, 11), (640, 160, 4096, 64, 3, 200),
    (1030, 96, 4224, 16, 300, 1), (1030, 160, 4096, 128, 5, 129), (1000, 64, 32768, 16, 4, 100), (557, 160, 23552, 32, 17, 7), (2050, 96, 512, 8, 3, 1000),
    # four row tiles a workgroup in the first half, K whole and in parts
    (2075, 4096, 64, 48, 9, 60), (2300, 64, 256, 64, 5, 1), (2049, 1088, 128, 100, 20, 7),
]


def test_shapes_cover_every_tile(M):
    tiles = {M.bctm_linear_tile(r, K, N, tiled=True) for r, K, N, *_ in SHAPES}
    assert tiles >= {(16, 16, 16), (32, 16, 16), (32, 32, 8), (16, 48, 8), (32, 48, 8), (64, 64, 2), (128, 64, 2), (128, 128, 2), (128, 128, 1),
                     (128, 256, 1), (256, 256, 1), (128, 512, 1)}


@pytest.mark.parametrize("rows,K,N,rank,n,run", SHAPES)
def test_linear(M, rows, K, N, rank, n, run):
    c = Case(rows, K, N, rank, n)
    (w,), lora = c.pack(M)
    ids = adapters(rows, n, rows + N, run)
    cols = some(N)
    y, slack = c.product(ids, 0, torch.zeros(N, device="cuda"), cols)
    out = M.bctm_linear_lora(c.x, w, lora, ids)
    close(out[:, cols], y, slack, "linear")
    tiled = M.bctm_pack_rows(c.x)
    if M.bctm_linear_tile(rows, K, N) == M.bctm_linear_tile(rows, K, N, tiled=True):
        assert same(M.bctm_linear_lora(tiled, w, lora, ids), out)
    else:
        close(M.bctm_linear_lora(tiled, w, lora, ids)[:, cols], y, slack, "linear, tiled x")
    r = c.res.clone()
    got = M.bctm_linear_lora(c.x, w, lora, ids, r, out=r)           # residual in place
    assert got is r
    close(r[:, cols], y + c.res[:, cols].double(), slack + 2.0 ** -20 * c.res[:, cols].double().abs(), "linear with residual")
    # rows without an adapter: the plain projection's bits
    none = (ids < 0) | (ids >= n)
    assert same(out[none], M.bctm_linear(c.x, w)[none]) and same(r[none], M.bctm_linear(c.x, w, c.res)[none])
    off = torch.full_like(ids, -1)
    assert same(M.bctm_linear_lora(c.x, w, lora, off), M.bctm_linear(c.x, w))


@pytest.mark.parametrize("rows,K,widths,rank,n,run", [
    (5, 64, (32, 16, 48), 16, 3, 1), (32, 4096, (4096, 4096, 4096), 16, 32, 1), (20, 96, (6144, 6144), 32, 4, 1),
    (300, 96, (112, 80, 64), 24, 6, 25), (640, 288, (4096, 1024, 1024), 16, 20, 31), (1030, 96, (4112, 96, 144), 64, 3, 100),
    (557, 64, (11792, 256, 11504), 16, 9, 1), (1000, 64, (16400, 16368), 48, 2, 333),
    # three outputs within 64 features
    (300, 96, (48, 16, 64), 16, 5, 7), (1030, 64, (16, 32, 4048), 48, 6, 21), (40, 64, (16, 16, 16), 40, 3, 1), (2100, 96, (272, 16, 480), 32, 9, 45)])
def test_split(M, rows, K, widths, rank, n, run):
    """Each output has an A of its own; borders between outputs inside and between the workgroups' tiles."""
    N = sum(widths)
    c = Case(rows, K, N, rank, n, segments=len(widths), scale=rows % 2 == 0)
    (w,), lora = c.pack(M)
    ids = adapters(rows, n, rows + N, run)
    seg = torch.cat([torch.full((v,), i, device="cuda") for i, v in enumerate(widths)])
    cols = torch.unique(torch.cat([some(N, 160)] + [torch.arange(max(0, e - 40), min(N, e + 40), device="cuda") for e in np.cumsum(widths)]))
    y, slack = c.product(ids, 0, seg, cols)
    outs = [torch.empty((rows, v), dtype=torch.bfloat16, device="cuda") for v in widths]
    for x in (c.x, M.bctm_pack_rows(c.x)):
        M.bctm_linear_split_lora(x, w, lora, ids, outs)
        close(torch.cat(outs, 1)[:, cols], y, slack, "split")
    plain = [torch.empty_like(o) for o in outs]
    M.bctm_linear_split(M.bctm_pack_rows(c.x), w, plain)
    none = (ids < 0) | (ids >= n)
    assert all(same(o[none], p[none]) for o, p in zip(outs, plain))


@pytest.mark.parametrize("rows,K,N,rank,n,run", [
    (1, 32, 32, 16, 1, 1), (16, 4096, 352, 16, 16, 1), (33, 96, 64, 40, 5, 1), (127, 320, 96, 64, 2, 50), (128, 96, 64, 16, 128, 1),
    (300, 160, 480, 32, 3, 70), (640, 64, 11008, 16, 5, 100), (1100, 96, 2112, 16, 70, 13), (2048, 64, 11008, 32, 4, 512), (557, 160, 11776, 16, 6, 20)])
def test_swiglu(M, rows, K, N, rank, n, run):
    c = Case(rows, K, N, rank, n, segments=2, mats=2)
    (wg, wu), lora = c.pack(M)
    ids = adapters(rows, n, rows + N, run)
    cols = some(N)
    g, sg = c.product(ids, 0, torch.zeros(N, device="cuda"), cols)
    u, su = c.product(ids, 1, torch.ones(N, device="cuda"), cols)
    want = g / (1.0 + torch.exp(-g)) * u
    slack = 1.1 * sg * u.abs() + (g.abs() + 1.0) * su + 2.0 ** -20 * (g * u).abs()
    out = M.bctm_swiglu_lora(c.x, wg, wu, lora, ids)
    close(out[:, cols], want, slack, "swiglu")
    xt = M.bctm_pack_rows(c.x)
    close(M.bctm_swiglu_lora(xt, wg, wu, lora, ids)[:, cols], want, slack, "swiglu, tiled x")
    none = (ids < 0) | (ids >= n)
    assert same(out[none], M.bctm_swiglu(c.x, wg, wu)[none])
    # a tiled output is the row-major one, packed
    t = M.bctm_swiglu_lora(xt, wg, wu, lora, ids, tiled=True)
    back = M.bctm_pack_rows(M.bctm_swiglu_lora(xt, wg, wu, lora, ids))
    full = rows // 32 * 32 * N
    assert same(t.data[:full], back.data[:full])


@pytest.mark.parametrize("rows,K,N", [(32, 256, 96), (300, 256, 512), (1030, 64, 4096)])
def test_an_adapter_reaches_its_own_rows_alone(M, rows, K, N):
    """NaN and infinities in one adapter's weights, in one row's activations, in the workspace."""
    n, rank = 4, 32
    c = Case(rows, K, N, rank, n)
    (w,), lora = c.pack(M)
    ids = (torch.arange(rows, device="cuda") * 7 % (n + 1) - 1).to(torch.int32)
    ws = torch.full((lora.workspace_bytes(rows),), 0xFF, dtype=torch.uint8, device="cuda")    # NaNs
    want = M.bctm_linear_lora(c.x, w, lora, ids, workspace=ws)
    assert not torch.isnan(want).any()
    for value in (float("nan"), float("inf"), -float("inf")):
        for where in ("a", "b"):
            a, b = c.a.clone(), c.b[0].clone()
            (a if where == "a" else b)[2] = value
            got = M.bctm_linear_lora(c.x, w, M.bctm_lora_pack(a, b, c.scale), ids, workspace=ws)
            assert same(got[ids != 2], want[ids != 2]) and not torch.isfinite(got[ids == 2]).any(), (value, where)
        x = c.x.clone()
        x[rows // 2] = value
        got = M.bctm_linear_lora(x, w, lora, ids, workspace=ws)
        keep = torch.arange(rows, device="cuda") != rows // 2
        assert same(got[keep], want[keep])


@pytest.mark.parametrize("rows", [4, 160])
def test_an_infinity_stays_one(M, rows):
    """Positive throughout, and one entry of A infinite: so are its outputs, with one addend of t (few rows) or two."""
    K, N, rank = 64, 128, 16
    g = torch.Generator(device="cuda").manual_seed(rows)
    r = lambda *s: (torch.rand(s, generator=g, device="cuda") + 0.5).bfloat16()
    x, w, a, b = r(rows, K), M.bctm_pack_weight(r(N, K)), r(2, rank, K), r(2, N, rank)
    a[1, 3, 5] = float("inf")
    ids = (torch.arange(rows, device="cuda") // 16 % 2).to(torch.int32)
    ids[::7] = 1
    out = M.bctm_linear_lora(x, w, M.bctm_lora_pack(a, b), ids).float()
    assert bool((out[ids == 1] == float("inf")).all()) and bool(torch.isfinite(out[ids == 0]).all())


@pytest.mark.parametrize("rows,K,rank", [(1, 4096, 16), (40, 4096, 16), (300, 2048, 64), (2047, 4096, 16), (2048, 4096, 64), (2100, 512, 240),
                                         (4100, 2048, 33)])
def test_the_workspace_is_not_left(M, rows, K, rank):
    """What lies behind the workspace stays as it was, and one of more rows serves as well."""
    c = Case(rows, K, 32, rank, 3)
    (w,), lora = c.pack(M)
    ids = adapters(rows, 3, rows, 5)
    n = lora.workspace_bytes(rows)
    ws = torch.full((n + 4096,), 0x5A, dtype=torch.uint8, device="cuda")
    out = M.bctm_linear_lora(c.x, w, lora, ids, workspace=ws[:n])
    assert bool((ws[n:] == 0x5A).all())
    assert same(out, M.bctm_linear_lora(c.x, w, lora, ids, workspace=torch.empty(lora.workspace_bytes(5000), dtype=torch.uint8, device="cuda")))


def test_one_weight_at_a_time_selects_the_right_operands(M):
    """A and B with a single one each: the output is that entry alone, at every place of the packed layouts."""
    rows, K, N, rank, n = 20, 64, 48, 32, 3
    x = torch.zeros((rows, K), dtype=torch.bfloat16, device="cuda")
    x[:] = torch.arange(1, K + 1, device="cuda").bfloat16()
    w = M.bctm_pack_weight(torch.zeros((N, K), dtype=torch.bfloat16, device="cuda"))
    ids = (torch.arange(rows, device="cuda") % n).to(torch.int32)
    for j in range(0, rank, 3):
        for k, f in ((j * 2 % K, j % N), ((5 * j + 1) % K, (7 * j + 17) % N)):
            a = torch.zeros((n, rank, K), dtype=torch.bfloat16, device="cuda")
            b = torch.zeros((n, N, rank), dtype=torch.bfloat16, device="cuda")
            a[:, j, k] = 1.0
            for i in range(n):
                b[i, f, j] = i + 1.0
            out = M.bctm_linear_lora(x, w, M.bctm_lora_pack(a, b), ids).float()
            want = torch.zeros((rows, N), device="cuda")
            want[:, f] = (k + 1.0) * (ids + 1).float()
            assert torch.equal(out, want), (j, k, f)


def test_rows_do_not_depend_on_their_neighbours(M):
    """Many adapters in any order: each row is that of a call whose other rows have other adapters or none."""
    rows, K, N, n = 48, 512, 320, 48
    c = Case(rows, K, N, 16, n)
    (w,), lora = c.pack(M)
    ids = torch.randperm(n, generator=torch.Generator().manual_seed(1)).to(torch.int32).cuda()
    out = M.bctm_linear_lora(c.x, w, lora, ids)
    for r in (0, 15, 16, 31, 47):
        other = torch.full_like(ids, -1)
        other[r] = ids[r]
        assert same(M.bctm_linear_lora(c.x, w, lora, other)[r], out[r])
        other = torch.full_like(ids, int(ids[r]))
        assert same(M.bctm_linear_lora(c.x, w, lora, other)[r], out[r])


def test_streams_and_a_captured_graph(M):
    rows, K, N, n = 32, 1024, 768, 8
    c = Case(rows, K, N, 16, n, segments=3)
    (w,), lora = c.pack(M)
    ids = adapters(rows, n, 3)
    outs = [torch.empty((rows, 256), dtype=torch.bfloat16, device="cuda") for _ in range(3)]
    want = [o.clone() for o in M.bctm_linear_split_lora(c.x, w, lora, ids, outs)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        M.bctm_linear_split_lora(c.x, w, lora, ids, outs)
    torch.cuda.current_stream().wait_stream(side)
    assert all(same(a, b) for a, b in zip(outs, want))
    # two graphs, each with a workspace that torch gives it; replayed in turn with eager calls between
    graphs = []
    for k in range(2):
        o, g = [torch.empty_like(t) for t in outs], torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            M.bctm_linear_split_lora(c.x, w, lora, ids, o)
        graphs.append((g, o))
    for step in range(4):
        ids.copy_(adapters(rows, n, 10 + step))
        c.x.mul_(0.5 if step % 2 else 2.0)
        want = [t.clone() for t in M.bctm_linear_split_lora(c.x, w, lora, ids, outs)]
        for g, o in graphs:
            for t in o:
                t.zero_()
            g.replay()
        torch.cuda.synchronize()
        for g, o in graphs:
            assert all(same(a, b) for a, b in zip(o, want)), step


def test_refusals(M):
    c = Case(4, 64, 32, 16, 2)
    (w,), lora = c.pack(M)
    ids = torch.zeros(4, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        M.bctm_linear_lora(c.x, w, lora, ids.long())
    with pytest.raises(ValueError):
        M.bctm_linear_lora(c.x, w, lora, ids[:3])
    with pytest.raises(ValueError):
        M.bctm_linear_lora(c.x, w, lora, ids.cpu())
    with pytest.raises(ValueError):
        M.bctm_swiglu_lora(c.x, w, w, lora, ids)                     # adapters of a plain projection
    with pytest.raises(ValueError):
        M.bctm_linear_lora(c.x, w, (c.a, c.b), ids)                  # not packed
    with pytest.raises(ValueError):
        M.bctm_linear_lora(c.x, M.bctm_pack_weight(torch.zeros((48, 64), dtype=torch.bfloat16, device="cuda")), lora, ids)
    with pytest.raises(ValueError):
        M.bctm_lora_pack(c.a, [torch.zeros((2, 32, 8), dtype=torch.bfloat16, device="cuda")])   # another rank
    with pytest.raises(M.BctModelError) as e:
        M.bctm_linear_lora(c.x, w, lora, ids, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    assert e.value.status == 3
    with pytest.raises(M.BctModelError):
        M.bctm_lora_pack(torch.zeros((1, 272, 64), dtype=torch.bfloat16, device="cuda"),
                         torch.zeros((1, 32, 272), dtype=torch.bfloat16, device="cuda"))        # rank beyond 256


@pytest.mark.parametrize("form,rows,K,N,rank", [
    ("linear", 130, 320, 256, 48), ("linear", 300, 1024, 512, 16), ("linear", 1030, 160, 4096, 32), ("linear", 557, 160, 23552, 32),
    ("linear", 640, 160, 4096, 64), ("linear", 1000, 64, 32768, 16), ("linear", 2075, 4096, 64, 48), ("split", 300, 96, 384, 24),
    ("split", 1030, 96, 4224, 40), ("swiglu", 300, 160, 480, 32), ("swiglu", 2048, 64, 11008, 32), ("swiglu", 557, 160, 11776, 16)])
def test_a_row_of_many_does_not_depend_on_its_neighbours(M, form, rows, K, N, rank):
    """From 128 rows on: a row's bits are the same where all rows have its adapter, where its neighbours have others, and where
    they have none; K whole and in two, several outputs within a tile, the ragged last rows."""
    n = 7
    segments, mats = {"linear": (1, 1), "split": (3, 1), "swiglu": (2, 2)}[form]
    c = Case(rows, K, N, rank, n, segments=segments, mats=mats)
    ws, lora = c.pack(M)

    def run(ids):
        if form == "linear":
            return M.bctm_linear_lora(c.x, ws[0], lora, ids)
        if form == "swiglu":
            return M.bctm_swiglu_lora(c.x, *ws, lora, ids)
        return torch.cat(M.bctm_linear_split_lora(c.x, ws[0], lora, ids, [torch.empty((rows, v), dtype=torch.bfloat16, device="cuda")
                                                                           for v in (16, 48, N - 64)]), 1)

    full = lambda v: torch.full((rows,), v, dtype=torch.int32, device="cuda")
    uniform = [run(full(a)) for a in range(n)]
    plain = run(full(-1))
    mixed = adapters(rows, n, rows)
    inside = (mixed >= 0) & (mixed < n)
    got = run(mixed)
    for a in range(n):
        assert same(got[mixed == a], uniform[a][mixed == a]), a
    assert same(got[~inside], plain[~inside])
    # one row in 13, and one stretch of rows, among rows without an adapter
    alone = full(-1)
    alone[::13] = 3
    alone[100:140] = 5
    got = run(alone)
    for a in (3, 5):
        assert same(got[alone == a], uniform[a][alone == a]), a
    assert same(got[alone < 0], plain[alone < 0])


@pytest.mark.parametrize("rows,N", [(40, 64), (150, 64), (300, 512), (1030, 4096)])
@pytest.mark.parametrize("run", [1, 1000000])
def test_the_term_has_24_bits(M, rows, N, run):
    """The projection cancels the adapters' term but for the sums' roundings: W = -A for every feature, B = 1, all entries positive.  Both
    sums are fp32, within 2^-20 of the products' absolute values together (see above), 2 t; 16 bits of t would leave 2^-17 of it
    in places.  In one adapter's rows and in mixed tiles."""
    K, rank = 64, 16
    g = torch.Generator(device="cuda").manual_seed(rows)
    r = lambda *s: (torch.rand(s, generator=g, device="cuda") + 0.5).bfloat16()
    x, a0 = r(rows, K), r(K)
    a = torch.zeros((2, rank, K), dtype=torch.bfloat16, device="cuda")
    a[:, 5] = a0
    b = torch.zeros((2, N, rank), dtype=torch.bfloat16, device="cuda")
    b[:, :, 5] = 1.0
    w = M.bctm_pack_weight((-a0).expand(N, K).contiguous())
    ids = (torch.arange(rows, device="cuda") // run % 2).to(torch.int32)
    out = M.bctm_linear_lora(x, w, M.bctm_lora_pack(a, b), ids).double()
    t = x.double() @ a0.double()
    assert bool((out.abs() <= 2.0 ** -20 * 2 * t[:, None]).all()), (out.abs() / t[:, None]).max().item()


@pytest.mark.parametrize("form", ["linear", "swiglu"])
@pytest.mark.parametrize("rows,N,rank,K", [(4, 128, 16, 64), (40, 64, 8, 64), (160, 128, 40, 64), (300, 512, 1, 64), (1030, 4096, 33, 64),
                                           (4, 128, 8, 4096), (33, 96, 50, 4096), (100, 12288, 1, 4096)])
def test_infinities_are_those_of_the_formula(M, form, rows, N, rank, K):
    """Ranks filled up to a multiple of 16 and addends of t multiply nothing by zero that the formula does not.  Positive
    throughout: an infinite activation, an infinite entry of A and one of B each make infinities, and no NaN.  (An infinite
    activation that is a NaN in the plain projection of few rows already, which the header allows, is not looked at.)"""
    n, mats = 3, 2 if form == "swiglu" else 1
    g = torch.Generator(device="cuda").manual_seed(rows)
    r = lambda *s: (torch.rand(s, generator=g, device="cuda") + 0.5).bfloat16()
    x, w = r(rows, K), [M.bctm_pack_weight(r(N, K)) for _ in range(mats)]
    a, b = r(n, mats, rank, K), [r(n, N, rank) for _ in range(mats)]
    a[2, :, rank // 2, 5] = float("inf")
    for t in b:
        t[1, 7::10, rank - 1] = float("inf")
    bad = torch.arange(rows, device="cuda") % 5 == 3
    x[bad, 11] = float("inf")
    call = M.bctm_swiglu_lora if form == "swiglu" else M.bctm_linear_lora
    lora = M.bctm_lora_pack(a, b)
    looked_at = ~torch.isnan((M.bctm_swiglu if form == "swiglu" else M.bctm_linear)(x, *w).float())
    assert bool(looked_at.all()) or K == 64 and rows < 128
    for run in (1, 16, 400):      # tiles of several adapters and of one
        ids = (torch.arange(rows, device="cuda") // run % (n + 1) - 1).to(torch.int32)
        out = call(x, *w, lora, ids).float()
        inf = (bad | (ids == 2))[:, None].expand(rows, N).clone()
        inf[:, 7::10] |= (ids == 1)[:, None]
        assert torch.equal((out == float("inf"))[looked_at], inf[looked_at]) and not torch.isnan(out[looked_at]).any(), run


@pytest.mark.parametrize("rows,N", [(40, 64), (160, 128), (1030, 4096)])
@pytest.mark.parametrize("what", ["any", "few bits"])
def test_an_infinite_weight_takes_the_sign_of_its_product(M, rows, N, what):
    """t of either sign, with bits in all of its addends or in the first alone."""
    K, rank = 32, 16
    g = torch.Generator(device="cuda").manual_seed(N)
    x = torch.randn((rows, K), generator=g, device="cuda").bfloat16()
    a, b = torch.zeros((1, rank, K), dtype=torch.bfloat16, device="cuda"), torch.zeros((1, N, rank), dtype=torch.bfloat16, device="cuda")
    if what == "any":
        a[0, 3] = torch.randn(K, generator=g, device="cuda").bfloat16()
    else:
        a[0, 3, 9] = 0.5
        x[:, 9] = torch.where(x[:, 9] < 0, -1.0, 2.0)
    b[0, ::3, 3] = float("inf")
    b[0, 1::3, 3] = -float("inf")
    b[0, 2::3, 3] = 1.0
    t = (x.double() @ a[0, 3].double())
    w = M.bctm_pack_weight(torch.zeros((N, K), dtype=torch.bfloat16, device="cuda"))
    for ids in (torch.zeros(rows, dtype=torch.int32, device="cuda"), torch.arange(rows, device="cuda").to(torch.int32) % 2):
        out = M.bctm_linear_lora(x, w, M.bctm_lora_pack(a, b), ids).double()
        mine = ids == 0
        inf = torch.full_like(t, float("inf"))[:, None] * t.sign()[:, None]
        assert bool((out[mine][:, ::3] == inf[mine]).all()) and bool((out[mine][:, 1::3] == -inf[mine]).all())
        # one term of at most 32 products, rounded to bf16: 2^-8, and the sum's 2^-20 of the products' absolute values
        slack = 2.0 ** -8 * t.abs() + 2.0 ** -20 * (x.double().abs() @ a[0, 3].double().abs())
        assert bool(((out[mine][:, 2::3] - t[mine][:, None]).abs() <= slack[mine][:, None]).all())
        assert bool((out[~mine] == 0).all())


@pytest.mark.parametrize("N", [64, 128])          # the streaming kernel, the matrix cores
@pytest.mark.parametrize("rows,K,rank,n,run", [
    # two row tiles a workgroup in the first half, one to four column tiles; four row tiles, three and four of them
    (3101, 4128, 16, 5, 100), (3101, 4128, 25, 30, 1), (3100, 4128, 48, 6, 300), (13000, 992, 64, 9, 37), (3443, 11040, 48, 7, 50),
    (3443, 11040, 64, 4, 1000), (9002, 4224, 112, 20, 3)])
def test_row_tiles_of_the_first_half(M, rows, K, rank, n, run, N):
    c = Case(rows, K, N, rank, n)
    (w,), lora = c.pack(M)
    ids = adapters(rows, n, rows + N, run)
    cols = torch.arange(N, device="cuda")
    y, slack = c.product(ids, 0, torch.zeros(N, device="cuda"), cols)
    size = lora.workspace_bytes(rows)
    ws = torch.full((size + 4096,), 0x5A, dtype=torch.uint8, device="cuda")
    out = M.bctm_linear_lora(c.x, w, lora, ids, workspace=ws[:size])
    close(out, y, slack, "linear")
    assert bool((ws[size:] == 0x5A).all())
    close(M.bctm_linear_lora(M.bctm_pack_rows(c.x), w, lora, ids), y, slack, "linear, tiled x")
    none = (ids < 0) | (ids >= n)
    assert same(out[none], M.bctm_linear(c.x, w)[none])
