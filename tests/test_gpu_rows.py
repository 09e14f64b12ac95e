"""The row operators on the GPU against their float64 oracle."""
import numpy as np
import pytest

import rows_oracle as ro
from paper_1302_1700_amd import workloads as wl

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def fsb():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1302_1700_amd import fragscan
    fragscan.load()
    return fragscan


def _np(t):
    return t.detach().cpu().double().numpy()


# -- log probabilities ---------------------------------------------------------------
def _scores(rng, rows, V, dtype, kind):
    x = rng.normal(0, 3, (rows, V))
    if kind == "ties":
        x = rng.integers(-2, 3, (rows, V)) * 0.5
        x[rng.random((rows, V)) < 0.1] = -0.0
    elif kind == "peaks":            # a few classes hold nearly all of it, the row's ends among them
        for i in range(rows):
            x[i, [i % V, V - 1 - i % min(V, 3)]] += 40
    elif kind == "rising":           # every score is a new best one
        x = np.sort(x, 1)
    elif kind == "masked":
        x[rng.random((rows, V)) < 0.6] = -np.inf
        x[rows // 2] = -np.inf
        x[0] = torch.finfo(DT[dtype]).min
        if rows > 3:
            x[1, V // 2] = np.nan
            x[2, V - 1] = np.inf
            x[3] = -np.inf
            x[3, V - 1] = 5
    elif kind == "far":
        x = x + 3e4
    return torch.from_numpy(x).to(DT[dtype])


def _bounds(x, T, table, norm, V):
    """Half steps of float32: the difference to the maximum, its scaling by 1 / T and the exponential's argument
    (4 + 4 |ln p|), the exponential itself and the logarithm (2 each), and the sum's additions, in partial sums
    no longer than V / 32 + 64."""
    sums = V / 32 + 64
    d = np.abs(np.where(np.isfinite(table), table, 0)) + np.where(np.isfinite(norm[:, 1:]), norm[:, 1:], 0)
    mean = np.where(np.isfinite(table), np.exp(table) * d, 0).sum(1, keepdims=True)
    log_s = ro.U32 * (8 + sums + 6 * mean + 2 * np.abs(np.nan_to_num(norm[:, 1:])))
    return ro.U32 * (4 + 4 * d) + log_s, log_s


@pytest.mark.parametrize("kind", ["plain", "ties", "peaks", "rising", "masked", "far"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,V,n_top", [
    (1, 1, 1), (7, 2, 2), (1000, 3, 1), (333, 4, 4), (65, 7, 9), (130, 10, 3), (77, 16, 16), (50, 31, 5), (41, 64, 20),
    (33, 65, 64), (20, 129, 1), (19, 250, 7), (17, 511, 20), (16, 513, 33), (9, 1000, 64), (7, 2049, 5), (5, 4097, 20),
    (3, 16384, 64), (4, 49999, 5), (1, 70001, 20), (2, 131072, 64)])
def test_logprobs(fsb, dtype, rows, V, n_top, kind):
    rng = np.random.default_rng(rows * 7 + V)
    T = [1.0, 0.7, 1.5][(rows + V) % 3]
    x = _scores(rng, rows, V, dtype, kind)
    labels = rng.integers(-1, V, rows).astype(np.int32)
    if rows > 6:
        labels[4], labels[5] = V, 2 ** 31 - 1
    print("logprobs", dtype, rows, V, n_top, kind, flush=True)
    r = fsb.logprobs(x.cuda(), torch.from_numpy(labels).cuda(), n_top, T)
    torch.cuda.synchronize()
    T32 = 1.0 / float(np.float32(1.0) / np.float32(T))
    logp, ent, norm, ids, tops, table = ro.logprobs(_np(x), labels, n_top, T32)
    assert np.array_equal(r.top_id.cpu().numpy(), ids)
    each, log_s = _bounds(_np(x), T32, table, norm, V)
    ro.close(_np(r.norm)[:, 0], norm[:, 0], 0, "largest")
    ro.close(_np(r.norm)[:, 1:], norm[:, 1:], log_s, "log of the sum")
    has = (labels >= 0) & (labels < V)
    ro.close(_np(r.logp), logp, np.where(has, each[np.arange(rows), np.where(has, labels, 0)], 0), "logp")
    tb = np.where(ids >= 0, np.take_along_axis(each, np.maximum(ids, 0), 1), 0)
    ro.close(_np(r.top_logp), tops, tb, "top logp")
    # the entropy: the sum's bound, and each term's p d: the bound on d, twice (p is its exponential), with |ln p|
    p = np.where(np.isfinite(table), np.exp(table), 0)
    d = np.where(np.isfinite(table), np.abs(table), 0) + np.nan_to_num(norm[:, 1:], nan=0, neginf=0)
    terms = (p * d * (ro.U32 * (10 + 6 * d + V / 32 + 64))).sum(1) + (p * d).sum(1) * log_s[:, 0] * 2
    ro.close(_np(r.entropy), ent, terms + log_s[:, 0], "entropy")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [600, 8192, 50000, 131072])
@pytest.mark.parametrize("rows", [2, 700])
def test_best_classes_in_few_hands(fsb, dtype, V, rows):
    """Rows of one value, and rows whose best classes all lie where one thread reads (16 bytes of every 1024): equal
    ones, and more of them than a list holds."""
    n, period, width = 64, 1024 // (4 if dtype == "f32" else 2), 4 if dtype == "f32" else 8
    x = torch.zeros((rows, V), dtype=DT[dtype], device="cuda")
    j = torch.arange(V, device="cuda")
    few = (j % period) < width
    x[1::2, few] = 3.0
    if rows > 2:
        x[3::2, few] = (j[few] * 37 % 101).to(DT[dtype])
        x[2] = -float("inf")
        x[2, V - 1] = 1.0
    print("few hands", dtype, V, rows, flush=True)
    r = fsb.logprobs(x, n_top=n)
    torch.cuda.synchronize()
    want = x[:4].float().cpu().sort(stable=True, dim=1, descending=True)
    ids = want.indices[:, :n].int()
    ids[want.values[:, :n] == -float("inf")] = -1
    assert torch.equal(r.top_id[:4].cpu(), ids)
    assert torch.equal(r.top_id[0::2][2:], r.top_id[:1].expand_as(r.top_id[0::2][2:]))
    if rows > 4:
        assert torch.equal(r.top_id[3::2], r.top_id[3:4].expand_as(r.top_id[3::2]))


@pytest.mark.parametrize("kind", ["plain", "peaks", "masked", "far"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,V", [(1, 1), (1000, 2), (333, 4), (65, 7), (130, 10), (41, 64), (33, 65), (17, 513),
                                    (9, 1000), (7, 2049), (5, 4097), (3, 49999), (1, 131072)])
@pytest.mark.parametrize("which", ["logp", "entropy", "both"])
def test_logprobs_grad(fsb, dtype, rows, V, kind, which):
    rng = np.random.default_rng(rows * 5 + V)
    T = [1.0, 0.7, 1.5][(rows + V) % 3]
    x = _scores(rng, rows, V, dtype, kind)
    labels = rng.integers(-1, V, rows).astype(np.int32)
    if rows > 6:
        labels[4], labels[5] = V, 2 ** 31 - 1
    gl = rng.normal(0, 1, rows).astype(np.float32) if which != "entropy" else None
    ge = rng.normal(0, 1, rows).astype(np.float32) if which != "logp" else None
    print("logprobs_grad", dtype, rows, V, kind, which, flush=True)
    dev = lambda a: None if a is None else torch.from_numpy(a).cuda()
    T32 = 1.0 / float(np.float32(1.0) / np.float32(T))
    r = fsb.logprobs(x.cuda(), temperature=T)
    got = fsb.logprobs_grad(x.cuda(), r.norm, dev(labels) if gl is not None else None, dev(gl), r.entropy, dev(ge), T)
    place = x.cuda()
    same = fsb.logprobs_grad(place, r.norm, dev(labels) if gl is not None else None, dev(gl), r.entropy, dev(ge), T,
                             out=place)
    torch.cuda.synchronize()
    assert same is place and torch.equal(same.view(torch.int16 if dtype == "bf16" else torch.int32),
                                         got.view(torch.int16 if dtype == "bf16" else torch.int32))
    want = ro.logprobs_grad(_np(x), labels, T32, gl, ge)
    _, ent, norm, _, _, table = ro.logprobs(_np(x), None, 0, T32)
    each, log_s = _bounds(_np(x), T32, table, norm, V)
    p = np.where(np.isfinite(table), np.exp(table), 0)
    l = np.where(np.isfinite(table), np.abs(table), 0)
    e = np.nan_to_num(ent)[:, None]
    off = p * (each + 8 * ro.U32)                      # of p
    bound = np.zeros_like(want)
    if gl is not None:
        bound += np.abs(gl)[:, None] * (off + 4 * ro.U32 * (p + (np.arange(V) == labels[:, None])))
    if ge is not None:
        d = l + np.nan_to_num(norm[:, 1:], nan=0, neginf=0)
        e_off = ((p * d * (ro.U32 * (10 + 6 * d + V / 32 + 64))).sum(1) + (p * d).sum(1) * log_s[:, 0] * 2 + log_s[:, 0])[:, None]
        bound += np.abs(ge)[:, None] * (off * (l + e) + p * (each + e_off + 4 * ro.U32 * (l + e)))
    bound = bound / T32 + ro.UOUT[dtype] * np.abs(np.nan_to_num(want)) * 1.01 + 2.0 ** -133  # bf16's and float32's smallest steps
    ro.close(_np(got), want, bound, "gradient")


def test_logprobs_rows_of_a_view(fsb):
    """Rows at a stride, rows that start off any alignment, the same row many times, one row, a class map's shape."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    for dt in (torch.float32, torch.bfloat16):
        big = torch.randn((6, 5, 301), generator=gen, device="cuda").to(dt)
        for view in (big[:, :, 1:300], big[:, 3], big[2:3, 4:], big[0, 0, :77], big[0, :1, 5:6].expand(4, 1),
                     big[0, 0, 3:203].expand(9, 200), big[:, :, 7:9], big[:0]):
            rows = view.reshape(-1, view.shape[-1]).contiguous()
            y = torch.randint(0, view.shape[-1], view.shape[:-1], generator=gen, device="cuda", dtype=torch.int32)
            got, want = fsb.logprobs(view, y, 4), fsb.logprobs(rows, y.reshape(-1), 4)
            for g, w in zip(got, want):
                assert torch.equal(g.reshape(w.shape), w)
            if view.numel() == 0:
                continue
            gl = torch.randn(y.shape, generator=gen, device="cuda")
            out = torch.zeros((*view.shape[:-1], view.shape[-1] + 3), dtype=dt, device="cuda")
            g = fsb.logprobs_grad(view, got.norm, y, gl, out=out[..., 1:-2])
            w = fsb.logprobs_grad(rows, want.norm, y.reshape(-1), gl.reshape(-1))
            assert torch.equal(g.reshape(w.shape), w)
            assert (out[..., 0] == 0).all() and (out[..., -2:] == 0).all()   # nothing beside the rows is written


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_logprobs_far_rows(fsb, dtype):
    """A row whose elements lie beyond 2^31 from the first."""
    V, stride = 1000, (1 << 29) + 7
    store = torch.empty(5 * stride + V, dtype=DT[dtype], device="cuda")
    view = store.as_strided((6, V), (stride, 1))
    x = torch.randn((6, V), generator=torch.Generator(device="cuda").manual_seed(2), device="cuda").to(DT[dtype])
    view.copy_(x)
    y = torch.tensor([0, 1, -1, 999, 500, 7], dtype=torch.int32, device="cuda")
    got, want = fsb.logprobs(view, y, 3), fsb.logprobs(x, y, 3)
    for g, w in zip(got, want):
        assert torch.equal(g, w)
    gl = torch.ones(6, device="cuda")
    w = fsb.logprobs_grad(x, want.norm, y, gl)
    assert torch.equal(fsb.logprobs_grad(view, want.norm, y, gl, out=view), w)


# -- projection ----------------------------------------------------------------------
def _problem(seed, dtype, N, K, M, r, n, ids, bias=True, scale=True):
    gen = torch.Generator().manual_seed(seed)
    rnd = lambda *s: torch.randn(s, generator=gen)
    d = {"x": rnd(N, K).tanh().to(DT[dtype]), "w": (rnd(M, K) * K ** -0.5).to(DT[dtype]), "g": rnd(N, M).to(DT[dtype]),
         "bias": rnd(M) if bias else None, "a": None, "b": None, "scale": None, "ids": None}
    if n:
        d["a"], d["b"] = (rnd(n, r, K) * K ** -0.5).to(DT[dtype]), (rnd(n, M, r) * r ** -0.5).to(DT[dtype])
        d["scale"] = torch.rand(n, generator=gen) + 0.5 if scale else None
        if ids == "runs":
            d["ids"] = (torch.arange(N) * n // max(N, 1)).to(torch.int32)
        elif ids == "one":
            d["ids"] = torch.full((N,), n - 1, dtype=torch.int32)
        elif ids == "none":
            d["ids"] = torch.full((N,), -1, dtype=torch.int32)
        else:
            d["ids"] = torch.randint(-1, n + (ids == "bad"), (N,), generator=gen, dtype=torch.int32)
            if ids == "bad" and N > 2:
                d["ids"][N // 2], d["ids"][N - 1] = 2 ** 31 - 1, -2 ** 31
    return d


def _f64(d):
    return {k: None if v is None else (v.numpy() if k == "ids" else v.double().numpy()) for k, v in d.items()}


def _cuda(d):
    return {k: None if v is None else v.cuda() for k, v in d.items()}


def _adapters(fsb, c):
    return None if c["a"] is None else fsb.Adapters(c["a"], c["b"], c["scale"])


def _absolute(o):
    return {k: np.abs(v) if v is not None and k != "ids" else v for k, v in o.items()}


def _check(got, want, absum, n_terms, dtype, what):
    """Each value: a rounding of every term and every addition (n_terms + 16 half steps of the sum of absolute
    values, what a sum of n terms in any order is off by at most), one of the output.  All together: roundings
    of random sign add up like their square root; eight times that."""
    bound = (n_terms + 16) * ro.U32 * absum + 1.01 * ro.UOUT[dtype] * np.abs(np.nan_to_num(want)) + 2.0 ** -133
    ro.close(_np(got), want, bound, what)
    fine = np.isfinite(want)
    norm = np.linalg.norm(want[fine])
    if norm:
        off = np.linalg.norm(_np(got)[fine] - want[fine])
        size = np.linalg.norm(absum[fine])
        assert off <= 8 * ro.U32 * (n_terms + 16) ** 0.5 * size + ro.UOUT[dtype] * norm, (what, off / norm)


SHAPES = [  # rows, k, m, rank, adapters, ids
    (1, 1, 1, 1, 1, "one"), (1, 64, 33, 3, 2, "mixed"), (5, 7, 2, 4, 3, "mixed"), (17, 200, 2, 4, 3, "runs"),
    (300, 200, 2, 4, 3, "runs"), (257, 100, 4, 8, 5, "mixed"), (64, 128, 10, 1, 64, "mixed"), (130, 33, 65, 5, 7, "mixed"),
    (129, 256, 128, 16, 4, "runs"), (32, 512, 384, 16, 32, "mixed"), (16, 1024, 520, 64, 9, "bad"), (200, 96, 160, 128, 3, "mixed"),
    (515, 320, 260, 17, 6, "bad"), (513, 64, 1000, 8, 513, "mixed"), (1000, 24, 18, 2, 1, "bad"), (260, 130, 70, 32, 5, "none"),
    (129, 257, 131, 0, 0, None), (3, 300, 500, 0, 0, None), (2050, 40, 3, 6, 2, "mixed"), (1, 2048, 1024, 8, 4, "one"),
    (700, 512, 256, 16, 2, "one"), (384, 1000, 129, 33, 12, "runs")]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,K,M,r,n,ids", SHAPES)
def test_project(fsb, dtype, N, K, M, r, n, ids):
    print("project", dtype, N, K, M, r, n, ids, flush=True)
    d = _problem(N + K + M, dtype, N, K, M, r, n, ids, bias=N % 2 == 1, scale=K % 2 == 0)
    c, o = _cuda(d), _f64(d)
    out = fsb.project(c["x"], c["w"], c["bias"], _adapters(fsb, c), c["ids"], return_hidden=n > 0)
    y, h = out if n else (out, None)
    torch.cuda.synchronize()
    keys = ("x", "w", "bias", "a", "b", "scale", "ids")
    wy, wh = ro.project(*(o[k] for k in keys))
    ab = _absolute(o)
    ay, ah = ro.project(*(ab[k] for k in keys))
    _check(y, wy, np.nan_to_num(ay), K + r, dtype, "y")
    if n:
        _check(h, wh, np.nan_to_num(ah), K, "f32", "hidden")
        again = fsb.project(c["x"], c["w"], c["bias"], _adapters(fsb, c), c["ids"])
        assert torch.equal(again.view(torch.uint8), y.view(torch.uint8))   # without its hidden rows


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,K,M,r,n,ids", SHAPES + [(0, 20, 30, 4, 3, "mixed")])
def test_project_grad(fsb, dtype, N, K, M, r, n, ids):
    print("project_grad", dtype, N, K, M, r, n, ids, flush=True)
    d = _problem(N + K + M, dtype, N, K, M, r, n, ids, scale=M % 2 == 0)
    c, o = _cuda(d), _f64(d)
    ad = _adapters(fsb, c)
    gx, ga, gb = fsb.project_grad(c["g"], c["x"], c["w"], ad, c["ids"])
    torch.cuda.synchronize()
    keys = ("g", "x", "w", "a", "b", "scale", "ids")
    wx, wa, wb = ro.project_grad(*(o[k] for k in keys))
    ab = _absolute(o)
    ax, aa, abb = ro.project_grad(*(ab[k] for k in keys))
    _check(gx, wx, np.nan_to_num(ax), M + 2 * r, dtype, "gx")
    if not n:
        return
    _check(ga, wa, aa, N + M, dtype, "ga")
    _check(gb, wb, abb, N + K, dtype, "gb")
    if N:
        h = fsb.project(c["x"], c["w"], None, ad, c["ids"], return_hidden=True)[1]
        _, ha, hb = fsb.project_grad(c["g"], c["x"], c["w"], ad, c["ids"], hidden=h, need_x=False)
        assert torch.equal(ha, ga) and torch.equal(hb, gb)                # the same sums either way, every time
        only = fsb.project_grad(c["g"], c["x"], c["w"], ad, c["ids"], need_adapters=False)
        assert torch.equal(only[0].view(torch.uint8), gx.view(torch.uint8)) and only[1] is None
    unused = np.setdiff1d(np.arange(n), o["ids"])
    assert (ga[unused] == 0).all() and (gb[unused] == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_project_rows_of_a_view(fsb, dtype):
    """Rows, weights and outputs at strides and off every alignment; nothing beside the output's rows is written."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda").to(DT[dtype])
    for N, K, M, r, n in ((37, 50, 9, 3, 4), (140, 129, 200, 16, 3), (6, 96, 64, 8, 2)):
        x, w = rnd(N, K + 5)[:, 3:3 + K], rnd(M, K + 3)[:, 1:1 + K]
        ad = fsb.Adapters(rnd(n, r, K), rnd(n, M, r), None)
        ids = torch.randint(-1, n, (N,), generator=gen, device="cuda", dtype=torch.int32)
        out = torch.zeros(N, M + 4, dtype=DT[dtype], device="cuda")
        y = fsb.project(x, w, None, ad, ids, out=out[:, 1:1 + M])
        assert torch.equal(y, fsb.project(x.contiguous(), w.contiguous(), None, ad, ids))
        assert (out[:, 0] == 0).all() and (out[:, 1 + M:] == 0).all()
        g = rnd(N, M + 7)[:, 5:5 + M]
        got = fsb.project_grad(g, x, w, ad, ids)
        want = fsb.project_grad(g.contiguous(), x.contiguous(), w.contiguous(), ad, ids)
        for a, b in zip(got, want):
            assert torch.equal(a, b)
        # a gradient broadcast over the rows, and the same row everywhere
        got = fsb.project_grad(g[:1].expand(N, M), x[:1].expand(N, K), w, ad, ids)
        want = fsb.project_grad(g[:1].expand(N, M).contiguous(), x[:1].expand(N, K).contiguous(), w.contiguous(), ad, ids)
        for a, b in zip(got, want):
            assert torch.equal(a, b)


def test_project_keeps_infinities_to_their_rows(fsb):
    """A NaN or infinity in a row, or in an adapter that other rows use, stays out of the rest."""
    for dtype in ("f32", "bf16"):
        d = _cuda(_problem(9, dtype, 70, 48, 40, 4, 3, "mixed"))
        clean = fsb.project(d["x"], d["w"], None, _adapters(fsb, d), d["ids"])
        d["x"][5, 3] = float("nan")
        d["x"][6, 4] = float("inf")
        bad = d["a"].clone()
        bad[1, 2, 7] = float("nan")
        d["a"] = bad
        y = fsb.project(d["x"], d["w"], None, _adapters(fsb, d), d["ids"])
        hit = (d["ids"] == 1)
        hit[5] = hit[6] = True
        assert torch.equal(y[~hit], clean[~hit])
        assert not torch.isfinite(y[hit]).all(1).any()


# Every tile size, and each way to share the work: tiles of 128 and 256 rows and columns with whole and cut steps,
# sixteen waves to a few rows, waves that share rows of few columns, rows enough for a wave to two sixteens of them.
LARGE = [
    (2100, 100, 2000, 16, 5, "mixed"), (2051, 2004, 70, 3, 3, "bad"), (3500, 128, 3600, 16, 5, "bad"),
    (3333, 3608, 128, 9, 4, "runs"), (3330, 3600, 64, 40, 2, "mixed"), (40, 1200, 40, 8, 3, "mixed"),
    (50, 40, 60, 128, 3, "mixed"), (70, 33, 50, 40, 2, "mixed"), (90, 100, 70, 20, 3, "bad"), (300, 3, 2, 1, 2, "mixed"),
    (70001, 40, 3, 5, 3, "bad"), (66000, 24, 30, 34, 4, "mixed"),
    # more adapters than rows, more than 1024 of them; a few adapters over several thousand rows
    (40, 70, 90, 3, 1500, "mixed"), (2500, 48, 80, 2, 1100, "bad"), (37, 1100, 90, 20, 1025, "bad"),
    (3000, 1030, 100, 4, 3, "mixed"), (1025, 520, 100, 4, 1024, "mixed")]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,K,M,r,n,ids", LARGE)
def test_project_large(fsb, dtype, N, K, M, r, n, ids):
    test_project(fsb, dtype, N, K, M, r, n, ids)
    test_project_grad(fsb, dtype, N, K, M, r, n, ids)


def test_no_rows_leave_zero_gradients(fsb):
    for dt in (torch.float32, torch.bfloat16):
        for K, M, r in ((20, 2, 4), (20, 30, 40)):
            e = lambda *s: torch.ones(s, dtype=dt, device="cuda")
            ids = torch.zeros(0, dtype=torch.int32, device="cuda")
            gx, ga, gb = fsb.project_grad(e(0, M), e(0, K), e(M, K), fsb.Adapters(e(3, r, K), e(3, M, r)), ids)
            assert gx.shape == (0, K) and (ga == 0).all() and (gb == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_project_far_rows(fsb, dtype):
    """Rows, gradients and outputs whose elements lie beyond 2^31 from the first."""
    gen = torch.Generator(device="cuda").manual_seed(6)
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda").to(DT[dtype])
    stride = (1 << 29) + 8
    for K, M, r in ((72, 9, 3), (96, 136, 16)):
        x, w, g, ad = rnd(6, K), rnd(M, K), rnd(6, M), fsb.Adapters(rnd(2, r, K), rnd(2, M, r))
        ids = torch.tensor([0, 1, -1, 1, 0, 1], dtype=torch.int32, device="cuda")
        store = torch.empty(5 * stride + 512, dtype=DT[dtype], device="cuda")
        far = lambda t, at: store[at:].as_strided(t.shape, (stride, 1)).copy_(t)
        fx, fg, out = far(x, 0), far(g, 128), store[300:].as_strided((6, M), (stride, 1))
        assert torch.equal(fsb.project(fx, w, None, ad, ids, out=out), fsb.project(x, w, None, ad, ids))
        for a, b in zip(fsb.project_grad(fg, fx, w, ad, ids), fsb.project_grad(g, x, w, ad, ids)):
            assert torch.equal(a, b)


# -- streams, graphs, the operators together --------------------------------------------
def test_on_another_stream_and_captured(fsb):
    """The four calls on a side stream, then captured once and replayed on new inputs, between the program's own work."""
    d = _cuda(_problem(21, "f32", 600, 200, 33, 4, 3, "mixed"))
    ad = _adapters(fsb, d)
    labels = torch.randint(-1, 33, (600,), device="cuda", dtype=torch.int32)
    gl = torch.full((600,), 1 / 600, device="cuda")

    def step(stream=None):
        y, h = fsb.project(d["x"], d["w"], d["bias"], ad, d["ids"], return_hidden=True, stream=stream)
        r = fsb.logprobs(y, labels, 3, stream=stream)
        gy = fsb.logprobs_grad(y, r.norm, labels, gl, stream=stream)
        return (y, *r, gy, *fsb.project_grad(gy, d["x"], d["w"], ad, d["ids"], hidden=h, stream=stream))

    want = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = step(side)
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert torch.equal(g, w)
    graphs = []
    for _ in range(2):           # two graphs of the same calls: neither may use the other's scratch memory
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            held = step()
        graphs.append((graph, held))
    for k in range(4):
        d["x"].copy_(torch.randn_like(d["x"]).tanh())
        labels.copy_(torch.randint(-1, 33, (600,), device="cuda", dtype=torch.int32))
        d["ids"].copy_(torch.randint(-1, 3, (600,), device="cuda", dtype=torch.int32))
        want = step()
        graph, held = graphs[k % 2]
        graph.replay()
        torch.cuda.synchronize()
        for g, w in zip(held, want):
            assert torch.equal(g, w)


def test_two_streams_at_once(fsb):
    """The same calls side by side on two streams give what each gives alone."""
    d = [_cuda(_problem(31 + k, "bf16", 900, 512, 300, 8, 5, "mixed")) for k in range(2)]
    ads = [_adapters(fsb, c) for c in d]
    x = [torch.randn((40, 60000), device="cuda", generator=torch.Generator(device="cuda").manual_seed(k)) for k in range(2)]

    def calls(k):
        y, h = fsb.project(d[k]["x"], d[k]["w"], d[k]["bias"], ads[k], d[k]["ids"], return_hidden=True)
        g = fsb.project_grad(d[k]["g"], d[k]["x"], d[k]["w"], ads[k], d[k]["ids"], hidden=h)
        r = fsb.logprobs(x[k], n_top=9)
        return (y, h, *g, r.entropy, r.norm, r.top_id, r.top_logp)

    want = [calls(k) for k in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(3):
        for k in range(2):
            with torch.cuda.stream(streams[k]):
                got[k].append(calls(k))
    torch.cuda.synchronize()
    for k in range(2):
        for result in got[k]:
            for a, b in zip(result, want[k]):
                assert torch.equal(a, b)


def test_adapter_of_a_net_s_last_layer(fsb):
    """The operators as they are used together: features of every window from a scan, the last layer with an adapter
    an image, the labels' log probabilities, and the adapters' gradients, against float64 differences of the mean."""
    w = wl.WORKLOADS[1]
    params, _ = wl.workload_inputs(1)
    layers = w.layers[:-1]
    img = wl.make_image(7, 3, 20, 23, 1)
    feats = fsb.Net(layers, params[:-1], 1).scan(torch.from_numpy(img).cuda())     # tanh features [3, h, w, 16]
    K, M, r = 16, 2, 2
    rng = np.random.default_rng(8)
    wt, bias = params[-1][0].reshape(M, K), params[-1][1]
    a, b = rng.normal(0, 0.5, (3, r, K)).astype(np.float32), rng.normal(0, 0.5, (3, M, r)).astype(np.float32)
    scale = np.array([1.0, 0.5, 2.0], np.float32)
    shape = tuple(feats.shape[:-1])
    ids = np.broadcast_to(np.arange(3, dtype=np.int32)[:, None, None], shape).copy()
    labels = rng.integers(-1, M, shape).astype(np.int32)
    cuda = lambda v: torch.from_numpy(np.ascontiguousarray(v)).cuda()
    ad = fsb.Adapters(cuda(a), cuda(b), cuda(scale))
    y, h = fsb.project(feats, cuda(wt), cuda(bias), ad, cuda(ids), return_hidden=True)
    lp = fsb.logprobs(y, cuda(labels), 1)
    n = (labels >= 0).sum()
    gy = fsb.logprobs_grad(y, lp.norm, cuda(labels), torch.full(shape, 1.0 / n, device="cuda"))
    _, ga, gb = fsb.project_grad(gy, feats, cuda(wt), ad, cuda(ids), hidden=h, need_x=False)
    x64 = _np(feats).reshape(-1, K)

    def mean(a64, b64):
        y64, _ = ro.project(x64, wt.astype(np.float64), bias.astype(np.float64), a64, b64, scale.astype(np.float64), ids.ravel())
        return ro.logprobs(y64, labels.ravel(), 0, 1.0)[0].sum() / n

    a64, b64 = a.astype(np.float64), b.astype(np.float64)
    assert abs(float(lp.logp.sum()) / n - mean(a64, b64)) < 1e-5
    for got, t in ((ga, a64), (gb, b64)):
        for i in [(0, 0, 0), (1, 1, 1), (2, 0, t.shape[2] - 1), (2, 1, 0)]:
            keep = t[i]
            t[i] = keep + 1e-4
            up = mean(a64, b64)
            t[i] = keep - 1e-4
            diff = (up - mean(a64, b64)) / 2e-4
            t[i] = keep
            # float32 sums over about 400 rows, differences of second order in 1e-4
            assert abs(float(got[i]) - diff) < 2e-6 + 1e-4 * abs(diff)
