"""Ways through the row operators that only certain sizes take: joins of more than a thousand runs, more units than a
grid's second axis holds, outputs that end inside a quad of a split product, and a temperature whose reciprocal is not
a float32."""
import numpy as np
import pytest

import rows_oracle as ro
from test_gpu_rows import DT, _adapters, _bounds, _check, _cuda, _f64, _np, _problem, _scores, fsb  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


# -- many runs, many units, cut quads ---------------------------------------------------
def _by_adapter(o):
    """project and project_grad in float64 (definitions as in rows_oracle), all rows of an adapter at a time."""
    x, g, w, a, b, ids = (o[k] for k in ("x", "g", "w", "a", "b", "ids"))
    y, gx = x @ w.T, g @ w
    if o["bias"] is not None:
        y = y + o["bias"]
    h, ga, gb = np.zeros((len(x), a.shape[1])), np.zeros_like(a), np.zeros_like(b)
    order = np.argsort(ids, kind="stable")
    lo, hi = np.searchsorted(ids[order], [np.arange(len(a)), np.arange(1, len(a) + 1)])
    for i in np.flatnonzero(hi > lo):
        at = order[lo[i]:hi[i]]
        s = 1.0 if o["scale"] is None else o["scale"][i]
        h[at] = x[at] @ a[i].T
        y[at] += s * (h[at] @ b[i].T)
        u = s * (g[at] @ b[i])
        gx[at] += u @ a[i]
        ga[i], gb[i] = u.T @ x[at], s * (g[at].T @ h[at])
    for t in (y, h, gx):
        t[ids >= len(a)] = np.nan
    return y, h, gx, ga, gb


def test_by_adapter_is_the_oracle():
    for ids in ("mixed", "bad"):
        o = _f64(_problem(3, "f32", 50, 6, 5, 3, 4, ids))
        y, h, gx, ga, gb = _by_adapter(o)
        want = ro.project(*(o[k] for k in ("x", "w", "bias", "a", "b", "scale", "ids"))) + \
            ro.project_grad(*(o[k] for k in ("g", "x", "w", "a", "b", "scale", "ids")))
        for g, w in zip((y, h, gx, ga, gb), want):
            assert np.allclose(g, w, rtol=1e-12, atol=1e-12, equal_nan=True)


def _check_all(fsb, dtype, N, K, M, r, n, ids):
    d = _problem(N + K + M, dtype, N, K, M, r, n, ids)
    c, o = _cuda(d), _f64(d)
    ad = _adapters(fsb, c)
    y, h = fsb.project(c["x"], c["w"], c["bias"], ad, c["ids"], return_hidden=True)
    kept = fsb.project_grad(c["g"], c["x"], c["w"], ad, c["ids"], hidden=h)
    gx, ga, gb = fsb.project_grad(c["g"], c["x"], c["w"], ad, c["ids"])
    torch.cuda.synchronize()
    for one, other in zip(kept[1:], (ga, gb)):
        assert torch.equal(one, other)
    want = _by_adapter(o)
    size = [np.nan_to_num(v) for v in _by_adapter({k: v if v is None or k == "ids" else np.abs(v) for k, v in o.items()})]
    for got, what, terms, kind, w, s in zip((y, h, gx, ga, gb), ("y", "hidden", "gx", "ga", "gb"),
                                            (K + r, K, M + 2 * r, N + M, N + K), (dtype, "f32", dtype, dtype, dtype), want, size):
        _check(got, w, s, terms, kind, what)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,K,M,r,n,ids", [
    (140001, 8, 2, 2, 3, "bad"),        # both factors' gradients in 1094 runs of rows
    (140001, 6, 2, 3, 2, "runs"),
    (70001, 8, 2, 1, 200, "mixed"),     # 109,400 runs of adapters
    (70001, 8, 70, 1, 1000, "bad"),     # 69,000 adapters' rows among 1024, either way round
    (20, 2048, 131, 8, 3, "mixed"),     # the summed axis split, outputs that end 3, 2 and 1 into a quad
    (20, 2048, 130, 3, 3, "bad"), (20, 2048, 129, 5, 2, "mixed"), (70, 1500, 67, 16, 4, "mixed"),
    (20, 131, 2048, 8, 3, "mixed"),     # the same of the rows' gradient, and gradients of 3, 2 and 1 values
    (20, 130, 2048, 3, 3, "bad"), (20, 129, 2048, 5, 2, "mixed"), (20, 3, 2048, 8, 3, "mixed"), (20, 2, 2048, 3, 2, "bad"),
    (33, 1, 1600, 7, 2, "mixed")])
def test_projection_paths(fsb, dtype, N, K, M, r, n, ids):
    print("paths", dtype, N, K, M, r, n, ids, flush=True)
    _check_all(fsb, dtype, N, K, M, r, n, ids)


# -- the largest sizes the calls take -----------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,K,M,r,n,ids", [
    (3, 1 << 20, 2, 4, 2, "one"), (3, 1 << 20, 66, 2, 2, "mixed"), (3, 8, 1 << 20, 2, 2, "mixed"), (40, 8, 6, 128, 3, "mixed"),
    (40, 70, 90, 128, 3, "bad"), (5, 2, 2, 1, 1 << 20, "mixed"), (5, 4, 66, 1, 1 << 20, "bad")])
def test_most_features_ranks_and_adapters(fsb, dtype, N, K, M, r, n, ids):
    print("largest", dtype, N, K, M, r, n, ids, flush=True)
    _check_all(fsb, dtype, N, K, M, r, n, ids)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_most_classes(fsb, dtype):
    """2^24 classes: list, statistics and gradient against torch's float64 on the GPU. The sum's additions are in
    partial sums of 2^24 / 16384 terms a lane and their joins; the bound counts 2^24 / 32."""
    V = 1 << 24
    x = torch.randn((2, V), generator=torch.Generator(device="cuda").manual_seed(4), device="cuda").to(DT[dtype])
    x[1, V - 1], x[1, 5] = 9, 9
    y = torch.tensor([V - 1, 7], dtype=torch.int32, device="cuda")
    print("most classes", dtype, flush=True)
    r = fsb.logprobs(x, y, 64)
    g = fsb.logprobs_grad(x, r.norm, y, torch.ones(2, device="cuda"))
    for i in range(2):
        d = x[i].double()
        m = float(d.max())
        want = d.sort(stable=True, descending=True)
        assert torch.equal(r.top_id[i].long(), want.indices[:64])
        log_s = float((d - m).exp().sum().log())
        bound = ro.U32 * (V / 32 + 64 + 6 * 20)
        assert float(r.norm[i, 0]) == m and abs(float(r.norm[i, 1]) - log_s) <= bound
        logp = float(d[y[i].long()]) - m - log_s
        assert abs(float(r.logp[i]) - logp) <= bound + ro.U32 * 8 * 30
        p = (d - m - log_s).exp()
        grad = -p
        grad[y[i].long()] += 1
        off = (g[i].double() - grad).abs() - p * (bound + ro.U32 * 300) - ro.UOUT[dtype] * 1.01 * grad.abs() - 2.0 ** -133
        off[y[i].long()] -= 4 * ro.U32                      # 1 - p's own rounding
        assert float(off.max()) <= 0
        del d, want, p, grad, off


# -- rows that overlap ------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("step", [1, 3, 8])
@pytest.mark.parametrize("N,K,M,r,n", [(70, 48, 40, 4, 3), (70, 48, 100, 8, 3), (2051, 40, 2004, 4, 3), (3500, 128, 3600, 16, 3),
                                       (40, 1200, 100, 8, 3)])
def test_overlapping_rows(fsb, dtype, step, N, K, M, r, n):
    """Windows of one long vector as rows: strides below the rows' length, for inputs of every call."""
    print("overlapping", dtype, step, N, K, M, r, n, flush=True)
    c = _cuda(_problem(N + step, dtype, N, K, M, r, n, "mixed"))
    gen = torch.Generator(device="cuda").manual_seed(step)
    x, g, w = (torch.randn((rows - 1) * step + length, generator=gen, device="cuda").to(DT[dtype]).as_strided((rows, length), (step, 1))
               for rows, length in ((N, K), (N, M), (M, K)))
    ad = _adapters(fsb, c)
    dense = [t.contiguous() for t in (x, g, w)]
    got = (fsb.project(x, w, c["bias"], ad, c["ids"]),) + fsb.project_grad(g, x, w, ad, c["ids"])
    want = (fsb.project(dense[0], dense[2], c["bias"], ad, c["ids"]),) + fsb.project_grad(dense[1], dense[0], dense[2], ad, c["ids"])
    large = dtype == "bf16" and N > 3000 and step != 8   # the largest tiles need aligned rows: other sums, same bounds
    for a, b in zip(got, want):
        if large and a.shape[0] == N:
            assert float((a.float() - b.float()).abs().max()) <= 2 * ro.UOUT[dtype] * float(b.float().abs().max())
        else:
            assert torch.equal(a, b)
    y = torch.randint(0, M, (N,), generator=gen, device="cuda", dtype=torch.int32)
    a, b = fsb.logprobs(g, y, 3), fsb.logprobs(dense[1], y, 3)
    gl = torch.ones(N, device="cuda")
    for p, q in zip(a + (fsb.logprobs_grad(g, a.norm, y, gl),), b + (fsb.logprobs_grad(dense[1], b.norm, y, gl),)):
        assert torch.equal(p, q)


# -- the temperature as it is given -------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["plain", "peaks", "far"])
@pytest.mark.parametrize("T", [0.7, 1.5, 0.01, 37.0])
@pytest.mark.parametrize("rows,V", [(50, 3), (41, 64), (17, 511), (9, 1000), (5, 16385)])
def test_temperature_is_the_divisor(fsb, dtype, T, kind, rows, V):
    """Against (x - m) / T itself. With D = |x - m| / T, in half steps: a log probability's difference, reciprocal and
    product are 3 D off and its last subtraction |ln p|, no more than the bound's 4 (|ln p| + ln S); a term of the sum
    has a difference, a reciprocal, log2(e), their product and the argument's, 5 D, where the bound has 6."""
    rng = np.random.default_rng(rows + V)
    T = float(np.float32(T))
    x = _scores(rng, rows, V, dtype, kind)
    labels = rng.integers(0, V, rows).astype(np.int32)
    print("temperature", dtype, T, kind, rows, V, flush=True)
    r = fsb.logprobs(x.cuda(), torch.from_numpy(labels).cuda(), 1, T)
    x64 = _np(x)
    logp, _, norm, ids, tops, table = ro.logprobs(x64, labels, 1, T)
    each, log_s = _bounds(x64, T, table, norm, V)
    assert np.array_equal(r.top_id.cpu().numpy(), ids)
    ro.close(_np(r.norm)[:, 1:], norm[:, 1:], log_s, "log of the sum")
    ro.close(_np(r.logp), logp, each[np.arange(rows), labels], "logp")
    ro.close(_np(r.top_logp), tops, np.take_along_axis(each, ids, 1), "top logp")
