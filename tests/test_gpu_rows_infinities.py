"""Infinite and very large values in the projection and its gradient: what the definition says of them, from every
kernel that the sizes may select."""
import numpy as np
import pytest

import rows_oracle as ro
from test_gpu_rows import DT, _absolute, _adapters, _check, _cuda, _f64, _problem, fsb  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

# rows, inputs, outputs, rank, adapters of the forward pass; for the rows' gradient inputs and outputs change places
FEW = [(70, 48, 40, 4, 3), (70, 48, 40, 8, 3)]                 # one pass over the rows
TILES = [(70, 48, 100, 3, 3), (70, 48, 100, 4, 3), (70, 48, 100, 8, 3), (70, 48, 100, 12, 3), (70, 48, 100, 24, 3),
         (70, 48, 100, 40, 2), (2051, 40, 2004, 4, 3), (2051, 40, 2004, 8, 3), (3500, 128, 3600, 16, 3)]
SPLIT = [(40, 1200, 100, 8, 3)]                                 # the summed axis in stretches
KEYS, GRAD_KEYS = ("x", "w", "bias", "a", "b", "scale", "ids"), ("g", "x", "w", "a", "b", "scale", "ids")


def _forward(fsb, d, dtype):
    """project against the definition: infinities of the same sign, NaN where it has them, the rest within bounds."""
    c, o = _cuda(d), _f64(d)
    K, r = d["x"].shape[1], d["a"].shape[1]
    y, h = fsb.project(c["x"], c["w"], c["bias"], _adapters(fsb, c), c["ids"], return_hidden=True)
    with np.errstate(invalid="ignore"):
        wy, wh = ro.project(*(o[k] for k in KEYS))
        ay, ah = ro.project(*(_absolute(o)[k] for k in KEYS))
        _check(y, wy, np.nan_to_num(ay), K + r, dtype, "y")
        _check(h, wh, np.nan_to_num(ah), K, "f32", "hidden")
    return wy


def _backward(fsb, d, dtype, need_adapters=True):
    c, o = _cuda(d), _f64(d)
    (N, K), M, r = d["x"].shape, d["g"].shape[1], d["a"].shape[1]
    gx, ga, gb = fsb.project_grad(c["g"], c["x"], c["w"], _adapters(fsb, c), c["ids"], need_adapters=need_adapters)
    with np.errstate(invalid="ignore"):
        wx, wa, wb = ro.project_grad(*(o[k] for k in GRAD_KEYS))
        ax, aa, ab = (np.nan_to_num(v) for v in ro.project_grad(*(_absolute(o)[k] for k in GRAD_KEYS)))
        _check(gx, wx, ax, M + 2 * r, dtype, "gx")
        if need_adapters:
            _check(ga, wa, aa, N + M, dtype, "ga")
            _check(gb, wb, ab, N + K, dtype, "gb")
    return wx, wa, wb


def _infinite_factor(fsb, dtype, N, K, M, r, n):
    print("infinite factor", dtype, N, K, M, r, n, flush=True)
    d = _problem(N + K + r, dtype, N, K, M, r, n, "mixed")
    d["b"][1, 5, r - 1], d["b"][1, 7, 0] = float("inf"), -float("inf")
    assert np.isinf(_forward(fsb, d, dtype)).any()
    d = _problem(N + K + r, dtype, N, M, K, r, n, "mixed")
    d["a"][1, r - 1, 5], d["a"][1, 0, 7] = float("inf"), -float("inf")
    assert np.isinf(_backward(fsb, d, dtype)[0]).any()


@pytest.mark.parametrize("N,K,M,r,n", FEW + TILES + SPLIT)
def test_infinite_factor_f32(fsb, N, K, M, r, n):
    """An infinite element of a factor gives the infinities of the definition, at ranks that leave operands unfilled."""
    _infinite_factor(fsb, "f32", N, K, M, r, n)


@pytest.mark.parametrize("N,K,M,r,n", FEW + TILES + SPLIT)
def test_infinite_factor_bf16(fsb, N, K, M, r, n):
    """The same where the hidden values are taken as three bf16 parts of either sign."""
    _infinite_factor(fsb, "bf16", N, K, M, r, n)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,K,M,r,n", FEW + TILES + SPLIT)
def test_infinite_hidden_values(fsb, dtype, N, K, M, r, n):
    """A_i x, and in the gradient B_i^T g, of +-infinity."""
    print("infinite hidden", dtype, N, K, M, r, n, flush=True)
    d = _problem(N + K + r, dtype, N, K, M, r, n, "mixed")
    d["a"][1, r - 1, 3] = float("inf")
    assert np.isinf(_forward(fsb, d, dtype)).any()
    d = _problem(N + K + r, dtype, N, M, K, r, n, "mixed")
    d["b"][1, 5, r - 1] = float("inf")
    assert np.isinf(_backward(fsb, d, dtype)[0]).any()


@pytest.mark.parametrize("N,K,M,r,n", FEW + TILES + SPLIT)
def test_hidden_values_past_the_largest_bf16(fsb, N, K, M, r, n):
    """Finite float32 values that would round to an infinite bf16: 3.4015e38, times 2^-20."""
    print("large hidden", N, K, M, r, n, flush=True)
    d = _problem(N + K + r, "bf16", N, K, M, r, n, "mixed", scale=False)
    d["x"][:, :2] = 1
    d["a"][1, 0] = 0
    d["a"][1, 0, 0], d["a"][1, 0, 1] = torch.finfo(torch.bfloat16).max, 1.2e36
    d["b"][1, :, 0] *= 2.0 ** -20
    assert np.abs(_forward(fsb, d, "bf16")).max() > 1e31
    d = _problem(N + K + r, "bf16", N, M, K, r, n, "mixed", scale=False)
    d["g"][:, :2] = 1
    d["b"][1, :, 0] = 0
    d["b"][1, 0, 0], d["b"][1, 1, 0] = torch.finfo(torch.bfloat16).max, 1.2e36
    d["a"][1, 0] *= 2.0 ** -20
    assert np.abs(_backward(fsb, d, "bf16", need_adapters=False)[0]).max() > 1e31


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,K,M,r", [(70, 48, 2, 4), (70, 48, 10, 9), (70, 48, 100, 9), (1030, 48, 2, 4), (1030, 33, 12, 16),
                                     (1030, 48, 30, 20)])
def test_factor_gradients_of_one_row_with_an_infinite_factor(fsb, dtype, N, K, M, r):
    """An adapter of one row: its gradient is that row's outer product, infinite where B_i^T g is."""
    print("one row an adapter", dtype, N, K, M, r, flush=True)
    d = _problem(N + K + r, dtype, N, K, M, r, N, "runs")
    assert (d["ids"] == torch.arange(N)).all()
    d["b"][3, 0, r - 2], d["b"][N - 1, 1, 0] = float("inf"), -float("inf")
    _, wa, _ = _backward(fsb, d, dtype)
    assert np.isinf(wa[3, r - 2]).all() and np.isinf(wa[N - 1, 0]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N", [0, 70, 1030])
@pytest.mark.parametrize("K,M,r", [(48, 2, 4), (48, 30, 20)])
def test_adapters_without_rows_have_zero_gradients_at_any_scale(fsb, dtype, N, K, M, r):
    d = _problem(N + K + r, dtype, N, K, M, r, 4, "runs")
    d["ids"][d["ids"] == 1] = 0
    d["ids"][d["ids"] == 2] = -1
    d["scale"] = torch.tensor([1.0, float("inf"), float("nan"), 0.5])
    print("no rows, scales not finite", dtype, N, K, M, r, flush=True)
    _, wa, wb = _backward(fsb, d, dtype)
    assert (wa[1:3] == 0).all() and (wb[1:3] == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,K,M,r,n", FEW + TILES + SPLIT + [(70, 48, 2, 4, 3), (600, 48, 12, 9, 3)])
def test_scale_multiplies_the_sum(fsb, dtype, N, K, M, r, n):
    """s (B h) of 2^80 where s times a hidden value, or a factor's element, would pass float32's range."""
    print("large scale", dtype, N, K, M, r, n, flush=True)
    d = _problem(N + K + r, dtype, N, K, M, r, n, "mixed")
    d["scale"] *= 2.0 ** 40
    d["a"] *= 2.0 ** 100
    d["b"] *= 2.0 ** -60
    assert np.abs(_forward(fsb, d, dtype)).max() < 2.0 ** 100
    d = _problem(N + K + r, dtype, N, K, M, r, n, "mixed")
    d["scale"] *= 2.0 ** 40
    d["b"] *= 2.0 ** 100
    d["g"] *= 2.0 ** -60
    assert np.abs(_backward(fsb, d, dtype)[1]).max() < 2.0 ** 110


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,K,M,r,n", FEW + TILES + SPLIT)
def test_infinities_stay_with_their_rows(fsb, dtype, N, K, M, r, n):
    """NaN and infinities in a row, a gradient row, or an adapter change nothing of the other rows and adapters."""
    print("isolation", dtype, N, K, M, r, n, flush=True)
    bits = lambda t: t.view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32)

    def spoil(c):
        c["x"][5, 3], c["x"][6, 4] = float("nan"), float("inf")
        c["g"][7, 1], c["g"][8, 2] = float("nan"), -float("inf")
        c["a"][1, r - 1, 7], c["b"][1, 3, 0] = float("nan"), float("inf")

    c = _cuda(_problem(N + r, dtype, N, K, M, r, n, "mixed"))
    clean = fsb.project(c["x"], c["w"], None, _adapters(fsb, c), c["ids"], return_hidden=True)
    spoil(c)
    got = fsb.project(c["x"], c["w"], None, _adapters(fsb, c), c["ids"], return_hidden=True)
    rest = c["ids"] != 1
    rest[5] = rest[6] = False
    for g, w in zip(got, clean):
        assert torch.equal(bits(g[rest]), bits(w[rest]))
    c = _cuda(_problem(N + r, dtype, N, M, K, r, n, "mixed"))
    clean = fsb.project_grad(c["g"], c["x"], c["w"], _adapters(fsb, c), c["ids"])
    spoil(c)
    got = fsb.project_grad(c["g"], c["x"], c["w"], _adapters(fsb, c), c["ids"])
    rest = c["ids"] != 1
    rest[7] = rest[8] = False
    assert torch.equal(bits(got[0][rest]), bits(clean[0][rest]))
    rest = torch.ones(n, dtype=torch.bool, device="cuda")
    rest[1] = False
    for row in (5, 6, 7, 8):
        if c["ids"][row] >= 0:
            rest[c["ids"][row].long()] = False
    for g, w in zip(got[1:], clean[1:]):
        assert torch.equal(bits(g[rest]), bits(w[rest]))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,K,M,r,n", FEW + TILES + SPLIT + [(70, 48, 2, 4, 3), (1030, 48, 12, 9, 3)])
def test_infinite_rows(fsb, dtype, N, K, M, r, n):
    """An infinite element of a row, or of its gradient, with an adapter and without one."""
    print("infinite rows", dtype, N, K, M, r, n, flush=True)
    d = _problem(N + r, dtype, N, K, M, r, n, "mixed")
    d["ids"][5], d["ids"][6] = -1, 1
    d["x"][5, 3], d["x"][6, 4] = float("inf"), -float("inf")
    assert np.isinf(_forward(fsb, d, dtype)[5]).all()
    d = _problem(N + r, dtype, N, M, K, r, n, "mixed")
    d["ids"][5], d["ids"][6], d["ids"][7] = -1, 1, 0
    d["g"][5, 1], d["g"][6, 0], d["x"][7, 1] = float("inf"), -float("inf"), float("inf")
    wx, _, wb = _backward(fsb, d, dtype)
    assert np.isinf(wx[5]).all() and np.isinf(wb[1, 0]).all()
