"""The row operators without a GPU: their oracle against differences, and every
refusal of the C-ABI and of the binding, made before anything is enqueued."""
import ctypes

import numpy as np
import pytest
import torch

import rows_oracle as ro
from paper_1302_1700_amd import fragscan as fsb

BAD = 0x10000  # an address that is never read: each call below is refused before


def _difference(f, x, eps=1e-5):
    g = np.zeros_like(x)
    for i in np.ndindex(*x.shape):
        keep = x[i]
        x[i] = keep + eps
        up = f()
        x[i] = keep - eps
        down = f()
        x[i] = keep
        g[i] = (up - down) / (2 * eps)
    return g


@pytest.mark.parametrize("T", [1.0, 0.7, 2.5])
def test_oracle_gradient_of_logprobs_is_the_difference(T):
    rng = np.random.default_rng(3)
    x = rng.normal(0, 2, (5, 7))
    x[1, 2] = -np.inf
    y = np.array([0, 3, -1, 6, 2])
    gl, ge = rng.normal(0, 1, 5), rng.normal(0, 1, 5)

    def f():
        logp, ent = ro.logprobs(x, y, 0, T)[:2]
        return float((gl * logp + ge * ent).sum())

    want = ro.logprobs_grad(x, y, T, gl, ge)
    # central differences: eps^2 / 6 of third derivatives of order one, and 1e-15 / eps of rounding;
    # a score of -inf stays one, so its difference is 0
    assert np.abs(_difference(f, x) - want).max() < 1e-8


def test_oracle_gradient_of_project_is_the_difference():
    rng = np.random.default_rng(4)
    N, K, M, r, n = 6, 5, 4, 2, 3
    x, w, c = rng.normal(0, 1, (N, K)), rng.normal(0, 1, (M, K)), rng.normal(0, 1, (N, M))
    a, b, s = rng.normal(0, 1, (n, r, K)), rng.normal(0, 1, (n, M, r)), rng.uniform(0.5, 2, n)
    ids = [0, 2, -1, 2, 0, 0]
    f = lambda: float((c * ro.project(x, w, None, a, b, s, ids)[0]).sum())
    gx, ga, gb = ro.project_grad(c, x, w, a, b, s, ids)
    for got, t in ((gx, x), (ga, a), (gb, b)):
        assert np.abs(got - _difference(f, t)).max() < 1e-8
    assert (ga[1] == 0).all() and (gb[1] == 0).all()


def _logprobs(lib, scores=BAD, rows=4, classes=10, stride=10, dtype=0, T=1.0, labels=BAD, n_top=2, logp=BAD, entropy=BAD,
              norm=BAD, top_id=BAD, top_logp=BAD, ws=BAD, have=1 << 30):
    return lib.fs_logprobs(scores, rows, classes, stride, dtype, T, labels, n_top, logp, entropy, norm, top_id, top_logp,
                           ws, have, None)


def _grad(lib, scores=BAD, rows=4, classes=10, stride=10, dtype=0, T=1.0, labels=BAD, norm=BAD, entropy=BAD, g_logp=BAD,
          g_entropy=BAD, g=BAD * 2, g_stride=10):
    return lib.fs_logprobs_grad(scores, rows, classes, stride, dtype, T, labels, norm, entropy, g_logp, g_entropy, g,
                                g_stride, None)


INVALID, UNSUPPORTED, WORKSPACE = fsb.FS_ERR_INVALID_ARG, fsb.FS_ERR_UNSUPPORTED, fsb.FS_ERR_WORKSPACE


@pytest.mark.parametrize("kw,status", [
    (dict(scores=None), INVALID), (dict(scores=BAD + 2), INVALID), (dict(scores=BAD + 1, dtype=1), INVALID),
    (dict(rows=-1), INVALID), (dict(rows=1 << 31), UNSUPPORTED), (dict(classes=0), INVALID),
    (dict(classes=(1 << 24) + 1), INVALID), (dict(stride=-1), INVALID), (dict(stride=1 << 60), UNSUPPORTED),
    (dict(dtype=2), INVALID), (dict(T=0.0), INVALID), (dict(T=-1.0), INVALID), (dict(T=float("nan")), INVALID),
    (dict(T=float("inf")), INVALID), (dict(T=1e-39), INVALID), (dict(labels=None), INVALID), (dict(n_top=-1), INVALID),
    (dict(n_top=65), INVALID), (dict(n_top=0), INVALID), (dict(labels=BAD + 2), INVALID), (dict(logp=BAD + 2), INVALID),
    (dict(norm=BAD + 1), INVALID), (dict(top_id=BAD + 3), INVALID),
    (dict(logp=None, entropy=None, norm=None, top_id=None, top_logp=None), INVALID)])
def test_logprobs_refuses(kw, status):
    lib = fsb.load()
    assert _logprobs(lib, **kw) == status
    assert lib.fs_last_error()


@pytest.mark.parametrize("kw,status", [
    (dict(scores=None), INVALID), (dict(g=None), INVALID), (dict(norm=None), INVALID), (dict(labels=None), INVALID),
    (dict(entropy=None), INVALID), (dict(g_logp=None, g_entropy=None), INVALID), (dict(g_stride=9), INVALID),
    (dict(g_stride=-3), INVALID), (dict(g=BAD, g_stride=11), INVALID), (dict(T=0.0), INVALID), (dict(rows=-2), INVALID),
    (dict(g=BAD + 2), INVALID), (dict(g_entropy=BAD + 2), INVALID), (dict(dtype=-1), INVALID), (dict(classes=0), INVALID)])
def test_logprobs_grad_refuses(kw, status):
    lib = fsb.load()
    assert _grad(lib, **kw) == status
    assert lib.fs_last_error()


def test_no_rows_are_no_work():
    lib = fsb.load()
    assert _logprobs(lib, rows=0, scores=None, ws=None, have=0) == fsb.FS_OK
    assert _grad(lib, rows=0, scores=None, g=None) == fsb.FS_OK
    assert _project(lib, rows=0, d_x=None, d_ids=None, y=None) == fsb.FS_OK


def _proj(**kw):
    d = dict(rows=4, k=6, m=70, dtype=0, n_adapters=2, rank=3, d_x=BAD, x_stride=6, d_w=BAD, w_stride=6, d_bias=BAD,
             d_a=BAD, d_b=BAD, d_scale=BAD, d_ids=BAD)
    d.update(kw)
    return fsb.fs_projection(**d)


def _project(lib, y=BAD, y_stride=70, hidden=None, ws=BAD, have=1 << 40, **kw):
    return lib.fs_project(ctypes.byref(_proj(**kw)), y, y_stride, hidden, ws, have, None)


def _project_grad(lib, g=BAD, g_stride=70, hidden=None, gx=BAD, gx_stride=6, ga=BAD, gb=BAD, ws=BAD, have=1 << 40, **kw):
    return lib.fs_project_grad(ctypes.byref(_proj(**kw)), g, g_stride, hidden, gx, gx_stride, ga, gb, ws, have, None)


PROJ = [(dict(rows=-1), INVALID), (dict(rows=1 << 31), UNSUPPORTED), (dict(k=0), INVALID), (dict(m=0), INVALID),
        (dict(k=(1 << 20) + 1), INVALID), (dict(m=(1 << 20) + 1), INVALID), (dict(dtype=7), INVALID),
        (dict(n_adapters=-1), INVALID), (dict(n_adapters=(1 << 20) + 1), INVALID), (dict(rank=0), INVALID),
        (dict(rank=129), INVALID), (dict(n_adapters=0), INVALID), (dict(n_adapters=0, rank=0), INVALID),
        (dict(d_x=None), INVALID), (dict(d_x=BAD + 2), INVALID), (dict(x_stride=-6), INVALID),
        (dict(x_stride=1 << 60), UNSUPPORTED), (dict(d_w=None), INVALID), (dict(w_stride=-1), INVALID),
        (dict(d_w=BAD + 1, dtype=1), INVALID), (dict(d_bias=BAD + 2), INVALID), (dict(d_a=None), INVALID),
        (dict(d_b=None), INVALID), (dict(d_b=BAD + 2), INVALID), (dict(d_scale=BAD + 1), INVALID),
        (dict(d_ids=None), INVALID), (dict(d_ids=BAD + 2), INVALID), (dict(hidden=BAD + 2), INVALID)]


@pytest.mark.parametrize("kw,status", PROJ + [
    (dict(y=None), INVALID), (dict(y_stride=69), INVALID), (dict(y=BAD + 2), INVALID),
    (dict(have=0), WORKSPACE), (dict(ws=None), INVALID), (dict(ws=BAD + 16), INVALID),
    (dict(n_adapters=0, rank=0, d_a=None, d_b=None, d_scale=None, d_ids=None, hidden=BAD), INVALID)])
def test_project_refuses(kw, status):
    lib = fsb.load()
    assert _project(lib, **kw) == status
    assert lib.fs_last_error()


@pytest.mark.parametrize("kw,status", PROJ + [
    (dict(g=None), INVALID), (dict(g_stride=-1), INVALID), (dict(gx_stride=5), INVALID), (dict(ga=None), INVALID),
    (dict(gb=None), INVALID), (dict(gx=None, ga=None, gb=None), INVALID), (dict(ga=BAD + 2), INVALID),
    (dict(have=0), WORKSPACE), (dict(ws=None), INVALID), (dict(ws=BAD + 128), INVALID),
    (dict(n_adapters=0, rank=0, d_a=None, d_b=None, d_scale=None, d_ids=None), INVALID)])
def test_project_grad_refuses(kw, status):
    lib = fsb.load()
    assert _project_grad(lib, **kw) == status
    assert lib.fs_last_error()


def test_workspace_calls_refuse():
    lib, need = fsb.load(), ctypes.c_size_t()
    assert lib.fs_logprobs_workspace(1, 5, 0, 1, None) == INVALID
    assert lib.fs_logprobs_workspace(1, 0, 0, 1, ctypes.byref(need)) == INVALID
    assert lib.fs_logprobs_workspace(1, 5, 3, 1, ctypes.byref(need)) == INVALID
    for f in (lib.fs_project_workspace, lib.fs_project_grad_workspace):
        assert f(None, ctypes.byref(need)) == INVALID
        assert f(ctypes.byref(_proj()), None) == INVALID
        assert f(ctypes.byref(_proj(rank=200)), ctypes.byref(need)) == INVALID
        assert f(ctypes.byref(_proj(d_x=None, d_w=None, d_ids=None)), ctypes.byref(need)) == fsb.FS_OK


def test_row_views():
    t = torch.zeros(4, 6, 10)
    assert fsb._rows_of(t, "t") == (24, 10, 10)
    assert fsb._rows_of(t[:, :, :7], "t") == (24, 7, 10)
    assert fsb._rows_of(t[:, 2], "t") == (4, 10, 60)
    assert fsb._rows_of(t[:, :, :1], "t") == (24, 1, 10)
    assert fsb._rows_of(t[1, 2], "t") == (1, 10, 10)
    assert fsb._rows_of(torch.zeros(10).expand(3, 5, 10), "t") == (15, 10, 0)
    assert fsb._rows_of(t[:0], "t") == (0, 10, 10)
    for bad in (t[:, :4], t.transpose(1, 2), t[:, :, ::2], torch.zeros(()), torch.zeros(3, 0), t.permute(1, 0, 2)):
        with pytest.raises(ValueError):
            fsb._rows_of(bad, "t")


def test_binding_refuses():
    x, y = torch.zeros(3, 4), torch.zeros(3, dtype=torch.int32)
    w, ad = torch.zeros(5, 4), fsb.Adapters(torch.zeros(2, 3, 4), torch.zeros(2, 5, 3))
    for call in (
            lambda: fsb.logprobs(x, y),                                             # not on a GPU
            lambda: fsb.logprobs(x.double(), y),
            lambda: fsb.logprobs(x, y.long()),
            lambda: fsb.logprobs(x, y[:2]),
            lambda: fsb.logprobs(x.t(), y),
            lambda: fsb.logprobs_grad(x, torch.zeros(3), y, torch.zeros(3)),
            lambda: fsb.logprobs_grad(x, torch.zeros(3, 2), y, torch.zeros(3).double()),
            lambda: fsb.logprobs_grad(x, torch.zeros(3, 2), y, torch.zeros(3)),     # not on a GPU
            lambda: fsb.project(x, w),                                              # not on a GPU
            lambda: fsb.project(x, w.bfloat16()),
            lambda: fsb.project(x, w.t()),
            lambda: fsb.project(x, w, torch.zeros(4)),
            lambda: fsb.project(x, w, None, ad),
            lambda: fsb.project(x, w, None, None, y),
            lambda: fsb.project(x, w, None, ad, y.long()),
            lambda: fsb.project(x, w, None, ad._replace(b=torch.zeros(2, 4, 3)), y),
            lambda: fsb.project(x, w, None, ad._replace(a=torch.zeros(3, 3, 4)), y),
            lambda: fsb.project(x, w, None, ad._replace(scale=torch.zeros(3)), y),
            lambda: fsb.project(x, w, None, ad._replace(a=torch.zeros(2, 0, 4), b=torch.zeros(2, 5, 0)), y),
            lambda: fsb.project(x, w, return_hidden=True),
            lambda: fsb.project_grad(torch.zeros(3, 4), x, w, ad, y),
            lambda: fsb.project_grad(torch.zeros(3, 5), x, w, None, None, need_x=False),
            lambda: fsb.project_grad(torch.zeros(3, 5), x, w, None, None, hidden=torch.zeros(3, 3)),
            lambda: fsb.project_grad(torch.zeros(3, 5), x, w, ad, y, hidden=torch.zeros(3, 2))):
        with pytest.raises(ValueError):
            call()
