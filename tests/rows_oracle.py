"""The row operators in float64 on the CPU, straight from their definitions,
and the bounds that their float32 or bf16 results keep."""
import numpy as np

U32 = 2.0 ** -24                      # half a step of float32, relative
UOUT = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def logprobs(x, labels, n_top, T):
    """x float64 [N, V] -> logp, entropy, norm [N, 2], ids, top logp, table of log p."""
    N, V = x.shape
    logp, ent, norm = np.zeros(N), np.zeros(N), np.zeros((N, 2))
    ids, tops = np.full((N, n_top), -1, np.int32), np.full((N, n_top), -np.inf)
    table = np.full((N, V), -np.inf)
    for i in range(N):
        r = x[i]
        y = -1 if labels is None else int(labels[i])
        if np.isnan(r).any() or (r == np.inf).any():
            logp[i], ent[i], norm[i], tops[i], table[i] = (0.0 if y < 0 else np.nan), np.nan, np.nan, np.nan, np.nan
            continue
        live = np.flatnonzero(r > -np.inf)
        if not len(live):
            norm[i] = (-np.inf, 0.0)
            logp[i] = 0.0 if y < 0 else np.nan if y >= V else -np.inf
            continue
        m = r[live].max()
        d = (r[live] - m) / T
        s = np.exp(d).sum()
        lp = d - np.log(s)
        table[i, live] = lp
        norm[i] = (m, np.log(s))
        ent[i] = -(np.exp(lp) * lp).sum()
        logp[i] = 0.0 if y < 0 else np.nan if y >= V else table[i, y]
        order = live[np.lexsort((live, -r[live]))][:n_top]
        ids[i, :len(order)] = order
        tops[i, :len(order)] = table[i, order]
    return logp, ent, norm, ids, tops, table


def logprobs_grad(x, labels, T, g_logp, g_entropy):
    N, V = x.shape
    _, ent, norm, _, _, table = logprobs(x, None, 0, T)
    g = np.zeros((N, V))
    for i in range(N):
        y = -1 if labels is None or g_logp is None else int(labels[i])
        if y >= V or np.isnan(norm[i, 0]):
            g[i] = np.nan
            continue
        if norm[i, 0] == -np.inf:
            continue
        p = np.exp(table[i])
        if y >= 0:
            hot = np.zeros(V)
            hot[y] = 1
            g[i] += g_logp[i] * (hot - p)
        if g_entropy is not None:
            lp = np.where(p > 0, table[i], 0.0)
            g[i] -= g_entropy[i] * p * (lp + ent[i])
        g[i] /= T
    return g


def project(x, w, bias, a, b, scale, ids):
    y = x @ w.T
    if bias is not None:
        y = y + bias
    h = np.zeros((len(x), a.shape[1])) if a is not None else None
    if a is not None:
        for n, i in enumerate(ids):
            if i >= len(a):
                y[n], h[n] = np.nan, np.nan
            elif i >= 0:
                h[n] = a[i] @ x[n]
                y[n] += (1.0 if scale is None else scale[i]) * (b[i] @ h[n])
    return y, h


def project_grad(g, x, w, a, b, scale, ids):
    gx = g @ w
    if a is None:
        return gx, None, None
    ga, gb = np.zeros_like(a), np.zeros_like(b)
    for n, i in enumerate(ids):
        if i >= len(a):
            gx[n] = np.nan
        elif i >= 0:
            s = 1.0 if scale is None else scale[i]
            u = s * (b[i].T @ g[n])
            gx[n] += a[i].T @ u
            ga[i] += np.outer(u, x[n])
            gb[i] += s * np.outer(g[n], a[i] @ x[n])
    return gx, ga, gb


def close(got, want, bound, what):
    """Same NaNs and infinities, the rest within the bound (an array or number)."""
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    fine = np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want)), what
    assert np.array_equal(got[~fine & ~np.isnan(want)], want[~fine & ~np.isnan(want)]), what
    assert np.isfinite(got[fine]).all(), what
    off = np.abs(got - want) - np.broadcast_to(bound, want.shape)
    off = off[fine]
    assert not off.size or off.max() <= 0, (what, float(off.max()), int(off.argmax()))
