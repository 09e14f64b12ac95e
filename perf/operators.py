"""The row operators whose time counts: log probabilities of labels (with
entropy and the best classes) and their gradient, a shared projection with
low-rank adapters and its gradient; listed cases, a generator of more of the
same ranges, and for each the inputs, one pass, the work it cannot do without
and the same outputs in float64.

A case names an operator and its sizes:

  op        "logprobs", "logprobs_grad", "project" or "project_grad"
  dtype     "f32" or "bf16" (storage of scores, rows, weights and factors)
  rows      windows, or positions of a batch of sequences
  classes   scores of a row (logprobs*); top: how many best classes; temp: the
            temperature; masked: some classes are -inf, now and then a whole row
  k, m      inputs and outputs of the projection; rank, adapters: the factors
  ids       "runs": each adapter's rows lie together (an image's windows, a
            prompt's positions); "mixed": any order, some rows without adapter
  hidden    project: return the rows times the first factor too;
            project_grad: that product is at hand from the forward pass
  gx        project_grad: the gradient of the rows is wanted too

``own`` false: the plain form, elementary float32 operations; true: the calls
of ``paper_1302_1700_amd.fragscan``.
"""
import math

import torch

own = False

_DT = {"f32": torch.float32, "bf16": torch.bfloat16}
_ES = {"f32": 4, "bf16": 2}


def _lp(op, dtype, rows, classes, top=0, temp=1.0, masked=False):
    return {"op": op, "dtype": dtype, "rows": rows, "classes": classes, "top": top, "temp": temp, "masked": masked}


def _pj(op, dtype, rows, k, m, rank, adapters, ids="runs", hidden=False, gx=False):
    return {"op": op, "dtype": dtype, "rows": rows, "k": k, "m": m, "rank": rank, "adapters": adapters, "ids": ids,
            "hidden": hidden, "gx": gx}


def listed():
    cases = [
        # one answer with its alternatives: the smallest call, one row of many classes
        ("logprobs_1x16384_top20", _lp("logprobs", "bf16", 1, 16384, top=20, temp=0.7)),
        # the class map of net N4 on eight 1024 x 1024 images: two classes, one label a window
        ("logprobs_map_8x930x930_2", _lp("logprobs", "f32", 8 * 930 * 930, 2, top=1)),
        # a batch of positions over a large vocabulary: odd rows of odd length, some classes ruled out
        ("logprobs_2047x49999_top5", _lp("logprobs", "bf16", 2047, 49999, top=5, masked=True)),
        # a small labelled batch
        ("logprobs_grad_64x1000", _lp("logprobs_grad", "f32", 64, 1000)),
        # every window of a 1536 x 1536 image, four classes (the bf16 workload's map)
        ("logprobs_grad_map_1476x1476_4", _lp("logprobs_grad", "f32", 1476 * 1476, 4, temp=1.5)),
        # a training batch of positions over a large vocabulary
        ("logprobs_grad_4096x32768", _lp("logprobs_grad", "bf16", 4096, 32768)),
        # one step of 32 requests, each with an adapter of its own choice
        ("project_32x4096x4096_r16", _pj("project", "bf16", 32, 4096, 4096, 16, 32, ids="mixed")),
        # the last layer of N4 over the windows of three 1024 x 1024 images, an adapter an image
        ("project_map_3x930x930_200_2", _pj("project", "f32", 3 * 930 * 930, 200, 2, 4, 3, hidden=True)),
        # whole prompts of seven requests, packed
        ("project_4093x4096x4096_r16", _pj("project", "bf16", 4093, 4096, 4096, 16, 7, hidden=True)),
        # float32 features, a thousand classes
        ("project_1500x1024x1000_r8", _pj("project", "f32", 1500, 1024, 1000, 8, 5, ids="mixed")),
        # fitting the last layer of N4 to eight 512 x 512 images: the features below it are not trained
        ("project_grad_map_8x418x418_200_2", _pj("project_grad", "f32", 8 * 418 * 418, 200, 2, 4, 8, hidden=True)),
        # fitting adapters inside a stack: the rows' gradient goes on down
        ("project_grad_4093x2048x4096_r16", _pj("project_grad", "bf16", 4093, 2048, 4096, 16, 7, hidden=True, gx=True)),
    ]
    return [dict(c, name=n) for n, c in cases]


# the most that a drawn case may hold or compute: about the largest listed ones
_MOST_SCORES = 4096 * 32768
_MOST_ROWS = 8 * 930 * 930
_MOST_VALUES = 3 * 930 * 930 * 200
_MOST_PRODUCTS = 4093 * 4096 * 2048


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        op = rng.choice(["logprobs", "logprobs_grad", "project", "project_grad"])
        dtype = rng.choice(["f32", "bf16"])
        if op.startswith("logprobs"):
            classes = _spread(rng, 2, 131072) if rng.random() < 0.75 else rng.randint(2, 16)
            rows = _spread(rng, 1, min(_MOST_ROWS, _MOST_SCORES // classes))
            # many short rows: at the plain form's cost of a pass over them for each best class
            top = rng.choice([0, 1, 5, 20]) if rows * classes <= _MOST_SCORES // 4 else rng.choice([0, 1, 5])
            return _lp(op, dtype, rows, classes, min(top, classes) if op == "logprobs" else 0,
                       rng.choice([1.0, 1.0, 0.7, 1.5]), rng.random() < 0.3)
        k, m = _spread(rng, 16, 4096), _spread(rng, 2, 4096)
        rows = _spread(rng, 1, _MOST_ROWS)
        rank = rng.choice([1, 2, 4, 8, 8, 16, 16, 32, 64, rng.randint(1, 64)])
        adapters = _spread(rng, 1, 64)
        # the plain form multiplies by the factors of every adapter
        if rows * max(k, m, adapters * rank) > _MOST_VALUES or rows * k * m > _MOST_PRODUCTS:
            continue
        if rows * (k + m) * adapters * rank > 2 * _MOST_PRODUCTS:
            continue
        return _pj(op, dtype, rows, k, m, rank, adapters, rng.choice(["runs", "mixed"]), rng.random() < 0.5,
                   op == "project_grad" and rng.random() < 0.5)


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(gen, shape, scale, dtype):
    return (torch.randn(shape, generator=gen, device="cuda") * scale).to(dtype)


def _inputs_scores(case, seed):
    gen, N, V = _gen(seed), case["rows"], case["classes"]
    x = _normal(gen, (N, V), 2.5, _DT[case["dtype"]])
    if case["masked"]:
        # one class in sixteen ruled out, and one row in 256 wholly
        for i in range(0, N, 65536):
            part = x[i:i + 65536]
            part.masked_fill_(torch.rand(part.shape, generator=gen, device="cuda") < 1 / 16, -math.inf)
            part.masked_fill_(torch.rand((part.shape[0], 1), generator=gen, device="cuda") < 1 / 256, -math.inf)
    labels = torch.randint(0, V, (N,), generator=gen, device="cuda", dtype=torch.int32)
    # windows or positions without a label
    labels.masked_fill_(torch.rand((N,), generator=gen, device="cuda") < 0.1, -1)
    d = {"x": x, "labels": labels}
    if case["op"] == "logprobs_grad":
        # the mean of the labels' log probabilities, a little entropy
        d["g_logp"] = torch.full((N,), -1.0 / N, device="cuda") * (1 + 0.1 * torch.randn((N,), generator=gen, device="cuda"))
        d["g_entropy"] = torch.full((N,), -0.01 / N, device="cuda")
    return d


def _inputs_rows(case, seed):
    gen, N, K, M = _gen(seed), case["rows"], case["k"], case["m"]
    r, n, dt = case["rank"], case["adapters"], _DT[case["dtype"]]
    d = {"x": torch.randn((N, K), generator=gen, device="cuda").tanh_().to(dt),
         "w": _normal(gen, (M, K), K ** -0.5, dt), "bias": torch.randn((M,), generator=gen, device="cuda") * 0.05,
         "a": _normal(gen, (n, r, K), K ** -0.5, dt), "b": _normal(gen, (n, M, r), 0.3 * r ** -0.5, dt),
         "scale": torch.rand((n,), generator=gen, device="cuda") + 0.5}
    if case["ids"] == "runs":
        # the adapters' rows one after the other, of uneven lengths
        cuts = torch.rand((n,), generator=gen, device="cuda").cumsum(0)
        cuts = cuts / cuts[-1] * N
        ids = torch.searchsorted(cuts, torch.arange(N, device="cuda") + 0.5).clamp_(max=n - 1)
        d["ids"] = ids.to(torch.int32)
    else:
        d["ids"] = torch.randint(-1 if n > 1 else 0, n, (N,), generator=gen, device="cuda", dtype=torch.int32)
    if case["op"] == "project_grad":
        d["g"] = _normal(gen, (N, M), 1.0 / N, dt)
    return d


def prepare(case, seed):
    """The inputs; for a gradient also what its forward pass left."""
    if case["op"].startswith("logprobs"):
        state = _inputs_scores(case, seed)
        if case["op"] == "logprobs_grad":
            _, state["entropy"], state["norm"] = _plain_logprobs(state["x"], state["labels"], case["temp"], 0)[:3]
    else:
        state = _inputs_rows(case, seed)
        state["h"] = None
        if case["op"] == "project_grad" and case["hidden"]:
            state["h"] = _plain_hidden(state["x"], state["a"], state["ids"])[0]
    state["case"] = case
    return state


# -- the plain form ------------------------------------------------------------
def _plain_logprobs(x, labels, temp, top):
    x = x.float()
    N, V = x.shape
    big = x.amax(1, keepdim=True)
    empty = big[:, 0] == -math.inf
    d = (x - torch.where(big == -math.inf, torch.zeros_like(big), big)) / temp
    e = d.exp()
    s = e.sum(1).where(~empty, torch.ones_like(big[:, 0]))
    log_s = s.log()
    entropy = log_s - (e * d.clamp(min=-1e30)).sum(1) / s
    y = labels.long()
    at = d.gather(1, y.clamp(min=0)[:, None])[:, 0]
    logp = torch.where(y < 0, torch.zeros_like(at), at - log_s)
    norm = torch.stack([big[:, 0], log_s], 1)
    if not top:
        return logp, entropy, norm
    ids, vals, left = [], [], d.clone()
    iota = torch.arange(V, device=x.device, dtype=torch.int32)
    for _ in range(top):
        v = left.amax(1, keepdim=True)
        i = torch.where(left == v, iota, V).amin(1)
        none = v[:, 0] == -math.inf
        ids.append(torch.where(none, -torch.ones_like(i), i))
        vals.append(v[:, 0] - log_s)
        left.scatter_(1, i.long()[:, None], -math.inf)
    return logp, entropy, norm, torch.stack(ids, 1).to(torch.int32), torch.stack(vals, 1)


def _plain_logprobs_grad(st, temp):
    x, norm, y = st["x"].float(), st["norm"], st["labels"].long()
    empty = norm[:, :1] == -math.inf
    logp = (x - torch.where(empty, torch.zeros_like(norm[:, :1]), norm[:, :1])) / temp - norm[:, 1:]
    p = logp.exp()
    gl = torch.where(y < 0, torch.zeros_like(st["g_logp"]), st["g_logp"])[:, None]
    g = -gl * p - st["g_entropy"][:, None] * p * (logp.clamp(min=-1e30) + st["entropy"][:, None])
    g.scatter_add_(1, y.clamp(min=0)[:, None], gl)
    return torch.where(empty, torch.zeros_like(g), g / temp).to(st["x"].dtype)


def _plain_hidden(x, a, ids):
    """Rows times every adapter's first factor, and which of the products count."""
    n, r, K = a.shape
    every = x.float() @ a.float().reshape(n * r, K).t()
    mine = ids[:, None] == torch.arange(n, device=x.device, dtype=torch.int32)
    kept = every.view(-1, n, r) * mine[:, :, None]
    return kept.sum(1), kept.reshape(-1, n * r), mine


def _plain_project(st, hidden):
    x, b = st["x"], st["b"].float()
    n, M, r = b.shape
    h, kept, _ = _plain_hidden(x, st["a"], st["ids"])
    fold = (b * st["scale"][:, None, None]).permute(1, 0, 2).reshape(M, n * r)
    y = (x.float() @ st["w"].float().t() + st["bias"] + kept @ fold.t()).to(x.dtype)
    return (y, h) if hidden else y


def _plain_project_grad(st, gx):
    x, g, a = st["x"].float(), st["g"].float(), st["a"].float()
    b = st["b"].float() * st["scale"][:, None, None]
    n, M, r = b.shape
    K = x.shape[1]
    if st["h"] is None:
        _, kept, mine = _plain_hidden(st["x"], st["a"], st["ids"])
    else:
        mine = st["ids"][:, None] == torch.arange(n, device=x.device, dtype=torch.int32)
        kept = (st["h"][:, None, :] * mine[:, :, None]).reshape(-1, n * r)
    u = (g @ b.permute(1, 0, 2).reshape(M, n * r)).view(-1, n, r) * mine[:, :, None]
    u = u.reshape(-1, n * r)
    ga = (u.t() @ x).view(n, r, K)
    gb = (kept.t() @ g).view(n, r, M).transpose(1, 2) * st["scale"][:, None, None]
    out = (ga.to(st["a"].dtype), gb.to(st["b"].dtype).contiguous())
    if not gx:
        return out
    return ((g @ st["w"].float() + u @ a.reshape(n * r, K)).to(st["x"].dtype),) + out


def run(state):
    case = state["case"]
    op = case["op"]
    if not own:
        if op == "logprobs":
            return _plain_logprobs(state["x"], state["labels"], case["temp"], case["top"])
        if op == "logprobs_grad":
            return _plain_logprobs_grad(state, case["temp"])
        if op == "project":
            return _plain_project(state, case["hidden"])
        return _plain_project_grad(state, case["gx"])
    from paper_1302_1700_amd import fragscan
    if op == "logprobs":
        r = fragscan.logprobs(state["x"], state["labels"], n_top=case["top"], temperature=case["temp"])
        return (r.logp, r.entropy, r.norm) + ((r.top_id, r.top_logp) if case["top"] else ())
    if op == "logprobs_grad":
        return fragscan.logprobs_grad(state["x"], state["norm"], state["labels"], state["g_logp"],
                                      entropy=state["entropy"], g_entropy=state["g_entropy"],
                                      temperature=case["temp"])
    adapters = fragscan.Adapters(state["a"], state["b"], state["scale"])
    if op == "project":
        return fragscan.project(state["x"], state["w"], state["bias"], adapters, state["ids"],
                                return_hidden=case["hidden"])
    gx, ga, gb = fragscan.project_grad(state["g"], state["x"], state["w"], adapters, state["ids"], hidden=state["h"],
                                       need_x=case["gx"])
    return (gx, ga, gb) if case["gx"] else (ga, gb)


def work(case):
    es, N = _ES[case["dtype"]], case["rows"]
    if case["op"].startswith("logprobs"):
        V = case["classes"]
        if case["op"] == "logprobs":
            return {"bytes": N * V * es + N * (4 + 16 + 8 * case["top"]), "flops": 6 * N * V}
        return {"bytes": 2 * N * V * es + N * 24, "flops": 8 * N * V}
    K, M, r = case["k"], case["m"], case["rank"]
    used = min(case["adapters"], N)
    factors = used * r * (K + M) * es
    if case["op"] == "project":
        return {"bytes": N * (K + M) * es + M * K * es + factors + 4 * (N + M) + (4 * N * r if case["hidden"] else 0),
                "flops": 2 * N * K * M + 2 * N * r * (K + M)}
    nbytes = N * (K + M) * es + 4 * N + factors + case["adapters"] * r * (K + M) * es + (4 * N * r if case["hidden"] else 0)
    flops = (4 * M + 2 * K + (0 if case["hidden"] else 2 * K)) * N * r
    if case["gx"]:
        nbytes += N * K * es + M * K * es
        flops += 2 * N * K * M + 2 * N * r * K
    return {"bytes": nbytes, "flops": flops}


# -- the definitions in float64 ----------------------------------------------------
def _exact_rows(x, labels, temp, top):
    z = x.double() / temp
    empty = (z == -math.inf).all(1)
    z0 = z.masked_fill(empty[:, None], 0.0)
    logp = z0 - z0.logsumexp(1, keepdim=True)
    p = logp.exp()
    entropy = -torch.where(p > 0, p * logp, torch.zeros_like(p)).sum(1)
    most = x.double().amax(1)
    log_s = z0.logsumexp(1) - z0.amax(1)
    logp = logp.masked_fill(empty[:, None], -math.inf)
    entropy, log_s = entropy.masked_fill(empty, 0.0), log_s.masked_fill(empty, 0.0)
    y = labels.long()
    given = torch.zeros_like(most)
    has = y >= 0
    given[has] = logp[has].gather(1, y[has][:, None])[:, 0]
    out = [given, entropy, torch.stack([most, log_s], 1)]
    if top:
        v, i = logp.sort(stable=True, dim=1, descending=True)
        v, i = v[:, :top].contiguous(), i[:, :top]
        out += [torch.where(v == -math.inf, torch.full_like(i, -1), i).to(torch.int32), v]
    return out, logp, p


def _exact_scores(case, seed):
    d = _inputs_scores(case, seed)
    x, y, temp = d["x"], d["labels"], case["temp"]
    # rows at a time, so that the float64 copies of the scores stay small
    step = max(1, (1 << 26) // case["classes"])
    parts = []
    for i in range(0, case["rows"], step):
        s = slice(i, i + step)
        out, logp, p = _exact_rows(x[s], y[s], temp, case["top"])
        if case["op"] == "logprobs_grad":
            gl, ge = d["g_logp"][s].double(), d["g_entropy"][s].double()
            gl = torch.where(y[s] < 0, torch.zeros_like(gl), gl)
            hot = torch.zeros_like(p)
            hot.scatter_(1, y[s].long().clamp(min=0)[:, None], 1.0)
            plogp = torch.where(p > 0, p * logp, torch.zeros_like(p))
            g = (gl[:, None] * (hot - p) - ge[:, None] * (plogp + p * out[1][:, None])) / temp
            out = [g.masked_fill((x[s] == -math.inf).all(1)[:, None], 0.0)]
        parts.append(out)
    whole = tuple(torch.cat(c) for c in zip(*parts))
    return whole if case["op"] == "logprobs" else whole[0]


def _exact_map(case, seed):
    d = _inputs_rows(case, seed)
    n, scale = case["adapters"], d["scale"].double()
    a, b, w = d["a"].double(), d["b"].double(), d["w"].double()
    N, K, M, r = case["rows"], case["k"], case["m"], case["rank"]
    wide = lambda cols: torch.zeros((N, cols), dtype=torch.float64, device="cuda")
    if case["op"] == "project":
        y, h = wide(M), wide(r)
        for i in range(-1, n):
            rows = (d["ids"] == i).nonzero()[:, 0]
            x = d["x"][rows].double()
            y[rows] = torch.addmm(d["bias"].double(), x, w.t().contiguous())
            if i >= 0:
                h[rows] = x @ a[i].t().contiguous()
                y[rows] += scale[i] * (h[rows] @ b[i].t().contiguous())
        return (y, h) if case["hidden"] else y
    ga, gb, gx = torch.zeros_like(a), torch.zeros_like(b), wide(K if case["gx"] else 0)
    for i in range(-1, n):
        rows = (d["ids"] == i).nonzero()[:, 0]
        x, g = d["x"][rows].double(), d["g"][rows].double()
        if case["gx"]:
            gx[rows] = g @ w
        if i >= 0:
            u = scale[i] * (g @ b[i])
            ga[i] = u.t().contiguous() @ x
            gb[i] = scale[i] * (g.t().contiguous() @ (x @ a[i].t().contiguous()))
            if case["gx"]:
                gx[rows] += u @ a[i]
    return (gx, ga, gb) if case["gx"] else (ga, gb)


def exact(case, seed):
    if case["op"].startswith("logprobs"):
        return _exact_scores(case, seed)
    return _exact_map(case, seed)
