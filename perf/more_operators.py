"""The operators around the expert layer that fine-tuning and adapted serving need, as they are measured: rows sorted by
expert and back, and low-rank adapters beside a shared projection.

* ``sort``: every token's row to the sorted places of its slots, by choice times the slot's gate.
* ``combine``: the gate-weighted sum of each token's sorted rows, by choice added to another matrix.
* ``combine_grad``: the gradient of that sum with respect to the sorted rows and to the gates.
* ``adapters``: y = add + s B (A x) with a pair (A, B) for each segment of rows: requests with adapters of their own beside
  a shared projection, or rows sorted by expert with one adapter an expert.
* ``adapters_grad``: its gradient with respect to x, A and B.

The plain forms are elementary torch operations in 32 bits.  ``own`` runs the library's calls instead.  Sizes are those of
a layer with 256 experts, hidden size 7168, expert size 2048 and a shared gate-up projection of 4096, and generic ones.
"""
from __future__ import annotations

from types import SimpleNamespace

import torch

own = False

DEVICE = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}


def _rows(name, kind, T, k, H, dtype="bf16", E=256, ep=1, weighted=True, add=False):
    return {"name": name, "kind": kind, "T": T, "k": k, "H": H, "dtype": dtype, "E": E, "ep": ep, "weighted": weighted,
            "add": add}


def _adapters(name, kind, T, L, r, K, N, dtype="bf16", wdtype="bf16", seqs=None, bare=False, order="requests", save=False):
    return {"name": name, "kind": kind, "T": T, "L": L, "r": r, "K": K, "N": N, "dtype": dtype, "wdtype": wdtype,
            "seqs": T if seqs is None else seqs, "bare": bare, "order": order, "save": save}


def listed():
    return [
        # One decoded token to its eight experts: latency alone.
        _rows("sort_t1", "sort", 1, 8, 7168, weighted=False),
        # Prefill: the largest batch of rows that is laid out for grouped products.
        _rows("sort_t8192", "sort", 8192, 8, 7168, weighted=False),
        # A ragged decode batch on one of eight ranks: most slots belong to other ranks.
        _rows("combine_t37_rank", "combine", 37, 8, 7168, ep=8),
        # Prefill, added to the shared expert's output.
        _rows("combine_t8192", "combine", 8192, 8, 7168, add=True),
        # A micro-batch of a fine-tuning run in fp32, odd in its number of tokens.
        _rows("combine_grad_t509_f32", "combine_grad", 509, 8, 2048, "f32"),
        # The training batch: rows and gradients of rows are the whole traffic.
        _rows("combine_grad_t8192", "combine_grad", 8192, 8, 7168),
        # Single-stream decode with one of eight loaded adapters beside the gate-up projection.
        _adapters("adapters_t1", "adapters", 1, 8, 16, 7168, 4096),
        # A decode batch: 61 requests over 48 adapters, some without one, beside the down projection.
        _adapters("adapters_t61", "adapters", 61, 48, 16, 2048, 7168, bare=True),
        # Prefill of 37 requests over 12 adapters, A x kept for the gradient.
        _adapters("adapters_t8192", "adapters", 8192, 12, 32, 7168, 4096, seqs=37, bare=True, save=True),
        # An adapter for each of 256 experts, fp32 masters, on rows sorted by expert.
        _adapters("adapters_experts", "adapters", 4096, 256, 8, 7168, 2048, wdtype="f32", order="sorted"),
        # A small micro-batch of three adapters with fp32 masters.
        _adapters("adapters_grad_t300", "adapters_grad", 300, 3, 8, 2048, 7168, wdtype="f32", seqs=5),
        # The training batch of one adapter of a larger rank.
        _adapters("adapters_grad_t8192", "adapters_grad", 8192, 1, 32, 7168, 4096, seqs=16),
    ]


def draw(rng):
    """One more call of the ranges above, sizes spread over their logarithm."""
    def log_int(lo, hi):
        return min(hi, max(lo, int(round(lo * (hi / lo) ** rng.random()))))

    kind = rng.choice(["sort", "combine", "combine_grad", "adapters", "adapters_grad"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind in ("sort", "combine", "combine_grad"):
        k, H = rng.choice([1, 2, 4, 6, 8, 8, 10, 16]), rng.choice([log_int(64, 8192), 8 * log_int(8, 1024)])
        T = log_int(1, max(1, min(8192, 8192 * 8 * 7168 * 2 // (k * H * SIZE[dtype]))))
        c = _rows("", kind, T, k, H, dtype, rng.choice([40, 64, 128, 256, 384]), rng.choice([1, 1, 8]),
                  rng.choice([True, True, False]), rng.choice([True, False]))
    else:
        r = rng.choice([4, 8, 16, 32, 64, log_int(1, 64)])
        K, N = (rng.choice([log_int(64, 7168), 8 * log_int(8, 896)]) for _ in range(2))
        most = 8192 * 32 * (7168 + 4096) // (r * (K + N))
        T = log_int(1, max(1, min(8192, most) // (SIZE[dtype] // 2)))
        c = _adapters("", kind, T, log_int(1, 64), r, K, N, dtype, rng.choice(["bf16", "bf16", "f32"]),
                      rng.choice([T, log_int(1, T)]), rng.choice([True, False]), rng.choice(["requests", "requests", "sorted"]),
                      rng.choice([True, False]))
    del c["name"]
    return c


# ---------------------------------------------------------------- inputs

def _generator(seed, what):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(1000033 * int(seed) + what)
    return g


def _randn(shape, seed, what):
    return torch.randn(shape, generator=_generator(seed, what), device=DEVICE)


def _rand(shape, seed, what):
    return torch.rand(shape, generator=_generator(seed, what), device=DEVICE)


def _activations(shape, seed, what):
    """Rows of normal values, a few channels 8 times as large."""
    x = _randn(shape, seed, what)
    x[:, torch.randint(0, shape[1], (max(1, shape[1] // 256),), generator=_generator(seed, what + 1), device=DEVICE)] *= 8
    return x


def _places(ids, n):
    """Stable order of the ids 0 .. n - 1 (others are left out): perm, its inverse (-1) and the offsets."""
    key = torch.where((ids >= 0) & (ids < n), ids, n)
    perm = torch.argsort(key, stable=True)
    inv = torch.empty_like(perm)
    inv[perm] = torch.arange(perm.numel(), device=DEVICE)
    count = torch.bincount(key, minlength=n + 1)[:n]
    offsets = torch.cat([torch.zeros(1, dtype=torch.int64, device=DEVICE), torch.cumsum(count, 0)])
    inv = torch.where(key < n, inv, -1)
    return perm.to(torch.int32), inv.to(torch.int32), offsets.to(torch.int32)


def _prepare_rows(s, case, seed):
    T, k, H, E, d = case["T"], case["k"], case["H"], case["E"], DTYPES[case["dtype"]]
    top = torch.topk(_randn((T, E), seed, 1) + 0.7 * _randn((1, E), seed, 2), k, dim=1)
    s.w = torch.softmax(top.values, dim=1).contiguous() if case["weighted"] else None
    ids = top.indices.reshape(-1)
    s.perm, s.inv, offsets = _places(ids, E // case["ep"])  # a rank holds the first experts, other slots are masked
    s.n = int(offsets[-1])
    shape = (T * k, H)
    if case["kind"] == "sort":
        s.x = _activations((T, H), seed, 3).to(d)
        s.rows = torch.zeros(shape, dtype=d, device=DEVICE)
        return
    s.rows = _activations(shape, seed, 3).to(d)
    if case["kind"] == "combine":
        s.add = _randn((T, H), seed, 5).to(d) if case["add"] else None
        s.y = torch.empty((T, H), dtype=d, device=DEVICE)
        return
    s.dy = (_randn((T, H), seed, 6) * 1e-2).to(d)
    s.drows = torch.zeros(shape, dtype=d, device=DEVICE)
    s.dw = torch.empty((T, k), device=DEVICE)


def _prepare_adapters(s, case, seed):
    T, L, r, K, N = (case[n] for n in ("T", "L", "r", "K", "N"))
    d, dw = DTYPES[case["dtype"]], DTYPES[case["wdtype"]]
    # Requests of random lengths, each with an adapter of its own choice or (bare) one in eight without any.
    if case["seqs"] >= T:
        request = torch.arange(T, device=DEVICE)
    else:
        cuts = torch.cumsum(_rand((case["seqs"],), seed, 1).double() + 0.1, 0)
        ends = torch.round(cuts / cuts[-1] * T)
        request = (torch.arange(T, device=DEVICE)[:, None] >= ends[None, :-1]).sum(dim=1)
    ids = torch.randint(0, L, (max(case["seqs"], T),), generator=_generator(seed, 2), device=DEVICE)[request]
    if case["bare"]:
        ids = torch.where(_rand((max(case["seqs"], T),), seed, 3)[request] < 1 / 8, -1, ids)
    s.perm, _, s.offsets = _places(ids, L)
    if case["order"] == "sorted":
        s.perm = None
    s.bounds = s.offsets.tolist()  # what the program that batches requests knows on the host
    s.x = _activations((T, K), seed, 4).to(d)
    s.a = (_randn((L, r, K), seed, 6) * K ** -0.5).to(dw)
    s.b = (_randn((L, N, r), seed, 7) * r ** -0.5).to(dw)
    s.scale = 0.5 + 1.5 * _rand((L,), seed, 8)
    if case["kind"] == "adapters":
        s.add = _randn((T, N), seed, 9).to(d)
        s.y = torch.zeros((T, N), dtype=d, device=DEVICE)
        s.u = torch.zeros((T, r), device=DEVICE) if case["save"] else None
        return
    s.dy = (_randn((T, N), seed, 10) * 1e-2).to(d)
    s.add = (_randn((T, K), seed, 11) * 1e-2).to(d)
    s.u = torch.zeros((T, r), device=DEVICE)  # what the forward call left
    for l, rows, p in _segments(s):
        s.u[p] = s.x[rows].float() @ s.a[l].float().t()
    s.dx = torch.zeros((T, K), dtype=d, device=DEVICE)
    s.da = torch.empty((L, r, K), device=DEVICE)
    s.db = torch.empty((L, N, r), device=DEVICE)


def prepare(case, seed):
    s = SimpleNamespace(case=dict(case), ws=None)
    (_prepare_rows if "H" in case else _prepare_adapters)(s, case, seed)
    return s


# ---------------------------------------------------------------- the plain forms

def _slots(s):
    """Row of each slot [T][k] (0 where there is none), its factor, and whether there is one."""
    inv = s.inv.view(s.case["T"], s.case["k"])
    return inv.clamp_min(0).long(), s.w if s.w is not None else torch.ones(inv.shape, device=DEVICE), inv >= 0


def _spread(s, x):
    """w x in sorted order, zeros behind the last row."""
    k = s.case["k"]
    slot = s.perm[: s.n].long()
    v = x.float()[slot // k]
    if s.w is not None:
        v = v * s.w.view(-1)[slot][:, None]
    out = torch.zeros((s.case["T"] * k, s.case["H"]), dtype=x.dtype, device=DEVICE)
    out[: s.n] = v.to(x.dtype)
    return out


def _plain_sort(s):
    return {"rows": _spread(s, s.x)}


def _plain_combine(s):
    at, w, ok = _slots(s)
    y = torch.zeros((s.case["T"], s.case["H"]), device=DEVICE) if s.add is None else s.add.float()
    for j in range(s.case["k"]):
        y = y + torch.where(ok[:, j, None], w[:, j, None] * s.rows[at[:, j]].float(), 0)
    return {"y": y.to(s.rows.dtype)}


def _plain_combine_grad(s):
    at, _, ok = _slots(s)
    dy = s.dy.float()
    dw = torch.stack([(dy * s.rows[at[:, j]].float()).sum(dim=1) for j in range(s.case["k"])], dim=1)
    return {"drows": _spread(s, s.dy), "dw": torch.where(ok, dw, 0)}


def _segments(s):
    """Adapter, rows of x and places of every segment that is not empty."""
    for l, (lo, hi) in enumerate(zip(s.bounds[:-1], s.bounds[1:])):
        if hi > lo:
            yield l, slice(lo, hi) if s.perm is None else s.perm[lo:hi].long(), slice(lo, hi)


def _plain_adapters(s):
    y = torch.zeros_like(s.y)
    u = torch.zeros((s.case["T"], s.case["r"]), device=DEVICE)
    for l, rows, p in _segments(s):
        u[p] = s.x[rows].float() @ s.a[l].float().t()
        y[rows] = (s.add[rows].float() + s.scale[l] * (u[p] @ s.b[l].float().t())).to(y.dtype)
    return {"y": y, "u": u} if s.u is not None else {"y": y}


def _plain_adapters_grad(s):
    dx, da, db = torch.zeros_like(s.dx), torch.zeros_like(s.da), torch.zeros_like(s.db)
    for l, rows, p in _segments(s):
        x, dy, a = s.x[rows].float(), s.dy[rows].float() * s.scale[l], s.a[l].float()
        g = dy @ s.b[l].float()
        dx[rows] = (s.add[rows].float() + g @ a).to(dx.dtype)
        da[l] = g.t() @ x
        db[l] = dy.t() @ s.u[p]
    return {"dx": dx, "da": da, "db": db}


_PLAIN = {"sort": _plain_sort, "combine": _plain_combine, "combine_grad": _plain_combine_grad, "adapters": _plain_adapters,
          "adapters_grad": _plain_adapters_grad}


def run(state):
    return (_OWN if own else _PLAIN)[state.case["kind"]](state)


# ---------------------------------------------------------------- the library's calls

def _own_sort(s):
    from paper_2607_23099_amd import damoe
    damoe.sort_rows(s.x, s.case["T"], s.case["k"], s.case["H"], s.inv, s.rows, w=s.w)
    return {"rows": s.rows}


def _own_combine(s):
    from paper_2607_23099_amd import damoe
    damoe.combine_rows(s.rows, s.case["T"], s.case["k"], s.case["H"], s.inv, s.y, w=s.w, add=s.add)
    return {"y": s.y}


def _own_combine_grad(s):
    from paper_2607_23099_amd import damoe
    damoe.combine_rows_grad(s.dy, s.rows, s.case["T"], s.case["k"], s.case["H"], s.inv, w=s.w, drows=s.drows, dw=s.dw)
    return {"drows": s.drows, "dw": s.dw}


def _own_adapters(s):
    from paper_2607_23099_amd import damoe
    T, L, r, K, N = (s.case[n] for n in ("T", "L", "r", "K", "N"))
    if s.ws is None:
        s.ws = torch.empty(damoe.adapters_workspace_size(T, L, r, K, N), dtype=torch.uint8, device=DEVICE)
    damoe.adapters(s.x, T, s.a, s.b, s.offsets, s.y, s.ws, perm=s.perm, scale=s.scale, add=s.add, u=s.u)
    return {"y": s.y, "u": s.u} if s.u is not None else {"y": s.y}


def _own_adapters_grad(s):
    from paper_2607_23099_amd import damoe
    T, L, r, K, N = (s.case[n] for n in ("T", "L", "r", "K", "N"))
    if s.ws is None:
        s.ws = torch.empty(damoe.adapters_grad_workspace_size(T, L, r, K, N), dtype=torch.uint8, device=DEVICE)
    damoe.adapters_grad(s.x, s.dy, s.u, T, s.a, s.b, s.offsets, s.da, s.db, s.ws, perm=s.perm, scale=s.scale, add=s.add,
                        dx=s.dx)
    return {"dx": s.dx, "da": s.da, "db": s.db}


_OWN = {"sort": _own_sort, "combine": _own_combine, "combine_grad": _own_combine_grad, "adapters": _own_adapters,
        "adapters_grad": _own_adapters_grad}


# ---------------------------------------------------------------- work and exact values

def work(case):
    T, b = case["T"], SIZE[case["dtype"]]
    if "H" in case:
        H, k = case["H"], case["k"]
        A = T * k / case["ep"]
        gates = T * k * (8 if case["weighted"] else 4)  # and the places
        if case["kind"] == "sort":
            return {"bytes": (T + A) * H * b + gates, "flops": A * H if case["weighted"] else 0}
        if case["kind"] == "combine":
            return {"bytes": (A + T * (2 if case["add"] else 1)) * H * b + gates, "flops": 2 * A * H}
        return {"bytes": (2 * A + T) * H * b + gates + T * k * 4, "flops": 3 * A * H}
    L, r, K, N = (case[n] for n in ("L", "r", "K", "N"))
    n = T * (7 / 8 if case["bare"] else 1)
    used = L * (1 - (1 - 1 / L) ** case["seqs"])
    weights = used * r * (K + N) * SIZE[case["wdtype"]]
    if case["kind"] == "adapters":
        return {"bytes": n * (K + 2 * N) * b + weights + (n * r * 4 if case["save"] else 0), "flops": 2 * n * r * (K + N)}
    return {"bytes": n * (3 * K + N) * b + weights + n * r * 4 + L * r * (K + N) * 4, "flops": 4 * n * r * (K + N)}


def _exact_rows(case, s):
    T, k, H = case["T"], case["k"], case["H"]
    w = torch.ones((T, k), dtype=torch.float64, device=DEVICE) if s.w is None else s.w.double()
    inv = s.inv.view(T, k).long()
    slots = []  # slot by slot: the tokens that have a row there, and which
    for j in range(k):
        t = torch.nonzero(inv[:, j] >= 0).view(-1)
        slots.append((j, t, inv[t, j]))
    if case["kind"] == "combine":
        y = torch.zeros((T, H), dtype=torch.float64, device=DEVICE) if s.add is None else s.add.double()
        for j, t, q in slots:
            y[t] += w[t, j, None] * s.rows[q].double()
        return {"y": y}
    rows = torch.zeros((T * k, H), dtype=torch.float64, device=DEVICE)
    dw = torch.zeros((T, k), dtype=torch.float64, device=DEVICE)
    for j, t, q in slots:
        v = (s.x if case["kind"] == "sort" else s.dy)[t].double()
        rows[q] = w[t, j, None] * v
        if case["kind"] == "combine_grad":
            dw[t, j] = torch.linalg.vecdot(v, s.rows[q].double())
    return {"rows": rows} if case["kind"] == "sort" else {"drows": rows, "dw": dw}


def exact(case, seed):
    s = prepare(case, seed)
    if "H" in case:
        return _exact_rows(case, s)
    T, L, r, K, N = (case[n] for n in ("T", "L", "r", "K", "N"))
    f64 = dict(dtype=torch.float64, device=DEVICE)
    order = torch.arange(T, device=DEVICE) if s.perm is None else s.perm.long()
    out = {"y": torch.zeros((T, N), **f64), "u": torch.zeros((T, r), **f64), "dx": torch.zeros((T, K), **f64),
           "da": torch.zeros((L, r, K), **f64), "db": torch.zeros((L, N, r), **f64)}
    place = torch.arange(T, device=DEVICE)
    segment = torch.searchsorted(s.offsets[1:].contiguous().long(), place, right=True)
    for l in range(L):
        p = place[segment == l]
        if not p.numel():
            continue
        t, scale = order[p], float(s.scale[l])
        a, b, x = s.a[l].double(), s.b[l].double(), s.x[t].double()
        if case["kind"] == "adapters":
            out["u"][p] = torch.matmul(x, a.t().contiguous())
            out["y"][t] = s.add[t].double() + torch.matmul(out["u"][p], (scale * b).t().contiguous())
            continue
        dy = s.dy[t].double()
        g = torch.matmul(dy, scale * b)
        out["dx"][t] = s.add[t].double() + torch.matmul(g, a)
        out["da"][l] = torch.matmul(g.t().contiguous(), x)
        out["db"][l] = torch.matmul((scale * dy).t().contiguous(), s.u[p].double())
    names = ["dx", "da", "db"] if case["kind"] == "adapters_grad" else ["y", "u"] if case["save"] else ["y"]
    return {n: out[n] for n in names}
