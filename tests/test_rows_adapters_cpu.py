"""What the row and adapter calls refuse, in the library and in the binding (no GPU: every call ends before a launch)."""
import os
import random

import pytest

torch = pytest.importorskip("torch")

from paper_2607_23099_amd import build, damoe

BAD, UNSUPPORTED, WORKSPACE = -1, -2, -3
P, Q, BIG = 0x10000, 0x20000, 1 << 40  # addresses that are never dereferenced


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not os.path.exists(damoe.LIB_PATH):
        build.build_damoe()


# Arguments of a valid call by name, in order.
SORT = dict(x=P, dtype=1, ldx=64, w=P, inv=P, T=4, k=2, H=64, R=8, rows=Q, ld_rows=64, stream=0)
COMBINE = dict(rows=P, dtype=1, ld_rows=64, w=P, inv=P, T=4, k=2, H=64, R=8, add=P, ld_add=64, y=Q, ldy=64, stream=0)
GRAD = dict(dy=P, dtype=1, ldy=64, rows=P, ld_rows=64, w=P, inv=P, T=4, k=2, H=64, R=8, drows=Q, ld_drows=64, dw=P, stream=0)
ADAPTERS = dict(x=P, xdtype=1, ldx=64, perm=P, offsets=P, T=4, L=3, a=P, b=P, wdtype=0, r=8, K=64, N=48, scale=P, add=P, ld_add=48,
                y=Q, ydtype=1, ldy=48, u=P, ws=P, ws_bytes=BIG, stream=0)
ADAPTERS_GRAD = dict(x=P, xdtype=1, ldx=64, dy=P, ydtype=1, ldy=48, u=P, perm=P, offsets=P, T=4, L=3, a=P, b=P, wdtype=0, r=8, K=64,
                     N=48, scale=P, add=P, ld_add=64, dx=Q, ld_dx=64, da=P, db=P, accumulate=0, ws=P, ws_bytes=BIG, stream=0)
ROWS = {BAD: [dict(T=-1), dict(T=(1 << 20) + 1), dict(k=0), dict(k=17), dict(H=0), dict(R=-1), dict(inv=0), dict(inv=P + 2), dict(w=P + 1)],
        UNSUPPORTED: [dict(dtype=2), dict(dtype=-1), dict(H=(1 << 20) + 1)]}
SIZES = {BAD: [dict(T=-1), dict(T=(1 << 20) + 1), dict(L=0), dict(L=1025), dict(r=0), dict(K=0), dict(N=0), dict(x=0), dict(x=P + 2),
               dict(ldx=63), dict(perm=P + 2), dict(offsets=0), dict(offsets=P + 2), dict(a=0), dict(b=0), dict(a=P + 1), dict(b=P + 1),
               dict(scale=P + 2), dict(u=P + 2), dict(ws=0), dict(ws=P + 8), dict(add=P + 2)],
         UNSUPPORTED: [dict(xdtype=2), dict(wdtype=2), dict(ydtype=-1), dict(r=129), dict(K=(1 << 20) + 1), dict(N=(1 << 20) + 1)],
         WORKSPACE: [dict(ws_bytes=0), dict(ws_bytes=255)]}
CALLS = [
    (3, damoe._SORT_WORDS, SORT, ROWS, {BAD: [dict(x=0), dict(x=P + 2), dict(ldx=63), dict(rows=0), dict(rows=Q + 2), dict(ld_rows=63)]}),
    (4, damoe._COMBINE_WORDS, COMBINE, ROWS, {BAD: [dict(rows=0), dict(rows=P + 2), dict(ld_rows=63), dict(add=P + 2), dict(ld_add=63),
                                                    dict(y=0), dict(y=Q + 2), dict(ldy=63), dict(add=Q, ld_add=65)]}),
    (5, damoe._COMBINE_GRAD_WORDS, GRAD, ROWS, {BAD: [dict(dy=0), dict(dy=P + 2), dict(ldy=63), dict(rows=0), dict(rows=P + 2),
                                                      dict(ld_rows=63), dict(drows=Q + 2), dict(ld_drows=63), dict(dw=P + 2),
                                                      dict(rows=Q, ld_rows=65)]}),
    (6, damoe._ADAPTERS_WORDS, ADAPTERS, SIZES, {BAD: [dict(y=0), dict(y=Q + 2), dict(ldy=47), dict(ld_add=47), dict(add=Q, ld_add=49)]}),
    (7, damoe._ADAPTERS_GRAD_WORDS, ADAPTERS_GRAD, SIZES, {BAD: [dict(dy=0), dict(dy=P + 2), dict(ldy=47), dict(u=0), dict(dx=Q + 2),
                                                                 dict(ld_dx=63), dict(ld_add=63), dict(add=Q, ld_add=65), dict(da=0),
                                                                 dict(db=0), dict(da=P + 2), dict(db=P + 1), dict(accumulate=2)]}),
]


@pytest.mark.parametrize("fn,pack,good,shared,own", CALLS, ids=["sort", "combine", "combine_grad", "adapters", "adapters_grad"])
def test_refusals_of_the_library(fn, pack, good, shared, own):
    call = damoe.lib().damoe_call_words
    for table in (shared, own):
        for status, changes in table.items():
            for change in changes:
                assert set(change) <= set(good), change
                words = {**good, **change}
                assert call(fn, pack(*words.values()), len(words)) == status, change
    for n in (0, len(good) - 1, len(good) + 1):
        assert call(fn, pack(*good.values()), n) == BAD
    assert call(fn, None, len(good)) == BAD


def test_calls_without_tokens_launch_nothing():
    call = damoe.lib().damoe_call_words
    for fn, pack, good, _, _ in CALLS[:4]:
        words = {**good, "T": 0, "x": 0, "rows": 0, "y": 0, "dy": 0}
        assert call(fn, pack(*[words[n] for n in good]), len(good)) == 0
    for change in (dict(R=0),):
        assert call(3, damoe._SORT_WORDS(*{**SORT, **change, "rows": 0}.values()), len(SORT)) == 0
    assert call(5, damoe._COMBINE_GRAD_WORDS(*{**GRAD, "drows": 0, "dw": 0}.values()), len(GRAD)) == 0


def test_workspace_sizes():
    for f in (damoe.adapters_workspace_size, damoe.adapters_grad_workspace_size):
        for bad in [(-1, 1, 1, 1, 1), (1, 0, 1, 1, 1), (1, 1025, 1, 1, 1), (1, 1, 0, 1, 1), (1, 1, 129, 1, 1), (1, 1, 1, 0, 1),
                    (1, 1, 1, 1, 0), ((1 << 20) + 1, 1, 1, 1, 1), (1, 1, 1, (1 << 20) + 1, 1)]:
            assert f(*bad) == 0
        assert f(0, 1, 1, 1, 1) > 0


@pytest.mark.parametrize("size", [damoe.adapters_workspace_size, damoe.adapters_grad_workspace_size], ids=["forward", "gradient"])
def test_a_workspace_for_more_rows_serves_fewer(size):
    for r, K, N in ((3, 200, 8192), (33, 8192, 100), (128, 4096, 4096), (16, 64, 64)):
        last = 0
        for T in sorted({1 << i for i in range(21)} | {(1 << i) + d for i in range(5, 14) for d in (-1, 1)}):
            now = size(T, 3, r, K, N)
            assert now >= last, (T, r, K, N)
            last = now


def _rows():
    T, k, H, R = 4, 2, 16, 8
    return T, k, H, dict(x=torch.zeros(T, H), rows=torch.zeros(R, H), inv=torch.zeros(T * k, dtype=torch.int32), w=torch.zeros(T, k),
                         y=torch.zeros(T, H), add=torch.zeros(T, H), drows=torch.zeros(R, H), dw=torch.zeros(T, k))


def test_refusals_of_the_binding_rows():
    T, k, H, good = _rows()

    def sort(**kw):
        t = {**good, **kw}
        damoe.sort_rows(t["x"], T, k, H, t["inv"], t["rows"], w=t["w"], stream=0)

    def combine(**kw):
        t = {**good, **kw}
        damoe.combine_rows(t["rows"], T, k, H, t["inv"], t["y"], w=t["w"], add=t["add"], stream=0)

    def grad(**kw):
        t = {**good, **kw}
        damoe.combine_rows_grad(t["x"], t["rows"], T, k, H, t["inv"], w=t["w"], drows=t["drows"], dw=t["dw"], stream=0)

    for call in (sort, combine, grad):
        with pytest.raises(ValueError, match="current device"):
            call()
        for inv in (good["inv"].long(), good["inv"][:-1], torch.zeros(2 * T * k, dtype=torch.int32)[::2]):
            with pytest.raises(ValueError, match="^inv_perm:"):
                call(inv=inv)
        for w in (good["w"].double(), good["w"][:-1], torch.zeros(1, 1).expand(T, k)):
            with pytest.raises(ValueError, match="^w:"):
                call(w=w)
        for rows in (good["rows"][:, :-1], good["rows"].view(-1), good["rows"].bfloat16(), torch.zeros(H, 8).t()):
            with pytest.raises(ValueError, match="^(rows|y|add|drows):"):
                call(rows=rows)
    for call, names in ((sort, ["x"]), (combine, ["y", "add"]), (grad, ["drows"])):
        for name in names:
            for bad in (good[name][:, :-1], good[name][:-1], good[name].half()):
                with pytest.raises((ValueError, damoe.DamoeError)):
                    call(**{name: bad})
    with pytest.raises(ValueError, match="dw needs"):
        grad(rows=None)
    for dw in (good["dw"].double(), good["dw"][:-1]):
        with pytest.raises(ValueError, match="^dw:"):
            grad(dw=dw)
    with pytest.raises(damoe.DamoeError, match="unsupported"):
        sort(**{n: good[n].half() for n in ("x", "rows")})


def test_refusals_of_the_binding_adapters():
    T, L, r, K, N = 5, 3, 4, 24, 16
    i32 = dict(dtype=torch.int32)
    good = dict(x=torch.zeros(T, K), a=torch.zeros(L, r, K), b=torch.zeros(L, N, r), offsets=torch.zeros(L + 1, **i32),
                y=torch.zeros(T, N), ws=torch.zeros(1 << 16, dtype=torch.uint8), perm=torch.zeros(T, **i32), scale=torch.ones(L),
                add=torch.zeros(T, N), u=torch.zeros(T, r), dy=torch.zeros(T, N), dx=torch.zeros(T, K), addx=torch.zeros(T, K),
                da=torch.zeros(L, r, K), db=torch.zeros(L, N, r))

    def forward(**kw):
        t = {**good, **kw}
        damoe.adapters(t["x"], T, t["a"], t["b"], t["offsets"], t["y"], t["ws"], perm=t["perm"], scale=t["scale"], add=t["add"],
                       u=t["u"], stream=0)

    def backward(**kw):
        t = {**good, **kw}
        damoe.adapters_grad(t["x"], t["dy"], t["u"], T, t["a"], t["b"], t["offsets"], t["da"], t["db"], t["ws"], perm=t["perm"],
                            scale=t["scale"], add=t["addx"], dx=t["dx"], stream=0)

    both = [("x", ("x",)), ("a", ("a", "b")), ("b", ("a", "b")), ("perm", ("perm",)), ("scale", ("scale",)), ("u", ("u",)),
            ("offsets", ("offsets",)), ("ws", ("ws",))]
    for call, names in ((forward, both + [("y", ("y", "add")), ("add", ("add",))]),
                        (backward, both + [("dy", ("dy",)), ("dx", ("dx",)), ("addx", ("add",)), ("da", ("da",)), ("db", ("db",))])):
        with pytest.raises(ValueError, match="current device"):
            call()
        for name, said in names:
            t = good[name]
            gaps = torch.zeros(2 * t.numel(), dtype=t.dtype)[::2] if t.dim() == 1 else t.new_zeros(*t.shape[:-1], 2 * t.shape[-1])[..., ::2]
            bad = [gaps]
            if name != "ws":
                bad.append(t[..., :-1])
            if name == "offsets":
                bad += [torch.zeros(L + 2, **i32), t.long()]
            if name in ("a", "b"):
                bad += [t.double(), t.transpose(1, 2), t[:-1]]
            for v in bad:
                with pytest.raises(ValueError, match="^(" + "|".join(said) + ")[:,]"):
                    call(**{name: v})
    with pytest.raises(damoe.DamoeError, match="unsupported"):
        forward(x=good["x"].half())


@pytest.mark.skipif(torch.cuda.is_available(), reason="the addresses are made up: a launch has to fail")
def test_a_workspace_of_the_named_size_is_enough_for_every_smaller_call():
    """Of T_max rows, for T of 0 to T_max, whatever way the call takes through its kernels."""
    rng = random.Random(1)
    sizes = [(4096, 3, 16, 7168, 4096), (1024, 1024, 64, 64, 8192), (1 << 20, 1, 1, 1, 1), (9000, 1, 128, 300, 5000), (200, 7, 33, 8, 8)]
    sizes += [(int(2 ** rng.uniform(0, 20)), rng.randint(1, 1024), rng.randint(1, 128), int(2 ** rng.uniform(0, 14)), int(2 ** rng.uniform(0, 14)))
              for _ in range(40)]
    call = damoe.lib().damoe_call_words
    for most, L, r, K, N in sizes:
        for d in (0, 1):
            common = dict(L=L, r=r, K=K, N=N, ldx=K, ldy=N, xdtype=d, ydtype=d)
            for fn, pack, good, ld, size in ((6, damoe._ADAPTERS_WORDS, ADAPTERS, dict(ld_add=N), damoe.adapters_workspace_size),
                                             (7, damoe._ADAPTERS_GRAD_WORDS, ADAPTERS_GRAD, dict(ld_add=K, ld_dx=K), damoe.adapters_grad_workspace_size)):
                room = size(most, L, r, K, N)
                for T in sorted({1, most, max(1, most // 3), min(most, 1024), min(most, 1025), min(most, 4095), min(most, 4096), min(most, 129)}):
                    words = {**good, **common, **ld, "T": T, "ws_bytes": room}
                    assert call(fn, pack(*words.values()), len(words)) not in (BAD, UNSUPPORTED, WORKSPACE), (fn, T, most, L, r, K, N)
