"""MXFP4 quantisation, its layouts, and the dense product, against float64 (tests/fp4_ref.py)."""
import numpy as np
import pytest

from paper_2607_23099_amd import damoe, synth
from tests import fp4_ref
from tests.gpu_common import TOL, bf16_rows, log, oracle_rows, row_err, torch_cuda

pytestmark = pytest.mark.gpu

LAYOUTS = {"rowmajor": damoe.LAYOUT_ROWMAJOR, "frag16": damoe.LAYOUT_FRAG16, "tile32": damoe.LAYOUT_TILE32}
FORM = {"rowmajor": lambda c, s: fp4_ref.rowmajor(c, s)[0].reshape(-1), "frag16": fp4_ref.frag16,
        "tile32": fp4_ref.tile32}


def _bf16(torch, a):
    return torch.from_numpy(np.ascontiguousarray(a, np.float32)).to(torch.bfloat16)


def _dev(torch, a, dtype):
    """Host float values on the device in `dtype`, and what they are exactly in float64."""
    t = torch.from_numpy(np.ascontiguousarray(a, np.float32))
    t = t.to(torch.bfloat16) if dtype == "bf16" else t
    return t.cuda(), t.to(torch.float64).numpy()


def _quantise(torch, x, rows, cols, layout, **kw):
    codes = torch.full((damoe.mxfp4_bytes(rows, cols, LAYOUTS[layout]) + 64,), 0xA5, dtype=torch.uint8, device="cuda")
    scales = torch.full((rows * cols // 32 + 64,), 0xA5, dtype=torch.uint8, device="cuda") if layout == "rowmajor" else None
    damoe.mxfp4_quantise(x, rows, cols, codes, scales, LAYOUTS[layout], **kw)
    torch.cuda.synchronize()
    assert (codes[-64:] == 0xA5).all() and (scales is None or (scales[-64:] == 0xA5).all())
    return codes[:-64], None if scales is None else scales[:-64]


SHAPES = [(1, 32, "rowmajor"), (5, 96, "rowmajor"), (300, 7168, "rowmajor"), (16, 128, "frag16"), (48, 384, "frag16"),
          (1, 32, "tile32"), (31, 256, "tile32"), (33, 288, "tile32"), (70, 2048, "tile32")]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols,layout", SHAPES)
def test_quantise_bit_for_bit(rows, cols, layout, dtype):
    torch = torch_cuda()
    log(f"quantise {rows}x{cols} {layout} {dtype}")
    x, exact = _dev(torch, fp4_ref.awkward(np.random.default_rng([rows, cols]), rows, cols), dtype)
    code, scale = fp4_ref.quantise(exact)
    codes, scales = _quantise(torch, x, rows, cols, layout)
    assert np.array_equal(codes.cpu().numpy(), FORM[layout](code, scale))
    if scales is not None:
        assert np.array_equal(scales.cpu().numpy(), scale.reshape(-1))
    # And back: the values that codes and scales stand for.
    want = fp4_ref.values(code, scale)
    for out_t in (torch.bfloat16, torch.float32):
        out = torch.full((rows, cols), 7.0, dtype=out_t, device="cuda")
        damoe.mxfp4_dequantise(codes, scales, rows, cols, out, LAYOUTS[layout])
        np.testing.assert_array_equal(out.double().cpu().numpy(), want)


@pytest.mark.parametrize("layout", sorted(LAYOUTS))
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strided_and_unaligned_rows(layout, dtype):
    torch = torch_cuda()
    rows, cols = 48, 384
    v = fp4_ref.awkward(np.random.default_rng(3), rows, cols)
    for ld, shift in [(cols + 8, 0), (cols + 3, 0), (cols, 1), (cols + 1, 3)]:
        buf = np.full(rows * ld + 8, np.nan)
        for r in range(rows):
            buf[shift + r * ld: shift + r * ld + cols] = v[r]
        x, _ = _dev(torch, buf, dtype)
        exact = _dev(torch, v, dtype)[1]
        code, scale = fp4_ref.quantise(exact)
        codes, scales = _quantise(torch, x[shift:], rows, cols, layout, ldx=ld)
        assert np.array_equal(codes.cpu().numpy(), FORM[layout](code, scale)), (ld, shift)
        # The way back leaves what lies between the rows alone.
        out = torch.full((rows * ld + 8,), 7.0, dtype=x.dtype, device="cuda")
        damoe.mxfp4_dequantise(codes, scales, rows, cols, out[shift:], LAYOUTS[layout], ldx=ld)
        got, want = out.double().cpu().numpy(), np.full(rows * ld + 8, 7.0)
        for r in range(rows):
            want[shift + r * ld: shift + r * ld + cols] = fp4_ref.values(code, scale)[r]
        np.testing.assert_array_equal(got, want)


def test_many_short_strided_rows():
    torch = torch_cuda()
    rows, cols, ld = 70001, 32, 40
    v = np.random.default_rng(8).standard_normal((rows, cols))
    x = torch.full((rows, ld), float("nan"), dtype=torch.bfloat16, device="cuda")
    x[:, :cols] = _bf16(torch, v).cuda()
    code, scale = fp4_ref.quantise(x[:, :cols].double().cpu().numpy())
    codes, scales = _quantise(torch, x, rows, cols, "rowmajor")
    assert np.array_equal(codes.cpu().numpy(), fp4_ref.rowmajor(code, scale)[0].reshape(-1))
    assert np.array_equal(scales.cpu().numpy(), scale.reshape(-1))
    out = torch.full((rows, ld), 7.0, dtype=torch.float32, device="cuda")
    damoe.mxfp4_dequantise(codes, scales, rows, cols, out, damoe.LAYOUT_ROWMAJOR)
    np.testing.assert_array_equal(out[:, :cols].double().cpu().numpy(), fp4_ref.values(code, scale))
    assert (out[:, cols:] == 7.0).all()


@pytest.mark.parametrize("layout", sorted(LAYOUTS))
def test_every_code_under_every_scale(layout):
    torch = torch_cuda()
    rows, cols = 256, 128
    code = np.tile(np.arange(16, dtype=np.uint8), rows * cols // 16).reshape(rows, cols)
    scale = np.repeat(np.arange(256, dtype=np.uint8)[:, None], cols // 32, axis=1)
    codes = torch.from_numpy(FORM[layout](code, scale)).cuda()
    scales = torch.from_numpy(scale.reshape(-1).copy()).cuda() if layout == "rowmajor" else None
    want = fp4_ref.values(code, scale)
    with np.errstate(over="ignore"):
        want = want.astype(np.float32)  # 6 x 2^126 and above are infinities of both types
    for out_t in (torch.float32, torch.bfloat16):
        out = torch.zeros((rows, cols), dtype=out_t, device="cuda")
        damoe.mxfp4_dequantise(codes, scales, rows, cols, out, LAYOUTS[layout])
        np.testing.assert_array_equal(out.float().cpu().numpy(), want)


def test_quantise_agrees_with_the_generator_and_the_packer():
    """The interchange layout is the one that the generator writes and damoe_pack_weights reads."""
    torch = torch_cuda()
    rows, cols, E = 512, 512, 2
    w = np.random.default_rng(5).standard_normal((E * rows, cols)).astype(np.float32)
    x = _bf16(torch, w)
    qh, sh = synth.mxfp4_quantize(x.float().numpy())
    x = x.cuda()
    codes, scales = _quantise(torch, x, E * rows, cols, "rowmajor")
    assert np.array_equal(codes.cpu().numpy(), np.asarray(qh).reshape(-1))
    assert np.array_equal(scales.cpu().numpy(), np.asarray(sh).reshape(-1))
    layer = damoe.make_layer(E, 1, cols, rows, damoe.W_MXFP4, codes, codes, codes, scales, scales, scales)
    dst = [torch.zeros(E * rows * cols * 17 // 32, dtype=torch.uint8, device="cuda") for _ in range(3)]
    damoe.pack_weights(layer, *dst)
    packed, _ = _quantise(torch, x, E * rows, cols, "frag16")
    assert torch.equal(packed, dst[0])


@pytest.mark.parametrize("rows,cols", [(1, 32), (33, 288), (64, 512), (100, 4096)])
def test_pack_equals_quantise(rows, cols):
    torch = torch_cuda()
    x, _ = _dev(torch, fp4_ref.awkward(np.random.default_rng([rows, 9]), rows, cols), "f32")
    codes, scales = _quantise(torch, x, rows, cols, "rowmajor")
    tiles = torch.full((damoe.mxfp4_bytes(rows, cols) + 64,), 0xA5, dtype=torch.uint8, device="cuda")
    damoe.mxfp4_pack(codes, scales, rows, cols, tiles)
    want, _ = _quantise(torch, x, rows, cols, "tile32")
    assert torch.equal(tiles[:-64], want) and (tiles[-64:] == 0xA5).all()


@pytest.mark.parametrize("layout", sorted(LAYOUTS))
def test_more_values_than_32_bits(layout):
    """The last rows of a matrix of 4.3e9 values, past every 32-bit offset."""
    torch = torch_cuda()
    cols, rows = 32768, (1 << 17) + 48
    log(f"quantise {rows}x{cols} {layout}")
    x = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda")
    x[:-48] = torch.randn((1, cols), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda()
    x[-48:] = torch.randn((48, cols), generator=torch.Generator().manual_seed(2)).to(torch.bfloat16).cuda()
    codes, scales = _quantise(torch, x, rows, cols, layout)
    want, want_s = _quantise(torch, x[-48:].contiguous(), 48, cols, layout)
    per = {"rowmajor": 48 * cols // 2, "frag16": 48 * cols // 32 * 17, "tile32": 2 * cols // 256 * 4352}[layout]
    # rows - 48 is a multiple of 32: the last rows' tiles are whole ones and as in the small matrix.
    assert torch.equal(codes[-per:], want[-per:])
    assert scales is None or torch.equal(scales[-48 * cols // 32:], want_s)
    out = torch.empty((48, cols), dtype=torch.bfloat16, device="cuda")
    damoe.mxfp4_dequantise(want, want_s, 48, cols, out, LAYOUTS[layout])
    damoe.mxfp4_dequantise(codes, scales, rows, cols, x, LAYOUTS[layout])
    assert torch.equal(x[-48:], out)


# ---------------------------------------------------------------- the product

class Linear:
    """A product's inputs on the device and its exact result."""

    def __init__(self, torch, T, N, K, seed=0, x_dtype="bf16", spread=6):
        rng = np.random.default_rng([T, N, K, seed])
        def rows(n):
            return rng.standard_normal((n, K)) * np.exp2(rng.integers(-spread, spread + 1, (n, K // 32))).repeat(32, axis=1)
        self.T, self.N, self.K = T, N, K
        self.x, xe = _dev(torch, rows(T), x_dtype)
        w, we = _dev(torch, rows(N), "bf16")
        self.tiles, _ = _quantise(torch, w, N, K, "tile32")
        self.xq, self.wq = fp4_ref.values(*fp4_ref.quantise(xe)), fp4_ref.values(*fp4_ref.quantise(we))
        self.y = self.xq @ self.wq.T
        self.mag = np.abs(self.xq) @ np.abs(self.wq).T
        self.ws = torch.zeros(damoe.mxfp4_linear_workspace_size(T, N, K), dtype=torch.uint8, device="cuda")

    def tol(self, out_dtype, want):
        """Exact products; fewer than K sums in fp32, each off by at most 2^-24 of the terms' magnitude, then one
        rounding of the result to its type."""
        t = (self.K + 2) * 2.0 ** -24 * self.mag + 2.0 ** -24 * np.abs(want)
        return t + (2.0 ** -8 * (np.abs(want) + t) if out_dtype == "bf16" else 0.0)


def _check(got, want, tol):
    got = got.double().cpu().numpy()
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4].tolist(), got[bad][:4], want[bad][:4])


TNK = [(1, 1, 32), (1, 7168, 2048), (2, 100, 96), (5, 33, 256), (16, 512, 7168), (31, 31, 288), (32, 256, 512),
       (33, 1000, 544), (37, 4096, 1024), (64, 64, 4096), (65, 257, 768), (100, 130, 2048), (129, 96, 256),
       (200, 2048, 1024), (255, 384, 1280), (300, 7168, 512), (513, 300, 2304), (1000, 513, 320), (2049, 1025, 1056),
       # every kernel of many tokens, with whole and with odd rows of y
       (129, 4100, 544), (300, 4104, 800), (513, 7001, 288), (700, 4096, 1056), (1100, 5000, 800), (600, 7169, 320),
       (2300, 4001, 1568), (2300, 4000, 1568), (600, 7168, 320), (1500, 5001, 1056), (3000, 3400, 1056),
       (4100, 2001, 8224), (600, 7168, 1568), (2300, 7168, 544), (3000, 5001, 1056),
       (2300, 7168, 3200), (2300, 7001, 3200), (1100, 7168, 544)]


@pytest.mark.parametrize("T,N,K", TNK)
def test_linear(T, N, K):
    torch = torch_cuda()
    for xd, yd in [("bf16", "bf16"), ("f32", "f32")]:
        log(f"linear T={T} N={N} K={K} {xd} -> {yd}")
        p = Linear(torch, T, N, K, x_dtype=xd)
        y = torch.full((T, N), float("nan"), dtype=torch.bfloat16 if yd == "bf16" else torch.float32, device="cuda")
        p.ws.fill_(0xFF)  # nothing is kept in the workspace
        damoe.mxfp4_linear(p.x, T, K, p.tiles, N, y, p.ws)
        _check(y, p.y, p.tol(yd, p.y))
        again = torch.zeros_like(y)
        damoe.mxfp4_linear(p.x, T, K, p.tiles, N, again, p.ws)
        assert torch.equal(again, y)  # a fixed order of sums


@pytest.mark.parametrize("T,N,K", [(3, 100, 320), (40, 77, 2048), (300, 301, 512), (150, 4096, 544), (513, 7001, 288),
                                   (600, 7168, 320), (2300, 4001, 1568), (2300, 4008, 1568), (1500, 5001, 1056),
                                   (3000, 3400, 1056), (4100, 2001, 8224), (600, 7168, 1568), (2300, 7168, 544),
                                   (3000, 5001, 1056), (2300, 7168, 3200), (2300, 7001, 3200), (1100, 7168, 544)])
@pytest.mark.parametrize("yd", ["bf16", "f32"])
def test_linear_add_and_strides(T, N, K, yd):
    torch = torch_cuda()
    log(f"linear with add T={T} N={N} K={K} {yd}")
    dt = torch.bfloat16 if yd == "bf16" else torch.float32
    p = Linear(torch, T, N, K, seed=1)
    # Rows of y and add that start at 16 bytes take wide accesses where N allows it.
    ldx, ldy, lda = (K + 5, N + 3, N + 1) if N % 8 else (K + 5, N + 16, N + 8)
    x = torch.full((T, ldx), float("nan"), dtype=torch.bfloat16, device="cuda")
    x[:, :K] = p.x
    add = torch.randn(T, lda, generator=torch.Generator().manual_seed(2)).to(dt).cuda()
    y = torch.full((T, ldy), 7.0, dtype=dt, device="cuda")
    damoe.mxfp4_linear(x, T, K, p.tiles, N, y, p.ws, add=add)
    want = p.y + add[:, :N].double().cpu().numpy()
    tol = p.tol(yd, want) + 2.0 ** -23 * np.abs(want)  # the sum with `add`, once more in fp32
    _check(y[:, :N], want, tol)
    assert (y[:, N:] == 7.0).all()
    # In place: add and y the same.
    y2 = add.clone()
    damoe.mxfp4_linear(x, T, K, p.tiles, N, y2, p.ws, add=y2)
    assert torch.equal(y2[:, :N], y[:, :N]) and torch.equal(y2[:, N:], add[:, N:])


@pytest.mark.parametrize("T,N,K", [(3, 64, 512), (70, 100, 512), (300, 300, 288)])
def test_linear_nan_blocks(T, N, K):
    """A block with an infinity or NaN makes its row of x, or its column of w, NaN, and nothing else."""
    torch = torch_cuda()
    rng = np.random.default_rng(T)
    xv, wv = rng.standard_normal((T, K)), rng.standard_normal((N, K))
    xv[T // 2, K - 1] = np.inf
    wv[N - 1, 0] = np.nan
    x, xe = _dev(torch, xv, "bf16")
    w, we = _dev(torch, wv, "bf16")
    tiles, _ = _quantise(torch, w, N, K, "tile32")
    ws = torch.zeros(damoe.mxfp4_linear_workspace_size(T, N, K), dtype=torch.uint8, device="cuda")
    y = torch.zeros((T, N), dtype=torch.float32, device="cuda")
    damoe.mxfp4_linear(x, T, K, tiles, N, y, ws)
    want = np.zeros((T, N), bool)
    want[T // 2, :] = True
    want[:, N - 1] = True
    assert np.array_equal(torch.isnan(y).cpu().numpy(), want)
    xq, wq = fp4_ref.values(*fp4_ref.quantise(xe)), fp4_ref.values(*fp4_ref.quantise(we))
    ref, mag = xq @ wq.T, np.abs(xq) @ np.abs(wq).T
    got = y.double().cpu().numpy()
    assert (np.abs(got - ref)[~want] <= ((K + 2) * 2.0 ** -24 * mag)[~want]).all()


@pytest.mark.parametrize("T", [1, 40, 300])
def test_linear_streams_and_graphs(T):
    """A call on another stream, and two captured graphs with a workspace each, replayed among eager work."""
    torch = torch_cuda()
    N, K = 512, 1024
    p = [Linear(torch, T, N, K, seed=s) for s in (3, 4)]

    def call(q, x):
        y = torch.zeros((T, N), dtype=torch.bfloat16, device="cuda")
        damoe.mxfp4_linear(x, T, K, q.tiles, N, y, q.ws)
        return y

    eager, other = [call(q, q.x) for q in p], [call(q, q.x.flip(0)) for q in p]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    y = torch.zeros((T, N), dtype=torch.bfloat16, device="cuda")
    side.wait_stream(torch.cuda.current_stream())
    damoe.mxfp4_linear(p[0].x, T, K, p[0].tiles, N, y, p[0].ws, stream=side)
    side.synchronize()
    assert torch.equal(y, eager[0])
    graphs, outs, xs = [], [], []
    for q in p:
        xs.append(q.x.clone())
        outs.append(torch.zeros((T, N), dtype=torch.bfloat16, device="cuda"))
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g, stream=side):
            damoe.mxfp4_linear(xs[-1], T, K, q.tiles, N, outs[-1], q.ws)
        graphs.append(g)
    for rep in range(3):
        for i in (0, 1):
            xs[i].copy_(p[i].x if rep != 1 else p[i].x.flip(0))
            outs[i].fill_(float("nan"))
        torch.cuda.synchronize()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for i in (0, 1):
            assert torch.equal(outs[i], eager[i] if rep != 1 else other[i]), (rep, i)


def test_linear_results_past_32_bits():
    torch = torch_cuda()
    T, N, K = 1 << 20, 1100, 32
    log(f"linear T={T} N={N} K={K}")
    p = Linear(torch, 64, N, K, seed=6)
    x = p.x.repeat(T // 64, 1)
    ws = torch.empty(damoe.mxfp4_linear_workspace_size(T, N, K), dtype=torch.uint8, device="cuda")
    small = torch.empty((64, N), dtype=torch.float32, device="cuda")
    damoe.mxfp4_linear(p.x, 64, K, p.tiles, N, small, p.ws)
    _check(small, p.y, p.tol("f32", p.y))
    for n in (N, 1097):  # rows of y at 16 bytes, and any
        y = torch.full((T, n), float("nan"), dtype=torch.float32, device="cuda")
        damoe.mxfp4_linear(x, T, K, p.tiles, n, y, ws)
        assert torch.isfinite(y[::4097]).all()
        # K = 32 is one product of one block: no sums whose order the kernels could differ in.
        for t0 in (0, T // 2, T - 64):
            _check(y[t0: t0 + 64], p.y[:, :n], p.tol("f32", p.y)[:, :n])
        del y


def test_linear_add_gives_the_same_bits_each_time():
    """Results in fp32 with rows added, many calls: stores whose data is overwritten too early differ now and then."""
    torch = torch_cuda()
    for T, N, K in [(600, 7168, 320), (1100, 7168, 544), (2300, 7168, 1056)]:
        log(f"linear with add, again and again, T={T} N={N} K={K}")
        p = Linear(torch, T, N, K, seed=8)
        add = torch.randn(T, N, device="cuda")
        want = p.y + add.double().cpu().numpy()
        y = torch.zeros((T, N), device="cuda")
        damoe.mxfp4_linear(p.x, T, K, p.tiles, N, y, p.ws, add=add)
        _check(y, want, p.tol("f32", want) + 2.0 ** -23 * np.abs(want))
        for _ in range(30):
            again = torch.zeros_like(y)
            damoe.mxfp4_linear(p.x, T, K, p.tiles, N, again, p.ws, add=add)
            assert torch.equal(again, y)


def test_two_products_at_once():
    """Two streams, a workspace each, many calls in flight."""
    torch = torch_cuda()
    ps = [Linear(torch, T, 512, 1024, seed=7) for T in (8, 200)]
    want, ys = [], []
    for p in ps:
        y = torch.zeros((p.T, 512), dtype=torch.float32, device="cuda")
        damoe.mxfp4_linear(p.x, p.T, 1024, p.tiles, 512, y, p.ws)
        want.append(y)
        ys.append([torch.zeros_like(y) for _ in range(20)])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for i in range(20):
        for p, s, y in zip(ps, streams, ys):
            damoe.mxfp4_linear(p.x, p.T, 1024, p.tiles, 512, y[i], p.ws, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(y, w) for w, all_y in zip(want, ys) for y in all_y)


def test_quantised_layer_with_a_shared_expert():
    """The operators as they are used: an expert layer's weights quantised from bf16 straight into the packed
    layout and run, and a dense product added to its output."""
    torch = torch_cuda()
    from paper_2607_23099_amd.moe import MxLinear, Path, quantise_layer
    sh = synth.Shape("quantised", E=4, k=2, H=512, I=512, shape_id=9, wdtype="mxfp4")
    T = 24
    src = {}
    for name in ("w1", "w3", "w2"):
        tid, r, c = synth.weight_dims(sh, name)
        t = torch.empty((sh.E, r, c), dtype=torch.bfloat16, device="cuda")
        synth.fill_bf16_device(t.data_ptr(), t.numel(), seed=sh.weight_seed, tensor=tid, slab_elems=r * c,
                               sigma=sh.w_sigma, stream=torch.cuda.current_stream().cuda_stream)
        src[name] = t
    dl = quantise_layer(sh, **src)
    path = Path(dl, T)
    r = synth.routing(sh.E, sh.k, T, 1.0, [1])
    path.set_routing(r)
    path.fill_x(T, 3)
    path.route(T)
    path.fused(T, force_variant=0)
    y = path.y[:T].clone()
    ref = oracle_rows(sh, r, 3, np.arange(T))  # the same generator's weights, quantised on the host
    assert row_err(bf16_rows(y, np.arange(T)), ref) <= TOL["bf16"]

    dense = torch.randn((sh.H, sh.H), generator=torch.Generator().manual_seed(4)).to(torch.bfloat16).cuda()
    lin = MxLinear(dense, T_max=T)
    out = lin(path.x[:T], add=y)
    xq = fp4_ref.values(*fp4_ref.quantise(path.x[:T].double().cpu().numpy()))
    wq = fp4_ref.values(*fp4_ref.quantise(dense.double().cpu().numpy()))
    want = xq @ wq.T + y.double().cpu().numpy()
    mag = np.abs(xq) @ np.abs(wq).T
    _check(out, want, (sh.H + 4) * 2.0 ** -24 * (mag + np.abs(want)) + 2.0 ** -8 * np.abs(want))
