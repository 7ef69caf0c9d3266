"""MxLinear and quantise_layer on a side stream: whose memory their results are, and the results themselves."""
import pytest

from paper_2607_23099_amd import damoe, synth
from tests.gpu_common import log, torch_cuda

pytestmark = pytest.mark.gpu


def _owner(torch, t):
    """Handle of the stream whose pool of the caching allocator holds the tensor."""
    for seg in torch.cuda.memory_snapshot():
        if seg["address"] <= t.data_ptr() < seg["address"] + seg["total_size"]:
            return seg["stream"]
    raise AssertionError("not the allocator's memory")


@pytest.mark.parametrize("handle", [False, True], ids=["stream", "handle"])
def test_shared_expert_on_a_side_stream(handle):
    """Gate and up, then down, on a side stream that waits for the input at its start and is waited for at its end, beside
    work of the current stream that allocates and frees blocks of the same sizes."""
    torch = torch_cuda()
    from paper_2607_23099_amd.moe import MxLinear
    g = torch.Generator().manual_seed(1)
    T, H, I = 300, 1024, 512
    up = MxLinear((torch.randn((I, H), generator=g) / H ** 0.5).to(torch.bfloat16).cuda(), T)
    down = MxLinear((torch.randn((H, I), generator=g) / I ** 0.5).to(torch.bfloat16).cuda(), T)
    side = torch.cuda.Stream()
    s = side.cuda_stream if handle else side
    for T in (1, 20, 300):
        log(f"shared expert on a side stream T={T} handle={handle}")
        x = torch.randn((T, H), generator=g).to(torch.bfloat16).cuda()
        add = torch.randn((T, H), generator=g).cuda()
        want = down(up(x), add=add)
        torch.cuda.synchronize()
        outs = []
        for _ in range(10):
            side.wait_stream(torch.cuda.current_stream())
            h = up(x, stream=s)
            y = down(h, add=add, stream=s)
            assert _owner(torch, h) == _owner(torch, y) == side.cuda_stream
            del h
            for n in (I, H):  # the current stream's own work, in blocks of the same sizes
                torch.full((T, n), float("nan"), dtype=torch.bfloat16, device="cuda")
            torch.cuda.current_stream().wait_stream(side)
            outs.append(y.clone())
        torch.cuda.synchronize()
        assert all(torch.equal(o, want) for o in outs)
        assert torch.equal(down(up(x, stream=0), add=add, stream=0), want)  # the default stream, by its handle


def test_a_layer_quantised_on_a_side_stream():
    torch = torch_cuda()
    from paper_2607_23099_amd.moe import quantise_layer
    sh = synth.Shape("streams", E=2, k=1, H=256, I=128, shape_id=9, wdtype="mxfp4")
    g = torch.Generator().manual_seed(2)
    w = {n: torch.randn((sh.E,) + tuple(synth.weight_dims(sh, n)[1:]), generator=g).to(torch.bfloat16).cuda()
         for n in ("w1", "w3", "w2")}
    want = quantise_layer(sh, **w)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = quantise_layer(sh, **w, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    for n, t in got.w.items():
        assert _owner(torch, t) == side.cuda_stream
        assert torch.equal(t, want.w[n])
    assert got.layer.layout == damoe.LAYOUT_FRAG16


def test_products_captured_with_results_of_their_own():
    """A shared expert whose results the captured calls allocate, replayed among eager calls of the same objects, and calls
    without rows."""
    torch = torch_cuda()
    from paper_2607_23099_amd.moe import MxLinear
    g = torch.Generator().manual_seed(3)
    T, H, I = 40, 512, 256
    up = MxLinear((torch.randn((I, H), generator=g) / H ** 0.5).cuda(), T)
    down = MxLinear((torch.randn((H, I), generator=g) / I ** 0.5).cuda(), T)
    xs = [torch.randn((T, H), generator=g).to(torch.bfloat16).cuda() for _ in range(3)]
    want = [down(up(x)) for x in xs]
    for lin, n in ((up, I), (down, H)):
        assert lin(torch.zeros((0, lin.K), dtype=torch.bfloat16, device="cuda")).shape == (0, n)
    x = xs[0].clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = down(up(x))
    for rep in range(4):
        x.copy_(xs[rep % 3])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want[rep % 3]), rep
        assert torch.equal(down(up(xs[0])), want[0])
        torch.cuda.synchronize()
