"""An expert layer with an adapter for each expert, forward and backward, of the library's calls alone: routing, rows to their
experts, adapters, rows back, and the gradient down to the router's logits; and requests with adapters of their own."""
import numpy as np
import pytest

from paper_2607_23099_amd import damoe
from tests import router_loss_ref, rows_ref as ref
from tests.gpu_common import log, torch_cuda
from tests.test_gpu_router_loss import REL
from tests.test_gpu_rows import close

pytestmark = pytest.mark.gpu


class Routed:
    def __init__(self, torch, ids, T, k, E):
        i32 = dict(dtype=torch.int32, device="cuda")
        self.counts, self.offsets = torch.empty(E, **i32), torch.empty(E + 1, **i32)
        self.perm, self.inv = torch.empty(T * k, **i32), torch.empty(T * k, **i32)
        nd, bucket = torch.zeros(2, dtype=torch.int64, device="cuda"), torch.zeros(1, **i32)
        ws = torch.zeros(damoe.workspace_layout(E, k, 128, 128, T)["h"], dtype=torch.uint8, device="cuda")
        damoe.route_histogram(ids, T, k, E, self.counts, self.offsets, self.perm, self.inv, nd, bucket, ws)


def host(t):
    return t.double().cpu().numpy()


class Layer:
    def __init__(self, torch, T, k, E, r, H, N, dtype, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        d = torch.bfloat16 if dtype == "bf16" else torch.float32
        randn = lambda *s, t=torch.float32: torch.randn(s, generator=g, device="cuda").to(t)
        self.sizes, self.dtype = (T, k, E, r, H, N), dtype
        self.logits = randn(T, E)
        top = torch.topk(self.logits, k, dim=1)
        self.ids = top.indices.to(torch.int32)
        self.ids[torch.rand(T, k, generator=g, device="cuda") < 0.1] = -1  # dropped slots
        self.w = torch.softmax(top.values, dim=1).contiguous()
        self.x, self.shared, self.dy = randn(T, H, t=d), randn(T, N, t=d), randn(T, N, t=d)
        self.a, self.b = randn(E, r, H) * H ** -0.5, randn(E, N, r) * r ** -0.5
        self.scale = torch.rand(E, generator=g, device="cuda") + 0.5
        R = T * k
        self.rows, self.out = (torch.zeros(R, n, dtype=d, device="cuda") for n in (H, N))
        self.y, self.dx = torch.empty_like(self.shared), torch.empty_like(self.x)
        self.drows, self.dout = torch.zeros_like(self.rows), torch.zeros_like(self.out)
        self.u, self.dw = torch.zeros(R, r, device="cuda"), torch.empty(T, k, device="cuda")
        self.da, self.db, self.dlogits = torch.empty_like(self.a), torch.empty_like(self.b), torch.empty_like(self.logits)
        self.tokens = torch.tensor([T, 1, T], dtype=torch.int32, device="cuda")
        self.ws = torch.empty(damoe.adapters_workspace_size(R, E, r, H, N), dtype=torch.uint8, device="cuda")
        self.gws = torch.empty(damoe.adapters_grad_workspace_size(R, E, r, H, N), dtype=torch.uint8, device="cuda")
        self.loss, self.lws = torch.empty(3, device="cuda"), torch.zeros(damoe.router_loss_workspace_size(T, E), dtype=torch.uint8, device="cuda")

    def route(self, torch):
        T, k, E, _, _, _ = self.sizes
        self.p = Routed(torch, self.ids, T, k, E)

    def forward(self):
        T, k, E, r, H, N = self.sizes
        damoe.sort_rows(self.x, T, k, H, self.p.inv, self.rows)
        damoe.adapters(self.rows, T * k, self.a, self.b, self.p.offsets, self.out, self.ws, scale=self.scale, u=self.u)
        damoe.combine_rows(self.out, T, k, N, self.p.inv, self.y, w=self.w, add=self.shared)

    def backward(self):
        T, k, E, r, H, N = self.sizes
        damoe.combine_rows_grad(self.dy, self.out, T, k, N, self.p.inv, w=self.w, drows=self.dout, dw=self.dw)
        damoe.adapters_grad(self.rows, self.dout, self.u, T * k, self.a, self.b, self.p.offsets, self.da, self.db, self.gws,
                            scale=self.scale, dx=self.drows)
        damoe.combine_rows(self.drows, T, k, H, self.p.inv, self.dx)
        damoe.router_loss(self.logits, self.ids, T, E, k, self.loss, self.p.counts, self.tokens, self.lws)
        damoe.router_loss_grad(self.logits, self.ids, T, E, k, self.p.counts, self.tokens, self.dlogits, w=self.w, dw=self.dw)

    def results(self):
        return [t.clone() for t in (self.y, self.u, self.dw, self.dx, self.da, self.db, self.dlogits)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,k,E,r,H,N", [(1, 2, 8, 4, 64, 48), (70, 4, 16, 8, 264, 130), (700, 8, 40, 16, 128, 256)])
def test_experts_with_adapters(T, k, E, r, H, N, dtype):
    """Each step against float64 on what the step before it left, so that every bound is one operator's."""
    torch = torch_cuda()
    log(f"T={T} k={k} E={E} r={r} H={H} N={N} {dtype}")
    m = Layer(torch, T, k, E, r, H, N, dtype)
    m.route(torch)
    m.forward(), m.backward()
    inv, off, w, scale, R = m.p.inv.cpu().numpy(), m.p.offsets.cpu().numpy(), host(m.w), host(m.scale), T * k
    a, b = host(m.a), host(m.b)
    close(m.rows, *ref.sort_rows(host(m.x), inv, k, R, np.zeros((R, H))), None, "rows")
    y, ey, u, eu = ref.adapters(host(m.rows), a, b, off, None, scale)
    # fp32 weights of bf16 rows: three products a weight.
    close(m.out, y, 3 * ey, dtype, "out")
    close(m.u, u, 3 * eu, "f32", "u")
    close(m.y, *ref.combine_rows(host(m.out), inv, T, k, w, host(m.shared)), dtype, "y")
    d, ed, dw, ew = ref.combine_rows_grad(host(m.dy), host(m.out), inv, k, np.zeros((R, N)), w)
    close(m.dout, d, ed, dtype, "dout")
    close(m.dw, dw, ew, "f32", "dw")
    dx, ex, da, ea, db, eb = ref.adapters_grad(host(m.rows), host(m.dout), host(m.u), a, b, off, None, scale)
    close(m.drows, dx, 3 * ex, dtype, "drows")
    close(m.da, da, 3 * ea, "f32", "da")
    close(m.db, db, eb, "f32", "db")
    close(m.dx, *ref.combine_rows(host(m.drows), inv, T, k), dtype, "dx")
    ids = m.ids.cpu().numpy()
    want, mag = router_loss_ref.grad(host(m.logits), ids, k, None, None, 0, 0.0, 0.0, m.p.counts.cpu().numpy()[None], 1.0, w, host(m.dw))
    close(m.dlogits, want, 2 * REL * mag + 1e-30, "f32", "dlogits")


def test_a_step_in_a_graph():
    """Forward and backward captured once and replayed on other inputs, with eager steps of another layer between."""
    torch = torch_cuda()
    m, other = (Layer(torch, 300, 4, 16, 8, 136, 264, "bf16", seed=s) for s in (1, 2))
    for l in (m, other):
        l.route(torch)
        l.forward(), l.backward()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        m.forward(), m.backward()
    for i in range(4):
        m.x.mul_(-0.5), m.dy.mul_(2), m.w.mul_(0.75)
        g.replay()
        other.forward(), other.backward()
        torch.cuda.synchronize()
        got = m.results()
        m.forward(), m.backward()
        assert all(torch.equal(p, q) for p, q in zip(got, m.results())), i


@pytest.mark.parametrize("T", [1, 61, 900])
def test_requests_with_adapters_beside_a_shared_product(T):
    """The rows' adapters as ids of a routing with one slot a token; those without keep the shared product."""
    torch = torch_cuda()
    L, r, K, N = 12, 16, 256, 320
    log(f"requests T={T}")
    g = torch.Generator(device="cuda").manual_seed(T)
    ids = torch.randint(-1, L, (T,), generator=g, device="cuda", dtype=torch.int32)
    p = Routed(torch, ids, T, 1, L)
    x, y = (torch.randn(T, n, generator=g, device="cuda").bfloat16() for n in (K, N))
    a, b = (torch.randn(s, generator=g, device="cuda").bfloat16() for s in ((L, r, K), (L, N, r)))
    before = y.clone()
    ws = torch.empty(damoe.adapters_workspace_size(T, L, r, K, N), dtype=torch.uint8, device="cuda")
    damoe.adapters(x, T, a, b, p.offsets, y, ws, perm=p.perm, add=y)
    want, err, _, _ = ref.adapters(host(x), host(a), host(b), p.offsets.cpu().numpy(), p.perm.cpu().numpy(), None, host(before), host(before))
    close(y, want, err, "bf16", "y")
    bare = ids < 0
    assert torch.equal(y[bare], before[bare])
