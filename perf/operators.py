"""The operators around the expert layer that are measured: MXFP4 quantisation, the MXFP4 product, the
router's loss and its gradient.

* ``quantise``: rows of bf16 or fp32 to MXFP4 (e2m1 codes, one power-of-two scale per 32 values) in one of
  the library's layouts, and back to the bf16 values that the codes stand for.
* ``linear``: y = Q(x) W^T of MXFP4 weights and activations that are quantised in the call.
* ``loss``: balance loss per sequence, z-loss, per-expert counts and mean probabilities of a batch of
  routed tokens.
* ``grad``: gradient of that loss and of the gates with respect to the router's logits.

The plain forms are elementary torch operations in 32 bits.  ``own`` runs the library's calls instead.
Sizes are those of a DeepSeek-V3-shaped (256 experts) and a Kimi-K2-shaped (384 experts) layer, hidden size
7168, expert size 2048, and generic ones.
"""
from __future__ import annotations

from types import SimpleNamespace

import torch

own = False

DEVICE = "cuda"
LAYOUTS = {"rowmajor": 0, "frag16": 1, "tile32": 2}
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
ALPHA, Z_COEF = 1e-2, 1e-3  # coefficients of the balance loss and of the z-loss


def _quantise(name, rows, cols, dtype, layout):
    return {"name": name, "kind": "quantise", "rows": rows, "cols": cols, "dtype": dtype, "layout": layout}


def _linear(name, T, N, K, x="bf16", y="bf16"):
    return {"name": name, "kind": "linear", "T": T, "N": N, "K": K, "x": x, "y": y}


def _router(name, kind, T, E, seqs, score, dtype="f32", dead=0):
    return {"name": name, "kind": kind, "T": T, "E": E, "k": 8, "seqs": seqs, "score": score, "dtype": dtype,
            "dead": dead}


def listed():
    return [
        # The activations of a ragged decode batch, as the product takes them.
        _quantise("quantise_tokens_t37", 37, 7168, "bf16", "tile32"),
        # One expert's W1 from an fp32 master copy, in the interchange layout.
        _quantise("quantise_expert_f32", 2048, 7168, "f32", "rowmajor"),
        # The W2 of 16 experts at once, straight into the expert layer's packed layout.
        _quantise("quantise_experts_w2", 16 * 7168, 2048, "bf16", "frag16"),
        # A dense down projection for one token: single-stream decode, launches and latencies.
        _linear("linear_down_t1", 1, 7168, 2048),
        # Gate and up projection of a shared expert for a ragged decode batch: the weight stream.
        _linear("linear_gate_up_t29", 29, 4096, 7168),
        # A short prompt: neither the weights nor the matrix cores alone.
        _linear("linear_down_t300", 300, 7168, 2048),
        # Prefill of the shared expert, and a generic square product with fp32 on both sides.
        _linear("linear_gate_up_t8192", 8192, 4096, 7168),
        _linear("linear_square_f32", 8192, 8192, 8192, x="f32", y="f32"),
        # A few tokens of one sequence: a micro-batch of a fine-tuning run.
        _router("loss_t64", "loss", 64, 256, 1, "softmax"),
        # A large packed batch of 37 ragged sequences with padding.
        _router("loss_t65536", "loss", 65536, 384, 37, "softmax"),
        # The gradient at a small batch with sigmoid scores, and at the large packed one.
        _router("grad_t509_sigmoid", "grad", 509, 256, 3, "sigmoid"),
        _router("grad_t65536", "grad", 65536, 384, 37, "softmax"),
    ]


def draw(rng):
    """One more call of the ranges above, sizes spread over their logarithm."""
    def log_int(lo, hi):
        return min(hi, max(lo, int(round(lo * (hi / lo) ** rng.random()))))

    family = rng.choice(["quantise", "linear", "linear", "loss", "grad"])
    if family == "quantise":
        layout = rng.choice(sorted(LAYOUTS))
        cols = 128 * log_int(2, 64) if layout == "frag16" else 32 * log_int(2, 256)
        rows = log_int(1, 1 << 15)
        rows = -(-rows // 16) * 16 if layout == "frag16" else rows
        c = _quantise("", rows, cols, rng.choice(sorted(DTYPES)), layout)
    elif family == "linear":
        c = _linear("", log_int(1, 8192), log_int(100, 8192), 32 * log_int(8, 256), rng.choice(["bf16", "bf16", "f32"]),
                    rng.choice(["bf16", "bf16", "f32"]))
    else:
        T, E = log_int(1, 65536), rng.choice([37, 64, 128, 160, 256, 384])
        c = _router("", family, T, E, log_int(1, min(64, T)), rng.choice(["softmax", "sigmoid"]),
                    rng.choice(["f32", "f32", "bf16"]), rng.choice([0, 0, E // 8]))
    del c["name"]
    return c


# ---------------------------------------------------------------- inputs

def _generator(seed, what):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(1000003 * int(seed) + what)
    return g


def _randn(shape, seed, what):
    return torch.randn(shape, generator=_generator(seed, what), device=DEVICE)


def _outliers(shape, seed, what):
    """Rows of an activation or weight matrix: normal values, a few channels 8 times as large."""
    x = _randn(shape, seed, what)
    x[:, torch.randint(0, shape[1], (max(1, shape[1] // 256),), generator=_generator(seed, what + 1), device=DEVICE)] *= 8
    return x


def _codes(x):
    """MXFP4 of fp32 rows: (codes 0..15 [R][C], scale exponents [R][C / 32])."""
    b = x.view(x.shape[0], -1, 32)
    m = b.abs().amax(dim=2)
    e = torch.where(m > 0, torch.frexp(m).exponent - 3, 0).clamp_min(-127)
    v = torch.ldexp(b.abs(), -e[:, :, None])
    step = torch.where(v < 2, 0.5, torch.where(v < 4, 1.0, 2.0))
    v = (torch.round(v / step) * step).clamp_max(6.0)  # round() takes ties to the even multiple
    code = torch.where(v < 2, v * 2, torch.where(v < 4, v + 2, v / 2 + 4)).to(torch.uint8)
    code = code | (torch.signbit(b).to(torch.uint8) << 3)
    return code.view(x.shape), e


def _values(code, e):
    """fp32 values of the codes."""
    m = (code & 7).float()
    v = torch.where(m < 4, m / 2, torch.where(m < 6, m - 2, 2 * m - 8))
    v = torch.where(code >= 8, -v, v).view(code.shape[0], -1, 32)
    return torch.ldexp(v, e[:, :, None]).view(code.shape)


def _tile32(code, e):
    """The library's operand layout: tiles of 32 rows x 256 columns, 4096 bytes of codes (four steps of
    64 columns, each 64 lanes x 16 bytes: lane = 32 * column half + row) and the lanes' 4 scale bytes."""
    R, C = code.shape
    rb, cb = -(-R // 32), -(-C // 256)
    q = torch.zeros((rb * 32, cb * 256), dtype=torch.uint8, device=DEVICE)
    q[:R, :C] = code
    s = torch.full((rb * 32, cb * 8), 127, dtype=torch.uint8, device=DEVICE)
    s[:R, : C // 32] = (e + 127).to(torch.uint8)
    q = q.view(rb, 32, cb, 4, 2, 16, 2)
    q = (q[..., 0] | (q[..., 1] << 4)).permute(0, 2, 3, 4, 1, 5).reshape(rb, cb, 4096)
    s = s.view(rb, 32, cb, 4, 2).permute(0, 2, 4, 1, 3).reshape(rb, cb, 256)
    return torch.cat([q, s], dim=2).contiguous()


def _packed(code):
    q = code.view(code.shape[0], -1, 2)
    return q[:, :, 0] | (q[:, :, 1] << 4)


def _routing(case, seed):
    """Logits, ids and gates as the router leaves them, padding mask and sequence offsets."""
    T, E, k, S = case["T"], case["E"], case["k"], case["seqs"]
    logits = _randn((T, E), seed, 1) + 0.7 * _randn((1, E), seed, 2)
    if case["dead"]:  # experts that are switched off
        logits[:, torch.randperm(E, generator=_generator(seed, 3), device=DEVICE)[: case["dead"]]] = float("-inf")
    logits = logits.to(DTYPES[case["dtype"]])
    top = torch.topk(logits.float(), k, dim=1)
    # Ragged sequences; the last ones may end before the buffer does.
    cuts = torch.rand(S, generator=_generator(seed, 4), device=DEVICE, dtype=torch.float64) + 0.1
    ends = torch.round(torch.cumsum(cuts, 0) / cuts.sum() * (T if S == 1 else max(1, T - T // 64))).to(torch.int32)
    offsets = torch.cat([torch.zeros(1, dtype=torch.int32, device=DEVICE), ends]).contiguous()
    # Padding: one token in sixteen of a packed batch.
    valid = torch.rand(T, generator=_generator(seed, 5), device=DEVICE) >= (1 / 16 if S > 1 else 0)
    return SimpleNamespace(logits=logits, ids=top.indices.to(torch.int32).contiguous(),
                           w=torch.softmax(top.values, dim=1).contiguous(), offsets=offsets,
                           valid=valid.to(torch.uint8), dw=_randn((T, k), seed, 6) * 1e-3,
                           dloss=torch.full((1,), 0.5, device=DEVICE))


def prepare(case, seed):
    s = SimpleNamespace(case=dict(case), ws=None)
    if case["kind"] == "quantise":
        R, C = case["rows"], case["cols"]
        s.x = _outliers((R, C), seed, 1).to(DTYPES[case["dtype"]])
        n = {"rowmajor": R * C // 2, "frag16": R * C * 17 // 32,
             "tile32": -(-R // 32) * -(-C // 256) * 4352}[case["layout"]]
        s.codes = torch.empty(n, dtype=torch.uint8, device=DEVICE)
        s.scales = torch.empty(R * C // 32, dtype=torch.uint8, device=DEVICE) if case["layout"] == "rowmajor" else None
        s.values = torch.empty((R, C), dtype=torch.bfloat16, device=DEVICE)
    elif case["kind"] == "linear":
        T, N, K = case["T"], case["N"], case["K"]
        s.x = _outliers((T, K), seed, 1).to(DTYPES[case["x"]])
        code, e = _codes(_outliers((N, K), seed, 3).mul_(K ** -0.5).to(torch.bfloat16).float())
        s.w_codes, s.w_exp, s.w_tiles = code, e, _tile32(code, e)
        s.y = torch.empty((T, N), dtype=DTYPES[case["y"]], device=DEVICE)
    else:
        s.__dict__.update(_routing(case, seed).__dict__)
        T, E, S = case["T"], case["E"], case["seqs"]
        s.loss = torch.empty(3, device=DEVICE)
        s.probs = torch.empty((S, E), device=DEVICE)
        s.dlogits = torch.empty_like(s.logits)
        if case["kind"] == "grad":  # what the forward call left
            r = _plain_loss(s)
            s.counts, s.tokens = r["counts"], r["tokens"]
        else:
            s.counts = torch.empty((S, E), dtype=torch.int32, device=DEVICE)
            s.tokens = torch.empty(S + 2, dtype=torch.int32, device=DEVICE)
    return s


# ---------------------------------------------------------------- the plain forms

def _plain_quantise(s):
    return {"values": _values(*_codes(s.x.float())).to(torch.bfloat16)}


def _plain_linear(s):
    y = _values(*_codes(s.x.float())) @ _values(s.w_codes, s.w_exp).t()
    return {"y": y.to(s.y.dtype)}


def _scores(logits, score):
    """(probabilities, softmax, log-sum-exp) of fp32 logits."""
    m = logits.amax(dim=1, keepdim=True)
    ex = torch.exp(logits - m)
    z = ex.sum(dim=1, keepdim=True)
    soft, lse = ex / z, (m + torch.log(z))[:, 0]
    if score == "softmax":
        return soft, soft, lse
    sg = 1 / (1 + torch.exp(-logits))
    return sg / sg.sum(dim=1, keepdim=True), soft, lse


def _sequence(s):
    """Sequence of each token (S for the tokens behind the last one), and whether the token counts."""
    t = torch.arange(s.logits.shape[0], device=DEVICE, dtype=torch.int32)
    seq = (t[:, None] >= s.offsets[None, 1:]).sum(dim=1)
    return seq, (s.valid != 0) & (seq < s.offsets.numel() - 1)


def _plain_loss(s):
    E, k, S = s.case["E"], s.case["k"], s.case["seqs"]
    p, _, lse = _scores(s.logits.float(), s.case["score"])
    seq, ok = _sequence(s)
    member = (seq[None, :] == torch.arange(S, device=DEVICE)[:, None]) & ok[None, :]  # [S][T]
    n = member.sum(dim=1)
    hot = torch.zeros(S * E + 1, dtype=torch.int32, device=DEVICE)
    at = torch.where(ok[:, None], seq[:, None] * E + s.ids.long(), S * E)
    counts = hot.index_add_(0, at.view(-1), torch.ones_like(at.view(-1), dtype=torch.int32))[:-1].view(S, E)
    live = n.clamp_min(1).float()
    probs = (member.float() @ p) / live[:, None]
    f = counts.float() * E / (k * live[:, None])
    n_seq, n_tok = (n > 0).sum(), n.sum()
    balance = (f * probs).sum() / n_seq.clamp_min(1)
    z = torch.where(ok, lse * lse, 0).double().sum().float() / n_tok.clamp_min(1)
    return {"loss": torch.stack([ALPHA * balance + Z_COEF * z, balance, z]), "counts": counts, "probs": probs,
            "tokens": torch.cat([n, n_seq[None], n_tok[None]]).to(torch.int32)}


def _plain_grad(s):
    E, k = s.case["E"], s.case["k"]
    p, soft, lse = _scores(s.logits.float(), s.case["score"])
    seq, ok = _sequence(s)
    seq = torch.where(ok, seq, 0)
    n = s.tokens[:-2].clamp_min(1).float()
    n_seq, n_tok = s.tokens[-2].float(), s.tokens[-1].float()
    f = (s.counts.float() * E / (k * n[:, None]))[seq]
    d = p * (f - (f * p).sum(dim=1, keepdim=True))
    if s.case["score"] == "sigmoid":
        d = d / (1 + torch.exp(s.logits.float()))
    d = d * (s.dloss * ALPHA / (n_seq * n[seq]))[:, None] + soft * (s.dloss * Z_COEF * 2 / n_tok * lse)[:, None]
    dl = s.w * (s.dw - (s.w * s.dw).sum(dim=1, keepdim=True))
    d = d.scatter_add(1, s.ids.long(), dl)
    return {"dlogits": torch.where(ok[:, None], d, 0).to(s.logits.dtype)}


def run(state):
    kind = state.case["kind"]
    if own:
        return _OWN[kind](state)
    return {"quantise": _plain_quantise, "linear": _plain_linear, "loss": _plain_loss, "grad": _plain_grad}[kind](state)


# ---------------------------------------------------------------- the library's calls

def _own_quantise(s):
    from paper_2607_23099_amd import damoe
    R, C, layout = s.case["rows"], s.case["cols"], LAYOUTS[s.case["layout"]]
    damoe.mxfp4_quantise(s.x, R, C, s.codes, s.scales, layout)
    damoe.mxfp4_dequantise(s.codes, s.scales, R, C, s.values, layout)
    return {"values": s.values}


def _own_linear(s):
    from paper_2607_23099_amd import damoe
    T, N, K = s.case["T"], s.case["N"], s.case["K"]
    if s.ws is None:
        s.ws = torch.zeros(damoe.mxfp4_linear_workspace_size(T, N, K), dtype=torch.uint8, device=DEVICE)
    damoe.mxfp4_linear(s.x, T, K, s.w_tiles, N, s.y, s.ws)
    return {"y": s.y}


def _score_id(s):
    return 1 if s.case["score"] == "sigmoid" else 0


def _own_loss(s):
    from paper_2607_23099_amd import damoe
    T, E, k, S = s.case["T"], s.case["E"], s.case["k"], s.case["seqs"]
    if s.ws is None:
        s.ws = torch.zeros(damoe.router_loss_workspace_size(T, E, S), dtype=torch.uint8, device=DEVICE)
    damoe.router_loss(s.logits, s.ids, T, E, k, s.loss, s.counts, s.tokens, s.ws, mask=s.valid, seq_offsets=s.offsets,
                      S=S, score=_score_id(s), alpha=ALPHA, z_coef=Z_COEF, probs=s.probs)
    return {"loss": s.loss, "counts": s.counts, "probs": s.probs, "tokens": s.tokens}


def _own_grad(s):
    from paper_2607_23099_amd import damoe
    T, E, k, S = s.case["T"], s.case["E"], s.case["k"], s.case["seqs"]
    damoe.router_loss_grad(s.logits, s.ids, T, E, k, s.counts, s.tokens, s.dlogits, mask=s.valid,
                           seq_offsets=s.offsets, S=S, score=_score_id(s), alpha=ALPHA, z_coef=Z_COEF,
                           dloss=s.dloss, w=s.w, dw=s.dw)
    return {"dlogits": s.dlogits}


_OWN = {"quantise": _own_quantise, "linear": _own_linear, "loss": _own_loss, "grad": _own_grad}


# ---------------------------------------------------------------- work and exact values

def work(case):
    size = {"bf16": 2, "f32": 4}
    if case["kind"] == "quantise":
        n = case["rows"] * case["cols"]
        return {"bytes": n * (size[case["dtype"]] + 2 * 17 / 32 + 2), "flops": 0}
    if case["kind"] == "linear":
        T, N, K = case["T"], case["N"], case["K"]
        return {"bytes": N * K * 17 / 32 + T * K * size[case["x"]] + T * N * size[case["y"]], "flops": 2 * T * N * K}
    T, E, k, S, b = case["T"], case["E"], case["k"], case["seqs"], size[case["dtype"]]
    if case["kind"] == "loss":
        return {"bytes": T * (E * b + 4 * k + 1) + S * E * 8, "flops": 4 * T * E}
    return {"bytes": T * (2 * E * b + 12 * k + 1) + S * E * 4, "flops": 8 * T * E}


def _exact_quantised(x):
    """The values that MXFP4 gives rows in float64: every value goes to the nearest of 15 levels of its
    block, found by its place among the midpoints between them (a value on one goes to the even code)."""
    b = x.double().reshape(x.shape[0], -1, 32)
    levels = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device=DEVICE)
    middle = (levels[1:] + levels[:-1]) / 2
    m = b.abs().amax(dim=2, keepdim=True)
    scale = torch.exp2(torch.floor(torch.log2(torch.where(m > 0, m, 4.0))) - 2)
    # log2 is rounded: the scale is the one with 4 <= m / scale < 8.
    scale = torch.where(m >= 8 * scale, 2 * scale, torch.where((m > 0) & (m < 4 * scale), scale / 2, scale))
    a = (b / scale).abs()
    low, high = torch.bucketize(a, middle), torch.bucketize(a, middle, right=True)
    level = levels[torch.where((low != high) & (low % 2 == 1), high, low)]
    return (torch.sign(b) * level * scale).reshape(x.shape)


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "quantise":
        return {"values": _exact_quantised(s.x)}
    if case["kind"] == "linear":
        w = _outliers((case["N"], case["K"]), seed, 3).mul_(case["K"] ** -0.5).to(torch.bfloat16)
        return {"y": _exact_quantised(s.x) @ _exact_quantised(w).t().contiguous()}
    E, k, S = case["E"], case["k"], case["seqs"]
    logits, bounds = s.logits.double(), s.offsets.tolist()
    soft = torch.softmax(logits, dim=1)
    lse = torch.logsumexp(logits, dim=1)
    sig = torch.sigmoid(logits)
    p = soft if case["score"] == "softmax" else sig / sig.sum(dim=1, keepdim=True)
    rows = [a + torch.nonzero(s.valid[a:b]).view(-1) for a, b in zip(bounds[:-1], bounds[1:])]
    n = [r.numel() for r in rows]
    n_seq, n_tok = max(1, sum(v > 0 for v in n)), max(1, sum(n))
    counts = torch.stack([torch.bincount(s.ids[r].view(-1).long(), minlength=E) for r in rows])
    probs = torch.stack([p[r].sum(dim=0) / max(1, r.numel()) for r in rows])
    f = torch.stack([c.double() * E / (k * max(1, m)) for c, m in zip(counts, n)])
    if case["kind"] == "loss":
        balance = (f * probs).sum() / n_seq
        z = sum((lse[r] ** 2).sum() for r in rows) / n_tok
        return {"loss": torch.stack([ALPHA * balance + Z_COEF * z, balance, z]), "counts": counts, "probs": probs,
                "tokens": torch.tensor(n + [sum(v > 0 for v in n), sum(n)])}
    g = float(s.dloss)
    out = torch.zeros_like(logits)
    w, dw = s.w.double(), s.dw.double()
    for i, r in enumerate(rows):
        if not n[i]:
            continue
        d = f[i] - (p[r] @ f[i])[:, None]
        d = p[r] * d if case["score"] == "softmax" else p[r] * (1 - sig[r]) * d
        d = g * ALPHA / (n_seq * n[i]) * d + (2 * g * Z_COEF / n_tok) * lse[r][:, None] * soft[r]
        out[r] = d.scatter_add(1, s.ids[r].long(), w[r] * (dw[r] - (w[r] * dw[r]).sum(dim=1, keepdim=True)))
    return {"dlogits": out}
