"""A program that drives its own layers: embedding, LayerNorm, projections, attention in a window, a tied head, the loss, the backward
pass and the update of every tensor, through the library's calls in the order such a program makes them, against float64 autograd; the
same captured into a graph; the calls on streams of their own and side by side."""
import math

import pytest
import torch

import paper_2204_06514_amd as fax
from oracle import operators as orc
from helpers import DEV, TOL_BF16, TOL_F32

pytestmark = pytest.mark.gpu
HP = (1e-3, 0.9, 0.999, 1e-8, 0.01)
V, D, H, HKV, DH, WINDOW, SINKS, EPS = 203, 64, 4, 2, 16, 9, 2, 1e-5
QKV = (H + 2 * HKV) * DH
SHAPES = {"emb": (V, D), "g1": (D,), "b1": (D,), "wqkv": (D, QKV), "bqkv": (QKV,), "wo": (H * DH, D), "bo": (D,), "g2": (D,), "b2": (D,)}
DECAYS = ("emb", "wqkv", "wo")
SCALE = math.sqrt(D)


def parameters(dtype, seed=0):
    gen = torch.Generator().manual_seed(seed)
    p = {n: (0.1 * torch.randn(s, generator=gen)) for n, s in SHAPES.items()}
    for n in ("g1", "g2"):
        p[n] += 1.0
    return {n: t.to(dtype) for n, t in p.items()}


def data(B, S, seed=1):
    gen = torch.Generator().manual_seed(seed)
    ids = torch.randint(0, V, (B, S + 1), generator=gen).to(torch.int32)
    return ids[:, :-1].contiguous(), ids[:, 1:].contiguous()


class Layers:
    """Buffers and calls of one training step."""

    def __init__(self, B, S, dtype, state):
        self.B, self.S, self.T, self.td, self.code = B, S, B * S, dtype, fax.dtype_code(dtype)
        new = lambda *s, t=dtype: torch.empty(s, dtype=t, device=DEV)  # noqa: E731
        T = self.T
        self.p = {n: t.to(DEV) for n, t in parameters(dtype).items()}
        self.master = self.p if dtype == torch.float32 else {n: t.float() for n, t in self.p.items()}
        self.grad = {n: new(*s, t=torch.float32) for n, s in SHAPES.items()}
        self.x, self.h, self.qkv, self.ctx, self.y, self.hf, self.logits = new(T, D), new(T, D), new(T, QKV), new(T, H * DH), new(T, D), new(T, D), new(T, V)
        self.dlogits, self.dhf, self.dy, self.dctx, self.dqkv, self.dh, self.dx = new(T, V), new(T, D), new(T, D), new(T, H * DH), new(T, QKV), new(T, D), new(T, D)
        self.stats = [new(T, t=torch.float32) for _ in range(4)]
        self.lse, self.rows, self.loss = new(B, H, S, t=torch.float32), new(T, t=torch.float32), torch.zeros(4, device=DEV)
        self.ones = torch.ones(T, 1, dtype=dtype, device=DEV)
        q, k, v = (t for t in self.heads(self.qkv))
        self.dims = fax.window_dims(q, k, WINDOW, SINKS)
        self.ws_bytes = max(fax.fax_window_attention_workspace_bytes(self.dims), fax.fax_embedding_bwd_workspace_bytes(T, V, D),
                            fax.fax_layernorm_bwd_workspace_bytes(D))
        self.ws = torch.empty(self.ws_bytes, dtype=torch.uint8, device=DEV)
        self.state, self.hp = state, fax.FaxAdamW(*HP)
        tensors = []
        self.m, self.v, self.scales = {}, {}, []
        for n, s in SHAPES.items():
            k = math.prod(s)
            kind = torch.float32 if state == fax.FAX_STATE_F32 else torch.float8_e4m3fn
            self.m[n], self.v[n] = torch.zeros(k, dtype=kind, device=DEV), torch.zeros(k, dtype=kind, device=DEV)
            e = dict(master=self.master[n], m=self.m[n], v=self.v[n], grad=self.grad[n], decay=n in DECAYS,
                     lowp=self.p[n] if dtype == torch.bfloat16 else None)
            if state == fax.FAX_STATE_E4M3:
                e.update(m_scale=torch.zeros((k + 255) // 256, device=DEV), v_scale=torch.zeros((k + 255) // 256, device=DEV))
                self.scales += [e["m_scale"], e["v_scale"]]
            tensors.append(e)
        self.table = fax.adamw_tensors(tensors)

    def heads(self, packed):
        return packed.view(self.B, self.S, H + 2 * HKV, DH).split([H, HKV, HKV], 2)

    def gradients(self, tokens, labels):
        c, T, p, g, ws, n = self.code, self.T, self.p, self.grad, self.ws, self.ws_bytes
        mu1, r1, mu2, r2 = self.stats
        heads = lambda t: t.view(self.B, self.S, H, DH)  # noqa: E731
        fax.fax_embedding_fwd(c, T, V, D, tokens, p["emb"], SCALE, self.x)
        fax.fax_layernorm_fwd(c, T, D, self.x, p["g1"], p["b1"], EPS, self.h, mu1, r1)
        fax.fax_gemm(c, 0, 0, T, QKV, D, self.h, D, p["wqkv"], QKV, self.qkv, QKV, bias=p["bqkv"])
        q, k, v = self.heads(self.qkv)
        fax.fax_window_attention_fwd(self.dims, q, k, v, None, None, heads(self.ctx), self.lse, ws, n)
        fax.fax_gemm(c, 0, 0, T, D, H * DH, self.ctx, H * DH, p["wo"], D, self.y, D, bias=p["bo"], residual=self.x, ldr=D)
        fax.fax_layernorm_fwd(c, T, D, self.y, p["g2"], p["b2"], EPS, self.hf, mu2, r2)
        fax.fax_gemm(c, 0, 1, T, V, D, self.hf, D, p["emb"], D, self.logits, V)
        fax.fax_cross_entropy(c, T, V, self.logits, labels, self.dlogits, self.rows, self.loss)
        # backward; weight gradients are fp32, column sums products with ones
        def column_sums(x, width, out):
            fax.fax_gemm(c, 1, 0, 1, width, T, self.ones, 1, x, width, out, width, c_f32=1)
        fax.fax_gemm(c, 1, 0, V, D, T, self.dlogits, V, self.hf, D, g["emb"], D, c_f32=1)
        fax.fax_gemm(c, 0, 0, T, D, V, self.dlogits, V, p["emb"], D, self.dhf, D)
        fax.fax_layernorm_bwd(c, T, D, self.dhf, self.y, mu2, r2, p["g2"], None, self.dy, g["g2"], g["b2"], 0, ws, n)
        fax.fax_gemm(c, 1, 0, H * DH, D, T, self.ctx, H * DH, self.dy, D, g["wo"], D, c_f32=1)
        column_sums(self.dy, D, g["bo"])
        fax.fax_gemm(c, 0, 1, T, H * DH, D, self.dy, D, p["wo"], D, self.dctx, H * DH)
        dq, dk, dv = self.heads(self.dqkv)
        fax.fax_window_attention_bwd(self.dims, q, k, v, None, None, heads(self.ctx), self.lse, heads(self.dctx), dq, dk, dv, ws, n)
        fax.fax_gemm(c, 1, 0, D, QKV, T, self.h, D, self.dqkv, QKV, g["wqkv"], QKV, c_f32=1)
        column_sums(self.dqkv, QKV, g["bqkv"])
        fax.fax_gemm(c, 0, 1, T, D, QKV, self.dqkv, QKV, p["wqkv"], QKV, self.dh, D)
        fax.fax_layernorm_bwd(c, T, D, self.dh, self.x, mu1, r1, p["g1"], self.dy, self.dx, g["g1"], g["b1"], 0, ws, n)
        fax.fax_embedding_bwd(c, T, V, D, tokens, self.dx, SCALE, g["emb"], 1, ws, n)  # onto the head's share

    def update(self, step, seed=3):
        fax.fax_adamw_multi_step(self.state, self.table, self.hp, step, seed)

    def everything(self):
        return [self.loss[:1], self.logits, *self.grad.values(), *self.master.values(), *self.p.values(), *[t.float() for t in self.m.values()],
                *[t.float() for t in self.v.values()], *self.scales]


def reference(p, tokens, labels):
    """Loss and gradients in float64 by autograd."""
    p = {n: t.double().requires_grad_() for n, t in p.items()}
    B, S = tokens.shape
    ln = lambda x, g, b: (x - x.mean(-1, keepdim=True)) / torch.sqrt(x.var(-1, unbiased=False, keepdim=True) + EPS) * g + b  # noqa: E731
    x = p["emb"][tokens.long()] * SCALE
    qkv = (ln(x, p["g1"], p["b1"]) @ p["wqkv"] + p["bqkv"]).view(B, S, H + 2 * HKV, DH)
    ctx = orc.window_attention(*qkv.split([H, HKV, HKV], 2), WINDOW, SINKS)["ctx"]
    y = x + ctx.reshape(B, S, H * DH) @ p["wo"] + p["bo"]
    logits = ln(y, p["g2"], p["b2"]) @ p["emb"].T
    loss = torch.nn.functional.cross_entropy(logits.view(-1, V), labels.long().view(-1))
    loss.backward()
    return loss.detach(), {n: t.grad for n, t in p.items()}


@pytest.mark.parametrize("dtype,state", [(torch.float32, fax.FAX_STATE_F32), (torch.bfloat16, fax.FAX_STATE_F32), (torch.bfloat16, fax.FAX_STATE_E4M3)],
                         ids=["f32", "bf16", "bf16-8bit"])
def test_a_training_step(dtype, state):
    B, S = 3, 41
    m = Layers(B, S, dtype, state)
    tokens, labels = data(B, S)
    m.gradients(tokens.to(DEV), labels.to(DEV))
    loss, grads = reference(parameters(dtype), tokens, labels)
    tol = TOL_F32 if dtype == torch.float32 else TOL_BF16
    assert abs(m.loss[0].item() - loss.item()) <= tol * abs(loss.item())
    for n, ref in grads.items():
        got = m.grad[n].cpu().double()
        keep = torch.ones_like(ref, dtype=torch.bool)
        if n == "bqkv":  # the softmax does not see a bias of all keys: its gradient is zero but for rounding
            keep[H * DH:(H + HKV) * DH] = False
        off, size = (got - ref)[keep], ref[keep]
        err = off.abs().max() / size.abs().max() if dtype == torch.float32 else off.norm() / size.norm()
        assert err <= tol, (n, err.item())
    # the update, from the gradients that are there
    before = {n: t.cpu().double() for n, t in m.master.items()}
    got_grads = {n: t.cpu().double() for n, t in m.grad.items()}
    m.update(1)
    for n in SHAPES:
        z = torch.zeros_like(before[n])
        p, _, _, e, _, _ = orc.adamw(before[n], z, z, got_grads[n], HP, 1, n in DECAYS)
        assert ((m.master[n].cpu().double() - p).abs() <= e).all(), n
        if dtype == torch.bfloat16:
            assert torch.equal(m.p[n], m.master[n].to(torch.bfloat16))


@pytest.mark.parametrize("state", [fax.FAX_STATE_F32, fax.FAX_STATE_E4M3], ids=["32bit", "8bit"])
@pytest.mark.parametrize("S", [41, 700])
def test_captured_and_replayed(S, state):
    """A graph of the whole step, replayed with the program's own eager work and new tokens between: every replay gives the eager bits."""
    B = 2
    eager, graphed = Layers(B, S, torch.bfloat16, state), Layers(B, S, torch.bfloat16, state)
    tokens, labels = (t.to(DEV) for t in data(B, S))
    warm = Layers(B, S, torch.bfloat16, state)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        warm.gradients(tokens, labels)
        warm.update(5)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            graphed.gradients(tokens, labels)
            graphed.update(5)
    for k in range(4):
        t, l = data(B, S, seed=10 + k)
        tokens.copy_(t.to(DEV))
        labels.copy_(l.to(DEV))
        eager.gradients(tokens, labels)
        eager.update(5)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(eager.everything(), graphed.everything()):
            assert torch.equal(a, b), k


def test_two_programs_side_by_side():
    """Two models, each on a stream of its own with a workspace of its own, enqueued in turn: the bits of either by itself."""
    B, S = 2, 300
    alone = []
    for k in range(2):
        m = Layers(B, S, torch.bfloat16, fax.FAX_STATE_E4M3)
        t, l = (x.to(DEV) for x in data(B, S, seed=20 + k))
        for step in (1, 2, 3):
            m.gradients(t, l)
            m.update(step)
        alone.append([x.clone() for x in m.everything()])
    torch.cuda.synchronize()
    both = [Layers(B, S, torch.bfloat16, fax.FAX_STATE_E4M3) for _ in range(2)]
    inputs = [[x.to(DEV) for x in data(B, S, seed=20 + k)] for k in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for step in (1, 2, 3):
        for m, (t, l), s in zip(both, inputs, streams):
            with torch.cuda.stream(s):
                m.gradients(t, l)
                m.update(step)
    torch.cuda.synchronize()
    for m, ref in zip(both, alone):
        for a, b in zip(m.everything(), ref):
            assert torch.equal(a, b)


def test_timing_report_names_them():
    m = Layers(2, 41, torch.bfloat16, fax.FAX_STATE_F32)
    tokens, labels = (t.to(DEV) for t in data(2, 41))
    fax.fax_timing_enable(1)
    m.gradients(tokens, labels)
    m.update(1)
    rows = {r["name"]: r for r in fax.fax_timing_report()}
    fax.fax_timing_enable(0)
    pairs = sum(min(i + 1, WINDOW) + min(SINKS, max(0, i + 1 - WINDOW)) for i in range(41)) * 2 * H
    assert rows["window_attention_fwd"]["work"] == 4.0 * DH * pairs and rows["window_attention_bwd"]["work"] == 10.0 * DH * pairs
    for n in ("embedding_fwd", "embedding_bwd", "adamw_multi"):
        assert rows[n]["launches"] == 1 and rows[n]["ms"] > 0 and rows[n]["work"] > 0
