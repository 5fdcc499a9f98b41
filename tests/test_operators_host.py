"""CPU-only: what the embedding, window-attention and many-tensor AdamW calls refuse, before anything is enqueued, their size
queries, and the oracle's own definitions against simpler ones."""
import math

import pytest
import torch

import paper_2204_06514_amd as fax
from oracle import operators as orc

A = 4096  # an address that is never read: every call here fails first


def refused(status, text, f, *a, **k):
    with pytest.raises(fax.FaxError) as e:
        f(*a, **k)
    assert e.value.status == status and text in str(e.value), str(e.value)


INVALID, UNSUPPORTED, WORKSPACE = fax.FAX_ERR_INVALID_ARG, fax.FAX_ERR_UNSUPPORTED, fax.FAX_ERR_WORKSPACE


def test_embedding_refusals():
    fwd = lambda dtype=fax.FAX_BF16, N=4, V=8, D=8, t=A, w=A, o=A: fax.fax_embedding_fwd(dtype, N, V, D, t, w, 1.0, o, stream=0)  # noqa: E731
    refused(INVALID, "dtype", fwd, dtype=5)
    for bad in (dict(N=-1), dict(V=0), dict(D=0)):
        refused(INVALID, "size", fwd, **bad)
    refused(UNSUPPORTED, "2^30", fwd, N=(1 << 30) + 1)
    refused(INVALID, "tokens", fwd, t=None)
    refused(INVALID, "table", fwd, w=None)
    refused(INVALID, "out", fwd, o=A + 2)
    fwd(N=0, t=None, w=None, o=None)  # nothing to do
    need = fax.fax_embedding_bwd_workspace_bytes(100, 50, 8)
    bwd = lambda N=100, t=A, d=A, g=A, w=A, n=need, dtype=fax.FAX_F32: fax.fax_embedding_bwd(dtype, N, 50, 8, t, d, 1.0, g, 0, w, n, stream=0)  # noqa: E731
    refused(INVALID, "dtable", bwd, g=None)
    refused(INVALID, "dout", bwd, d=A + 8)
    refused(INVALID, "ws", bwd, w=None)
    refused(WORKSPACE, "workspace", bwd, n=need - 1)
    refused(INVALID, "dtype", bwd, dtype=2)
    fax.fax_embedding_bwd(fax.FAX_F32, 0, 50, 8, None, None, 1.0, A, 1, None, 0, stream=0)  # nothing to add
    refused(INVALID, "size", fax.fax_embedding_bwd_workspace_bytes, 1, 0, 1)


def dims(**kw):
    d = dict(B=2, Sq=64, Sk=64, H=4, Hkv=2, dh=64, dtype=fax.FAX_BF16, window=16, sinks=2)
    strides = {n: kw.pop(n, fax.FaxStrides()) for n in ("q", "kv", "ctx")}
    d.update(kw)
    return fax.FaxWindowDims(*d.values(), *strides.values())


def test_window_refusals():
    size = fax.fax_window_attention_workspace_bytes
    assert size(dims()) > 0
    for bad in (dict(B=0), dict(Sq=0), dict(Sk=-1), dict(H=0), dict(Hkv=0), dict(dh=0)):
        refused(INVALID, "non-positive", size, dims(**bad))
    refused(INVALID, "multiple", size, dims(H=3))
    refused(INVALID, "window", size, dims(window=0))
    refused(INVALID, "sinks", size, dims(sinks=-1))
    refused(INVALID, "dtype", size, dims(dtype=7))
    refused(UNSUPPORTED, "256", size, dims(dh=264))
    refused(UNSUPPORTED, "2^30", size, dims(B=1 << 20, Sk=1 << 11))
    refused(INVALID, "negative", size, dims(q=fax.FaxStrides(64, -64, 1)))
    refused(UNSUPPORTED, "2^40", size, dims(kv=fax.FaxStrides(1 << 41, 64, 64)))
    refused(INVALID, "overlap", size, dims(ctx=fax.FaxStrides(64 * 256, 255, 64)))
    need = size(dims())
    fwd = lambda d=dims(), q=A, k=A, v=A, ctx=A, lse=A, ws=A, n=need, pos=None: fax.fax_window_attention_fwd(d, q, k, v, pos, None, ctx, lse, ws, n, stream=0)  # noqa: E731
    for name in ("q", "k", "v", "ctx"):
        refused(INVALID, name, fwd, **{name: None})
        refused(INVALID, name, fwd, **{name: A + 1})
    refused(INVALID, "lse", fwd, lse=A + 2)
    refused(INVALID, "q_pos", fwd, pos=A + 2)
    refused(INVALID, "ws", fwd, ws=None)
    refused(WORKSPACE, "workspace", fwd, n=need - 1)
    bwd = lambda d=dims(), lse=A, dk=A, n=need: fax.fax_window_attention_bwd(d, A, A, A, None, None, A, lse, A, A, dk, A, A, n, stream=0)  # noqa: E731
    refused(INVALID, "lse", bwd, lse=None)
    refused(INVALID, "dk", bwd, dk=None)
    refused(WORKSPACE, "workspace", bwd, n=need - 1)
    # a key head that two sequences share may be read, but not be written
    shared = dims(kv=fax.FaxStrides(0, 128, 64))
    assert size(shared) > 0
    refused(INVALID, "dims.kv", bwd, d=shared)
    refused(INVALID, "dims.q", bwd, d=dims(q=fax.FaxStrides(64 * 256, 256, 32)))


def test_window_dims_of_views():
    qkv = torch.zeros(2, 10, 4 + 2 * 2, 16, dtype=torch.bfloat16)
    q, k, v = qkv.split([4, 2, 2], 2)
    d = fax.window_dims(q, k, 5, 1)
    assert (d.B, d.Sq, d.Sk, d.H, d.Hkv, d.dh, d.window, d.sinks) == (2, 10, 10, 4, 2, 16, 5, 1)
    assert (d.q.batch, d.q.row, d.q.head) == (1280, 128, 16) == (d.kv.batch, d.kv.row, d.kv.head)
    with pytest.raises(AssertionError):
        fax.window_dims(q.transpose(2, 3), k, 5)
    # a tensor in another layout than dims say is not handed on
    need = fax.fax_window_attention_workspace_bytes(d)
    ctx = torch.zeros(2, 10, 4, 16, dtype=torch.bfloat16)
    for args in ((q.contiguous(), k, v, ctx), (q, k.contiguous(), v, ctx), (q, k, v, q), (q, k, v[:, :9], ctx)):
        with pytest.raises(AssertionError):
            fax.fax_window_attention_fwd(d, *args[:3], None, None, args[3], None, 4096, need, stream=0)


def test_adamw_multi_refusals():
    hp = fax.FaxAdamW(1e-3, 0.9, 0.999, 1e-8, 0.01)
    step = lambda e=None, state=fax.FAX_STATE_F32, count=1, hp=hp, t=1: fax.fax_adamw_multi_step(state, (e, count), hp, t, 0, stream=0)  # noqa: E731

    def entry(**kw):
        d = dict(master=A, m=A, v=A, grad=A, lowp=None, m_scale=None, v_scale=None, n=16, grad_dtype=fax.FAX_F32, decay=1)
        d.update(kw)
        return (fax.FaxAdamWTensor * 1)(fax.FaxAdamWTensor(*d.values()))

    refused(INVALID, "state", step, entry(), state=2)
    refused(INVALID, "count", step, entry(), count=-1)
    refused(INVALID, "tensors", step, None)
    refused(INVALID, "hp", step, entry(), hp=None)
    refused(INVALID, "step", step, entry(), t=0)
    for n in ("master", "m", "v", "grad"):
        refused(INVALID, "tensors[0]." + n, step, entry(**{n: None}))
        refused(INVALID, "aligned", step, entry(**{n: A + 4}))
    refused(INVALID, "lowp", step, entry(lowp=A + 8))
    refused(INVALID, "grad_dtype", step, entry(grad_dtype=3))
    refused(UNSUPPORTED, "elements", step, entry(n=1 << 43))
    refused(INVALID, "m_scale", step, entry(), state=fax.FAX_STATE_E4M3)
    refused(INVALID, "v_scale", step, entry(m_scale=A, v_scale=A + 2), state=fax.FAX_STATE_E4M3)
    step(None, count=0)
    step(entry(n=0, master=None), state=fax.FAX_STATE_E4M3)


# ---- the oracle ---------------------------------------------------------------------------------------
def test_oracle_window_against_differences_and_full_attention():
    torch.manual_seed(0)
    B, S, H, Hkv, dh = 2, 7, 4, 2, 4
    q, k, v, d = (torch.randn(B, S, h, dh, dtype=torch.float64) for h in (H, Hkv, Hkv, H))
    q_pos, k_len = torch.tensor([0, -2]), torch.tensor([7, 4])
    r = orc.window_attention(q, k, v, 3, 1, q_pos, k_len, d)
    assert (r["ctx"][1, :2] == 0).all() and torch.isinf(r["lse"][1, :, :2]).all()  # before the first key
    f = lambda **t: (orc.window_attention(t.get("q", q), t.get("k", k), t.get("v", v), 3, 1, q_pos, k_len)["ctx"] * d).sum()  # noqa: E731
    for name, x in (("q", q), ("k", k), ("v", v)):
        g = r["d" + name]
        for at in [(0, 0, 0, 0), (0, 3, 1, 2), (1, 5, 1, 1), (1, 2, 0, 3), (0, 6, 0, 0)]:
            e = torch.zeros_like(x)
            e[at] = 1e-6
            diff = (f(**{name: x + e}) - f(**{name: x - e})) / 2e-6
            assert abs(diff - g[at]) < 1e-7 * (1 + abs(diff)), (name, at)
    # a window as long as the sequence is causal attention
    full = orc.window_attention(q, q[:, :, :2], v, S, 0)
    s = torch.einsum("bihd,bjhd->bhij", q, q[:, :, :2].repeat_interleave(2, 2)) / 2.0
    P = torch.softmax(s.masked_fill(torch.ones(S, S).triu(1).bool(), -math.inf), -1)
    assert torch.allclose(full["ctx"], torch.einsum("bhij,bjhd->bihd", P, v.repeat_interleave(2, 2)), atol=1e-12)


def test_oracle_e4m3_is_torchs_format():
    codes = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float()
    values = codes[torch.isfinite(codes)].double()
    assert values.max() == 448.0 and values[values > 0].min() == 2.0 ** -9
    assert torch.equal(orc.e4m3_nearest(values), values)
    x = torch.linspace(-448, 448, 4001, dtype=torch.float64) ** 3 / 448 ** 2
    assert torch.equal(orc.e4m3_nearest(x), x.float().to(torch.float8_e4m3fn).double())
    # rounding at random keeps the mean
    u = (torch.arange(1 << 12, dtype=torch.float64) + 0.5) / (1 << 12)
    for y in (0.013, 0.3, 5.1, 200.0):
        assert abs(orc.e4m3_random(torch.full_like(u, y), u).mean() - y) < 2e-4 * max(y, 0.1)
    r = orc.random20(7, 3, 1, 1 << 16)
    assert abs(r.mean() - 0.5) < 5e-3 and abs((r * r).mean() - 1 / 3) < 5e-3
    assert abs((r[1:] * r[:-1]).mean() - 0.25) < 5e-3


def test_window_sizes_that_launches_do_not_reach():
    size = fax.fax_window_attention_workspace_bytes
    refused(UNSUPPORTED, "2^27", size, dims(B=1 << 12, Sq=1 << 14, H=4))
    refused(UNSUPPORTED, "2^27", size, dims(B=1 << 12, Sk=1 << 15, H=2, Hkv=2))
    refused(UNSUPPORTED, "2^21", size, dims(B=1 << 21, Sq=1, Sk=1, H=2, Hkv=2))
    size(dims(B=1 << 20, Sq=1, Sk=1, H=2, Hkv=2))
    size(dims(B=1, Sq=1 << 22, Sk=1 << 22, H=32, Hkv=32))


def test_window_sinks_without_end_take_no_workspace_without_end():
    """Half of the keys as sinks: their parts stay within some thousand tiles of 64 keys, dK and dV in fp32."""
    for dtype in (fax.FAX_F32, fax.FAX_BF16):
        for S, sinks in ((1 << 17, 1 << 16), (1 << 20, 1000), (40000, 20000)):
            d = dims(B=1, Sq=S, Sk=S, H=8, Hkv=8, dh=128, window=1024, sinks=sinks, dtype=dtype)
            delta = 4 * S * 8
            assert fax.fax_window_attention_workspace_bytes(d) - delta < 2 * 4096 * 64 * 2 * 128 * 4


def test_adamw_of_more_than_memory_holds():
    one = (fax.FaxAdamWTensor * 1)(fax.FaxAdamWTensor(A, A, A, A, None, None, None, (1 << 35) + 1, fax.FAX_F32, 1))
    hp = fax.FaxAdamW(1e-3, 0.9, 0.95, 1e-8, 0.1)
    refused(UNSUPPORTED, "elements", fax.fax_adamw_multi_step, fax.FAX_STATE_F32, (one, 1), hp, 1, 0, stream=0)


def test_window_tensors_are_as_dims_say():
    import torch
    q, k = torch.zeros(1, 5, 2, 8), torch.zeros(1, 5, 2, 8)
    d = fax.window_dims(q, k, 3)
    call = lambda v, ctx=q: fax.fax_window_attention_fwd(d, q, k, v, None, None, ctx, None, A, 1 << 20, stream=0)  # noqa: E731
    for v in (k.bfloat16(), k[:, :4], torch.zeros(1, 5, 2, 16)[..., :8], k.permute(0, 1, 3, 2)):
        with pytest.raises(AssertionError):
            call(v)
    with pytest.raises(AssertionError):
        call(k, ctx=q.bfloat16())
