"""fax_window_attention_*: every form that its sizes can take, each at a size that takes it (fax_window_attention_route says so), against
float64 with derived bounds."""
import math

import pytest
import torch

import paper_2204_06514_amd as fax
from oracle import operators as orc
from helpers import DEV
from test_gpu_window import TD, both, check, make, run

pytestmark = pytest.mark.gpu


def route(B, Sq, Sk, H, Hkv, dh, dtype, window, sinks):
    code = fax.FAX_F32 if dtype == "f32" else fax.FAX_BF16
    return fax.fax_window_attention_route(fax.FaxWindowDims(B, Sq, Sk, H, Hkv, dh, code, window, sinks, *[fax.FaxStrides()] * 3))


def forms(r):
    return {n: getattr(r, n) for n, _ in r._fields_}


# Whole workgroups of four wavefronts, in every head width class; the sinks' keys cut and not.
@pytest.mark.parametrize("dh", [40, 64, 80, 128, 104])
@pytest.mark.parametrize("H,Hkv", [(32, 32), (40, 10)])
@pytest.mark.parametrize("window,sinks", [(100, 4), (2000, 130)])
def test_four_wavefronts(dh, H, Hkv, window, sinks):
    S = 2100 if Hkv == 32 else 1700
    if Hkv == 10 and dh in (40, 104):
        pytest.skip("two widths are enough for grouped heads")
    r = route(1, S, S, H, Hkv, dh, "bf16", window, sinks)
    assert (r.waves, r.fwd_splits, r.dq_splits) == (4, 1, 1) and r.sink_splits > 1 or window > 100, forms(r)
    if Hkv == 32:
        assert r.key_splits == 1, forms(r)
    both(1, S, S, H, Hkv, dh, "bf16", window, sinks, torch.tensor([0], dtype=torch.int32), torch.tensor([S - 70], dtype=torch.int32))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh", [24, 64, 96, 128])
@pytest.mark.parametrize("S,H,Hkv,window,sinks", [(1500, 2, 1, 10000, 0), (1500, 4, 4, 1000, 3), (1500, 8, 1, 64, 70), (1500, 1, 1, 700, 1500)])
def test_cut_streams(S, H, Hkv, window, sinks, dh, dtype):
    r = route(1, S, S, H, Hkv, dh, dtype, window, sinks)
    if H == 2 or (H == 4 and dtype == "bf16"):
        assert min(r.dq_splits, r.key_splits) > 1 and (r.fwd_splits > 1 or H == 4) and (r.sink_splits > 1) == (H == 4), forms(r)
    if sinks == 70:
        assert r.sink_splits > 1, forms(r)
    if sinks == 1500:
        assert r.sink_splits == 1 and r.key_splits > 1, forms(r)
    both(1, S, S, H, Hkv, dh, dtype, window, sinks)


# Two groups of wavefronts with the same rows, which take every other tile: even and odd numbers of tiles, runs of whole ones among them, rows that see
# one group's tiles only, workgroups with fewer tiles than groups.
@pytest.mark.parametrize("dh", [40, 64, 80, 128])
@pytest.mark.parametrize("B,S,H,Hkv,window,sinks,dq", [(8, 400, 8, 4, 200, 0, 1), (4, 1000, 8, 8, 300, 3, 2), (2, 1111, 14, 7, 333, 70, 2), (6, 600, 8, 8, 600, 0, 2)])
def test_two_groups(B, S, H, Hkv, window, sinks, dq, dh):
    r = route(B, S, S, H, Hkv, dh, "bf16", window, sinks)
    assert (r.waves, r.fwd_groups, r.dq_groups, r.fwd_splits, r.dq_splits) == (4, 2, dq, 1, 1), forms(r)
    short = torch.arange(B, dtype=torch.int32)
    k_len = (S - 37 * short).clamp(min=1)
    k_len[-1] = 50 if B > 3 else 0
    both(B, S, S, H, Hkv, dh, "bf16", window, sinks, 3 * short, k_len)


@pytest.mark.parametrize("dh", [64, 80, 128])
def test_two_groups_at_their_edges(dh):
    """Large scores; what no query sees is not used, whatever it holds; a NaN reaches the queries that see it, through whichever group's tiles."""
    B, S, H, window, sinks = 4, 700, 8, 400, 2
    r = route(B, S, S, H, H, dh, "bf16", window, sinks)
    assert (r.fwd_groups, r.dq_groups, r.fwd_splits, r.dq_splits) == (2, 2, 1, 1), forms(r)
    both(B, S, S, H, H, dh, "bf16", window, sinks, sharp=40.0)
    q, k, v, d = make(B, S, S, H, H, dh, "bf16")
    q_pos, k_len = torch.zeros(B, dtype=torch.int32), torch.tensor([700, 300, 90, 0], dtype=torch.int32)
    ref = orc.window_attention(q.double(), k.double(), v.double(), window, sinks, q_pos, k_len, d.double(), TD["bf16"])
    for b in range(B):
        k[b, k_len[b]:], v[b, k_len[b]:] = math.inf, math.nan
    check(run(*(t.to(DEV) for t in (q, k, v, d)), window, sinks, q_pos, k_len), ref)
    for at in (70, 150):
        k[0], v[0] = 1.0, 1.0
        v[0, at] = math.nan
        got = run(*(t.to(DEV) for t in (q, k, v, d)), window, sinks, q_pos, k_len)
        see = orc.window_mask(S, S, window, sinks, q_pos.long(), k_len.long())[0][:, at]
        for name in ("ctx", "dq"):
            assert torch.equal(torch.isnan(got[name][0]).any(-1).any(-1), see), name
        assert torch.isfinite(got["ctx"][1:]).all()


# Head widths above 128 (bf16): whole workgroups of rows, a wavefront's rows, cut and whole streams, sinks in parts, tokens, infinities where nobody looks.
@pytest.mark.parametrize("dh", [136, 192, 256])
@pytest.mark.parametrize("B,Sq,Sk,H,Hkv,window,sinks", [(2, 500, 500, 4, 2, 130, 3), (1, 1300, 1300, 1, 1, 2000, 0), (3, 700, 700, 30, 30, 100, 70), (2, 9, 600, 4, 2, 300, 2),
                                                        (5, 1, 900, 8, 2, 400, 4)])
def test_wide_heads(B, Sq, Sk, H, Hkv, window, sinks, dh):
    r = route(B, Sq, Sk, H, Hkv, dh, "bf16", window, sinks)
    assert (r.form, r.waves, r.fwd_groups, r.dq_groups) == (fax.FAX_ATTENTION_EDGE, 4 if Sq > 32 else 1, 1, 1), forms(r)
    if H == 1 or Sq == 1:
        assert r.fwd_splits > 1 and r.dq_splits > 1, forms(r)
    if H == 30:
        assert r.fwd_splits == 1 and r.dq_splits == 1 and r.key_splits == 1, forms(r)
    q, k, v, d = make(B, Sq, Sk, H, Hkv, dh, "bf16")
    k_len = (Sk - 60 * torch.arange(B)).to(torch.int32)
    q_pos = k_len - Sq
    ref = orc.window_attention(q.double(), k.double(), v.double(), window, sinks, q_pos, k_len, d.double(), TD["bf16"])
    for b in range(B):
        k[b, k_len[b]:], v[b, k_len[b]:] = math.inf, math.nan
    check(run(*(t.to(DEV) for t in (q, k, v, d)), window, sinks, q_pos, k_len), ref)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_sinks_alone_are_cut(dtype):
    B, S, H, window, sinks = 6, 1400, 8, 20, 5
    r = route(B, S, S, H, H, 64, dtype, window, sinks)
    assert r.sink_splits > 1 and r.key_splits == 1, forms(r)
    both(B, S, S, H, H, 64, dtype, window, sinks)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh", [64, 80, 128])
def test_single_tokens_of_many_caches(dh, dtype):
    B, Sk = 40, 1030
    k_len = torch.randint(0, Sk + 1, (B,), generator=torch.Generator().manual_seed(1), dtype=torch.int32)
    for H, Hkv in ((8, 8), (16, 2)):
        both(B, 1, Sk, H, Hkv, dh, dtype, 500, 4, k_len - 1, k_len, backward=False)


def test_scalar_kernels_take_the_rest():
    for dh, dtype in ((33, "bf16"), (132, "bf16"), (256, "f32"), (6, "f32")):
        assert route(1, 50, 50, 2, 2, dh, dtype, 10, 0).form == fax.FAX_ATTENTION_SCALAR
        both(1, 50, 50, 2, 2, dh, dtype, 10, 2)


def test_offsets_beyond_32_bits():
    """Rows, then heads and sequences so far apart that the last ones' places do not fit 32 bits, in elements or bytes."""
    dh, apart, Sk = 64, (1 << 24) - 8, 300
    room = torch.empty(Sk * apart, dtype=torch.bfloat16, device=DEV)  # 10 GB
    k, v = (room.as_strided((1, Sk, 1, dh), (0, apart, 0, 1), o) for o in (0, dh))
    q, kk, vv, d = make(1, Sk, Sk, 2, 1, dh, "bf16")
    k.copy_(kk)
    v.copy_(vv)
    assert fax.fax_window_attention_route(fax.window_dims(q, k, 100, 2)).form == fax.FAX_ATTENTION_MFMA
    dims = fax.window_dims(q.to(DEV), k, 100, 2)
    dk, dv = (room.as_strided((1, Sk, 1, dh), (0, apart, 0, 1), o) for o in (2 * dh, 3 * dh))
    n = fax.fax_window_attention_workspace_bytes(dims)
    ws = torch.empty(n, dtype=torch.uint8, device=DEV)
    qd, dd = q.to(DEV), d.to(DEV)
    ctx, dq, lse = torch.empty_like(qd), torch.empty_like(qd), torch.empty(1, 2, Sk, device=DEV)
    fax.fax_window_attention_fwd(dims, qd, k, v, None, None, ctx, lse, ws, n)
    fax.fax_window_attention_bwd(dims, qd, k, v, None, None, ctx, lse, dd, dq, dk, dv, ws, n)
    got = {"ctx": ctx, "lse": lse, "dq": dq, "dk": dk, "dv": dv}
    check({a: b.cpu().double() for a, b in got.items()},
          orc.window_attention(q.double(), kk.double(), vv.double(), 100, 2, None, None, d.double(), TD["bf16"]))
    far = (2 ** 31 + 64, dh, 7 * 10 ** 8, 1)
    k, v = (room.as_strided((2, 40, 3, dh), far, o) for o in (0, 40 * dh))
    q, kk, vv, d = make(2, 40, 40, 6, 3, dh, "bf16", seed=1)
    k.copy_(kk)
    v.copy_(vv)
    got = run(q.to(DEV), k, v, None, 9, 2, backward=False)
    check(got, orc.window_attention(q.double(), kk.double(), vv.double(), 9, 2, dtype=TD["bf16"]))


def test_more_rows_than_a_launch_has_threads():
    """The scalar kernels at one feature, a wavefront to a row: the last rows and keys as they are by themselves."""
    S, H, tail = (1 << 21) + 9, 33, 50
    gen = torch.Generator(device=DEV).manual_seed(0)
    q, k, v, d = (torch.randn(1, S, H, 1, generator=gen, device=DEV).bfloat16() for _ in range(4))

    def run_one(q, k, v, d):
        dims = fax.window_dims(q, k, 5)
        n = fax.fax_window_attention_workspace_bytes(dims)
        ws = torch.empty(n, dtype=torch.uint8, device=DEV)
        ctx, lse, dq, dk, dv = torch.empty_like(q), torch.empty(1, H, q.shape[1], device=DEV), torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
        fax.fax_window_attention_fwd(dims, q, k, v, None, None, ctx, lse, ws, n)
        fax.fax_window_attention_bwd(dims, q, k, v, None, None, ctx, lse, d, dq, dk, dv, ws, n)
        return ctx, lse.transpose(1, 2), dq, dk, dv

    full = run_one(q, k, v, d)
    part = run_one(*(t[:, -tail:].contiguous() for t in (q, k, v, d)))
    for name, a, b in zip(("ctx", "lse", "dq", "dk", "dv"), full, part):
        x, y = a[:, -tail + 8:].double(), b[:, 8:].double()
        # fp32 sums of at most 5 terms below 100 in another order (5 * 2^-24 * 100 = 3e-5), which may move a bf16 value to its neighbour (2^-7 of it)
        assert ((x - y).abs() <= 3e-5 + (y.abs() * 2 ** -7 if a.dtype == torch.bfloat16 else 0.0)).all(), name
        assert torch.isfinite(a).all(), name
