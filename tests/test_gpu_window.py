"""fax_window_attention_fwd / _bwd against float64 with derived bounds: windows, sinks, grouped heads, head widths, positions and lengths that
leave rows empty, strides, values in masked places."""
import math

import pytest
import torch

import paper_2204_06514_amd as fax
from oracle import operators as orc
from helpers import DEV

pytestmark = pytest.mark.gpu
TD = {"f32": torch.float32, "bf16": torch.bfloat16}


def make(B, Sq, Sk, H, Hkv, dh, dtype, seed=0, sharp=1.5):
    gen = torch.Generator().manual_seed(seed + Sq + 3 * Sk + 7 * dh)
    r = lambda S, h, f: (f * torch.randn(B, S, h, dh, generator=gen)).to(TD[dtype])  # noqa: E731
    return r(Sq, H, sharp), r(Sk, Hkv, 1.0), r(Sk, Hkv, 1.0), r(Sq, H, 1.0)


def run(q, k, v, dctx, window, sinks, q_pos=None, k_len=None, ctx_like=None, backward=True, lse=True):
    """Everything on the device in the layout that it has; -> dict of CPU float64."""
    to = lambda t: None if t is None else t.to(DEV)  # noqa: E731
    B, Sq, H, dh = q.shape
    ctx = torch.full((B, Sq, H, dh), 9.0, dtype=q.dtype, device=DEV) if ctx_like is None else ctx_like
    d = fax.window_dims(q, k, window, sinks, ctx if ctx_like is not None else None)
    n = fax.fax_window_attention_workspace_bytes(d)
    ws = torch.full((n + 256,), 255, dtype=torch.uint8, device=DEV)
    L = torch.full((B, H, Sq), 9.0, device=DEV) if lse else None
    q_pos, k_len = to(q_pos), to(k_len)
    fax.fax_window_attention_fwd(d, q, k, v, q_pos, k_len, ctx, L, ws, n)
    out = {"ctx": ctx}
    if lse:
        out["lse"] = L
    if backward:
        # full_like would lay views out densely; each in a buffer of its own, as far as the view reaches
        dq, dk, dv = (torch.full((1 + sum((n - 1) * s for n, s in zip(t.shape, t.stride())),), 9.0, dtype=t.dtype, device=DEV)
                      .as_strided(t.shape, t.stride()) for t in (q, k, v))
        fax.fax_window_attention_bwd(d, q, k, v, q_pos, k_len, ctx, L, dctx, dq, dk, dv, ws, n)
        out.update(dq=dq, dk=dk, dv=dv)
    torch.cuda.synchronize()
    assert (ws[n:] == 255).all()
    return {a: b.cpu().double() for a, b in out.items()}


def check(got, ref):
    for name, x in got.items():
        y, b = ref[name], ref["bound"][name]
        same = torch.isinf(y) & (x == y)
        off = torch.where(same, 0.0, (x - y).abs())
        assert (off <= b).all(), (name, (off / b).max().item(), (off > b).nonzero()[:4].tolist())


def both(B, Sq, Sk, H, Hkv, dh, dtype, window, sinks, q_pos=None, k_len=None, backward=True, seed=0, sharp=1.5):
    q, k, v, d = make(B, Sq, Sk, H, Hkv, dh, dtype, seed, sharp)
    got = run(*(t.to(DEV) for t in (q, k, v, d)), window, sinks, q_pos, k_len, backward=backward)
    ref = orc.window_attention(q.double(), k.double(), v.double(), window, sinks, q_pos, k_len, d.double() if backward else None, TD[dtype])
    check(got, ref)
    return got


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh", [1, 7, 8, 20, 32, 40, 64, 72, 80, 96, 100, 128, 136, 256])
def test_head_widths(dh, dtype):
    both(2, 150, 150, 2, 1, dh, dtype, 40, 3)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("S", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 257, 513])
@pytest.mark.parametrize("dh", [64, 128])
def test_lengths(S, dh, dtype):
    both(1, S, S, 2, 2, dh, dtype, 50, 4)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (2, 63), (31, 64), (32, 65), (63, 0), (64, 1), (65, 130), (100, 0), (128, 4), (129, 300), (400, 400), (10000, 0), (2 ** 31 - 1, 2 ** 31 - 1)])
def test_windows_and_sinks(window, sinks, dtype):
    both(1, 333, 333, 2, 1, 64, dtype, window, sinks)
    both(1, 333, 333, 1, 1, 128, dtype, window, sinks)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,Hkv", [(1, 1), (3, 1), (6, 2), (8, 1), (8, 8), (15, 5), (40, 1)])
def test_grouped_heads(H, Hkv, dtype):
    both(2, 140, 140, H, Hkv, 64, dtype, 33, 2)
    both(1, 70, 70, H, Hkv, 80, dtype, 33, 2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Sq,Sk", [(1, 1), (1, 2), (1, 63), (1, 64), (1, 1000), (1, 3001), (2, 700), (5, 64), (33, 900), (130, 1030), (70, 40)])
@pytest.mark.parametrize("dh", [64, 128])
def test_chunks_and_single_tokens(Sq, Sk, dh, dtype):
    for window, sinks in ((1, 1), (300, 4), (5000, 0)):
        both(2, Sq, Sk, 4, 2, dh, dtype, window, sinks)                     # the last Sq positions


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh", [64, 80, 128])
def test_positions_and_lengths_of_sequences(dh, dtype):
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32)  # noqa: E731
    # a padded batch for training, one of its sequences empty; lengths outside the room
    both(5, 200, 200, 2, 1, dh, dtype, 40, 3, i32(0, 0, 0, 0, 0), i32(200, 77, 0, -5, 1000))
    # tokens over caches of different length; queries before the first key, far behind the last, at the ends of the type
    for Sq in (1, 3, 140):
        both(6, Sq, 300, 4, 2, dh, dtype, 40, 3, i32(299, 100, -2, 900, 2 ** 31 - 1, -2 ** 31), i32(300, 101, 50, 300, 120, 30))
    both(2, 100, 260, 2, 2, dh, dtype, 40, 0, i32(130, 300), i32(200, 260))  # without sinks: the second sees nothing


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_counts(dtype):
    """All scores equal: ctx holds how many keys of each residue a query sees, over how many it sees at all.  Sums are whole numbers, so
    only the quotient and its rounding are off: one key too many or too few is far outside."""
    B, S, dh = 1, 500, 64
    q = torch.zeros(B, S, 2, dh, dtype=TD[dtype])
    k = torch.randn(B, S, 1, dh).to(TD[dtype])
    v = torch.nn.functional.one_hot(torch.arange(S) % dh, dh).to(TD[dtype]).view(B, S, 1, dh)
    for window, sinks in ((1, 0), (37, 5), (64, 0), (200, 70), (499, 1)):
        got = run(*(t.to(DEV) for t in (q, k, v, q)), window, sinks, backward=False)
        see = orc.window_mask(S, S, window, sinks, torch.zeros(B, dtype=torch.long), torch.full((B,), S))
        ref = see.double() @ v[:, :, 0].double() / see.sum(-1, keepdim=True)
        assert ((got["ctx"] - ref[:, :, None]).abs() <= ref[:, :, None] * (orc.half_step(TD[dtype]) + 3 * orc.U)).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strides(dtype):
    """Views into a packed projection, caches with heads outside of rows, rows that start on no 16 bytes, one key head for several sequences."""
    B, S, H, Hkv, dh = 2, 130, 4, 2, 64
    q, k, v, d = make(B, S, S, H, Hkv, dh, dtype)
    ref = orc.window_attention(q.double(), k.double(), v.double(), 30, 2, None, None, d.double(), TD[dtype])
    packed = torch.cat([q, k, v], 2).to(DEV)
    check(run(*packed.split([H, Hkv, Hkv], 2), d.to(DEV), 30, 2), ref)
    outside = [t.to(DEV).permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3) for t in (q, k, v, d)]  # [B, heads, S, dh] in memory
    check(run(*outside, 30, 2, ctx_like=torch.empty_like(outside[0])), ref)
    odd = torch.zeros(B, S, H + 2 * Hkv, dh + 1, dtype=TD[dtype], device=DEV)[..., 1:]
    odd.copy_(packed)
    check(run(*odd.split([H, Hkv, Hkv], 2), d.to(DEV), 30, 2), ref)  # rows of 65 elements
    wide = torch.zeros(B, 3 * S, H + 2 * Hkv, dh, dtype=TD[dtype], device=DEV)[:, ::3]
    wide.copy_(packed)
    check(run(*wide.split([H, Hkv, Hkv], 2), d.to(DEV), 30, 2), ref)
    shared = [t[:1].expand(B, -1, -1, -1) for t in (k, v)]
    ref = orc.window_attention(q.double(), *(t.double() for t in shared), 30, 2, dtype=TD[dtype])
    check(run(q.to(DEV), *(t[:1].to(DEV).expand(B, -1, -1, -1) for t in (k, v)), None, 30, 2, backward=False), ref)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh", [64, 80, 128, 20])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf, 3e38])
def test_values_in_masked_places(bad, dh, dtype):
    """What no query sees (behind the last key of a sequence) is not used; what some see spoils those alone."""
    if dtype == "bf16" and bad == 3e38:
        bad = torch.finfo(torch.bfloat16).max
    B, S, H, Hkv = 2, 200, 4, 2
    q, k, v, d = make(B, S, S, H, Hkv, dh, dtype)
    q_pos, k_len = torch.zeros(B, dtype=torch.int32), torch.tensor([200, 90], dtype=torch.int32)
    ref = orc.window_attention(q.double(), k.double(), v.double(), 30, 2, q_pos, k_len, d.double(), TD[dtype])
    clean = {n: t.clone() for n, t in ref.items() if n != "bound"}
    k[1, 90:], v[1, 90:] = bad, bad                       # a cache's rows that hold nothing yet
    q[1, 130:], d[1, 130:] = bad, bad                     # queries behind the last key's window still see the sinks: see below
    got = run(*(t.to(DEV) for t in (q, k, v, d)), 30, 2, q_pos, k_len)
    rows = torch.ones(B, S, dtype=torch.bool)
    rows[1, 130:] = False
    for name in ("ctx", "dq"):
        off = (got[name] - clean[name]).abs()[rows]
        assert (off <= ref["bound"][name][rows]).all(), name
    off = (got["lse"] - clean["lse"]).abs().permute(0, 2, 1)[rows]
    assert (off <= ref["bound"]["lse"].permute(0, 2, 1)[rows]).all()
    keys = torch.ones(B, S, dtype=torch.bool)
    keys[1, :2] = False                                   # the sinks that those queries see
    for name in ("dk", "dv"):
        off = (got[name] - clean[name]).abs()[keys]
        assert (off <= ref["bound"][name][keys]).all(), name


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh", [64, 128])
def test_a_nan_reaches_the_queries_that_see_it(dh, dtype):
    S, window, sinks, at = 300, 40, 3, 150
    q, k, v, d = make(1, S, S, 2, 1, dh, dtype)
    v[0, at] = math.nan
    got = run(*(t.to(DEV) for t in (q, k, v, d)), window, sinks)
    see = orc.window_mask(S, S, window, sinks, torch.zeros(1, dtype=torch.long), torch.tensor([S]))[0]
    assert torch.equal(torch.isnan(got["ctx"]).all(-1)[0].any(-1), see[:, at])
    assert torch.equal(torch.isnan(got["ctx"]).any(-1)[0].any(-1), see[:, at])
    assert torch.isfinite(got["lse"]).all()
    v[0, at] = 1.0
    ref = orc.window_attention(q.double(), k.double(), v.double(), window, sinks, None, None, d.double(), TD[dtype])
    ok = ~see[:, at]
    for name in ("ctx", "dq"):
        assert ((got[name] - ref[name]).abs() <= ref["bound"][name])[0][ok].all(), name
    far = ~(see[see[:, at]].any(0))                       # keys that none of the spoiled queries sees
    for name in ("dk", "dv"):
        assert ((got[name] - ref[name]).abs() <= ref["bound"][name])[0][far].all(), name


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_scores(dtype):
    """Scores of some hundred: one key takes a row, and none overflows."""
    both(1, 200, 200, 2, 1, 64, dtype, 60, 2, sharp=40.0)


def test_lse_may_be_left_out_and_bits_repeat():
    q, k, v, d = (t.to(DEV) for t in make(2, 300, 300, 4, 2, 128, "bf16"))
    a, b = run(q, k, v, d, 100, 4), run(q, k, v, d, 100, 4)
    assert all(torch.equal(a[n], b[n]) for n in a)
    c = run(q, k, v, d, 100, 4, backward=False, lse=False)
    assert torch.equal(a["ctx"], c["ctx"])
