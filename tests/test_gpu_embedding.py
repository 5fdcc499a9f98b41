"""fax_embedding_fwd / _bwd against float64, at sizes where sorting, chunks and vectors have edges."""
import math

import pytest
import torch

import paper_2204_06514_amd as fax
from oracle import operators as orc
from helpers import DEV

pytestmark = pytest.mark.gpu
TD = {"f32": torch.float32, "bf16": torch.bfloat16}


def tokens_of(kind, N, V, gen):
    if kind == "same":
        return torch.full((N,), V - 1, dtype=torch.int32)
    if kind == "padding":
        t = torch.randint(-2, V + 2, (N,), generator=gen)
        return t.to(torch.int32)
    if kind == "none":
        return torch.full((N,), -1, dtype=torch.int32)
    if kind == "frequent":  # half of the positions hold one id
        t = torch.randint(0, V, (N,), generator=gen)
        return torch.where(torch.rand(N, generator=gen) < 0.5, torch.tensor(V // 2), t).to(torch.int32)
    return torch.randint(0, V, (N,), generator=gen).to(torch.int32)


SIZES = [(1, 1, 1), (1, 7, 8), (5, 3, 33), (31, 1000, 64), (32, 2, 64), (33, 5, 129), (64, 1, 256), (127, 50304, 16), (1000, 300, 2056),
         (1024, 511, 24), (1025, 512, 24), (4097, 513, 40), (5000, 70000, 12), (20000, 37, 72), (40000, 300000, 4)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,V,D", SIZES)
def test_lookup(N, V, D, dtype):
    gen = torch.Generator().manual_seed(N + V + D)
    t = tokens_of("padding", N, V, gen)
    table = torch.randn(V, D, generator=gen).to(TD[dtype])
    scale = math.sqrt(D)
    out = torch.full((N, D), 7.0, dtype=TD[dtype], device=DEV)
    fax.fax_embedding_fwd(fax.dtype_code(out), N, V, D, t.to(DEV), table.to(DEV), scale, out)
    ref = orc.embedding(t, table.double(), torch.tensor(scale, dtype=torch.float32).double())
    # the scale is an fp32 argument; one product in fp32, one rounding to the type
    bound = ref.abs() * ((0 if dtype == "f32" else orc.U) + orc.half_step(TD[dtype])) * 1.01
    assert ((out.cpu().double() - ref).abs() <= bound).all()


def gradient(t, dout, V, scale, before=None, ws=None):
    N, D = dout.shape
    g = before.clone().to(DEV) if before is not None else torch.full((V, D), 5.0, device=DEV)
    need = fax.fax_embedding_bwd_workspace_bytes(N, V, D)
    ws = torch.empty(need, dtype=torch.uint8, device=DEV) if ws is None else ws
    assert ws.numel() >= need
    fax.fax_embedding_bwd(fax.dtype_code(dout), N, V, D, t.to(DEV), dout.to(DEV), scale, g, before is not None, ws, ws.numel())
    return g.cpu()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["uniform", "same", "padding", "none", "frequent"])
@pytest.mark.parametrize("N,V,D", SIZES)
def test_gradient(N, V, D, kind, dtype):
    if V == 300000 and kind != "uniform":
        pytest.skip("one kind of tokens is enough for a large table")
    gen = torch.Generator().manual_seed(N + V + D)
    t = tokens_of(kind, N, V, gen)
    dout = torch.randn(N, D, generator=gen).to(TD[dtype])
    scale = 0.375
    for before in (None, torch.randn(V, D, generator=gen)):
        got = gradient(t, dout, V, scale, before)
        ref, bound = orc.embedding_grad(t, dout.double(), V, scale, None if before is None else before.double())
        assert ((got.double() - ref).abs() <= bound).all()
        untouched = torch.ones(V, dtype=torch.bool)
        untouched[t[(t >= 0) & (t < V)].long()] = False
        assert torch.equal(got[untouched], torch.zeros_like(got[untouched]) if before is None else before[untouched])


# Several positions to a wavefront, rows in pieces, rows without a position written beside the sort.
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["uniform", "padding", "frequent", "none"])
@pytest.mark.parametrize("N,V,D", [(70000, 900, 20), (66000, 30000, 260), (3000, 20000, 516), (5001, 700, 33), (4500, 66000, 65)])
def test_gradient_in_pieces(N, V, D, kind, dtype):
    test_gradient(N, V, D, kind, dtype)


def test_gradient_repeats_its_bits_and_leaves_its_workspace_usable():
    gen = torch.Generator().manual_seed(3)
    N, V, D = 30000, 1000, 64
    t = tokens_of("frequent", N, V, gen)
    dout = torch.randn(N, D, generator=gen).to(torch.bfloat16)
    ws = torch.full((fax.fax_embedding_bwd_workspace_bytes(N, V, D),), 255, dtype=torch.uint8, device=DEV)
    first = gradient(t, dout, V, 1.0, ws=ws)
    small = gradient(t[:777], dout[:777], V, 1.0, ws=ws)  # on what the first call left behind
    assert torch.equal(first, gradient(t, dout, V, 1.0, ws=ws))
    assert torch.equal(small, gradient(t[:777], dout[:777], V, 1.0))


def test_a_nan_reaches_its_own_row_alone():
    N, V, D = 300, 40, 16
    gen = torch.Generator().manual_seed(4)
    t = tokens_of("uniform", N, V, gen)
    dout = torch.randn(N, D, generator=gen)
    dout[17] = math.nan
    g = gradient(t, dout, V, 1.0)
    bad = torch.isnan(g).any(1)
    assert bad[t[17]] and int(bad.sum()) == 1
    t[17] = -1  # padding: not read into any sum
    assert torch.isfinite(gradient(t, dout, V, 1.0)).all()


def test_no_positions():
    g = torch.full((5, 8), 3.0, device=DEV)
    fax.fax_embedding_bwd(fax.FAX_F32, 0, 5, 8, None, None, 1.0, g, 1, None, 0)
    assert (g == 3.0).all()
    fax.fax_embedding_bwd(fax.FAX_F32, 0, 5, 8, None, None, 1.0, g, 0, None, 0)
    assert (g == 0.0).all()


@pytest.mark.parametrize("N,V", [(3, (1 << 26) + 7), (600, (1 << 28) + 5), (600, (1 << 30) - 3)])
def test_more_rows_than_a_launch_has_threads(N, V):
    """A table of one feature: the workgroups of all its rows do not fit one dimension of a launch."""
    gen = torch.Generator().manual_seed(N)
    t = torch.randint(0, V, (N,), generator=gen).to(torch.int32)
    t[0], t[1], t[2] = V - 1, 0, V
    dout = torch.randint(1, 100, (N, 1), generator=gen).to(torch.float32)
    g = torch.full((V, 1), 7.0, device=DEV)
    n = fax.fax_embedding_bwd_workspace_bytes(N, V, 1)
    ws = torch.empty(n, dtype=torch.uint8, device=DEV)
    fax.fax_embedding_bwd(fax.FAX_F32, N, V, 1, t.to(DEV), dout.to(DEV), 0.5, g, 0, ws, n)
    at, where = torch.unique(t[t < V].long(), return_inverse=True)
    sums = torch.zeros(len(at), dtype=torch.float64).index_add_(0, where, 0.5 * dout[t < V, 0].double())  # small halves: exact
    assert (g[at.to(DEV), 0].cpu().double() == sums).all()
    g[at.to(DEV)] = 0
    assert torch.count_nonzero(g).item() == 0
