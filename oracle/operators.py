"""Plain float64 definitions (torch, CPU) of the operators for programs that drive their own layers: attention in a window with sinks,
the embedding and its gradient, AdamW with moments of 8 bits.  Each comes with the bound on an implementation's rounding errors that
follows from its arithmetic: U = 2^-24 per fp32 operation, `half` = half a step of the type that is stored (2^-24 for fp32, 2^-8 for
bf16)."""
import math

import torch

U = 2.0 ** -24


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


# ---- attention in a window --------------------------------------------------------------------------
def window_mask(Sq, Sk, window, sinks, q_pos, k_len):
    """[B, Sq, Sk]: whether a query sees a key."""
    p = (q_pos[:, None] + torch.arange(Sq))[:, :, None]
    j = torch.arange(Sk)[None, None]
    return (j < k_len.clamp(0, Sk)[:, None, None]) & (j <= p) & ((j > p - window) | (j < sinks))


def window_attention(q, k, v, window, sinks, q_pos=None, k_len=None, dctx=None, dtype=torch.float32):
    """q [B, Sq, H, dh], k, v [B, Sk, Hkv, dh] (float64 holding values of `dtype`) -> dict of ctx, lse, with dctx of dq, dk, dv, and
    under "bound" how far an implementation that rounds as stated may be off, element by element: scores, exponentials and sums in
    fp32, probabilities and dS in `dtype` as factors of the second products, ctx in `dtype` in delta."""
    B, Sq, H, dh = q.shape
    Sk, Hkv = k.shape[1:3]
    G = H // Hkv
    q_pos = torch.full((B,), Sk - Sq) if q_pos is None else q_pos.long()
    k_len = torch.full((B,), Sk) if k_len is None else k_len.long()
    see = window_mask(Sq, Sk, window, sinks, q_pos, k_len)[:, None]
    scale = 1.0 / math.sqrt(dh)
    Q = q.permute(0, 2, 1, 3)
    K, V = (t.permute(0, 2, 1, 3).repeat_interleave(G, 1) for t in (k, v))
    any_key = see.any(2, keepdim=True).permute(0, 1, 3, 2)                 # keys some query sees: others may hold anything
    K, V = torch.where(any_key, K, 0.0), torch.where(any_key, V, 0.0)
    s = torch.where(see, Q @ K.transpose(-1, -2) * scale, -math.inf)
    lse = torch.logsumexp(s, -1)
    empty = torch.isinf(lse)[..., None]
    P = torch.where(empty, 0.0, torch.exp(s - torch.where(empty, 0.0, lse[..., None])))
    ctx = P @ V
    half = half_step(dtype)
    # a score is dh multiply-adds and a scaling, the difference to the reference one more, relative to the scores themselves
    ds = torch.where(see, (Q.abs() @ K.abs().transpose(-1, -2)) * scale * (dh + 3) * U + 4 * U * s.abs().nan_to_num(0.0, 0.0, 0.0), 0.0).amax(-1, keepdim=True)
    n = see.sum(-1, keepdim=True)
    rel = 2 * ds + (n + 12) * U                                           # of a probability: numerator and denominator
    back = lambda t: t.permute(0, 2, 1, 3)  # noqa: E731
    PV = P @ V.abs()
    e_ctx = (rel + (half if dtype != torch.float32 else 0.0)) * PV + half * ctx.abs()
    out = {"ctx": back(ctx), "lse": lse}
    bound = {"ctx": back(e_ctx), "lse": torch.where(empty[..., 0], 0.0, (ds + (n + 8) * U + 2 * U * lse.abs()[..., None])[..., 0].nan_to_num(0.0, 0.0, 0.0))}
    if dctx is not None:
        dO = dctx.permute(0, 2, 1, 3)
        dP = dO @ V.transpose(-1, -2)
        delta = (dO * ctx).sum(-1, keepdim=True)
        dS = P * (dP - delta)
        fold = lambda t: t.reshape(B, Hkv, G, Sk, dh).sum(2).permute(0, 2, 1, 3)  # noqa: E731
        out["dq"] = back(dS @ K * scale)
        out["dk"], out["dv"] = fold(dS.transpose(-1, -2) @ Q * scale), fold(P.transpose(-1, -2) @ dO)
        e_dP = (dh + 2) * U * (dO.abs() @ V.abs().transpose(-1, -2))
        e_delta = (dO.abs() * (e_ctx + dh * U * ctx.abs())).sum(-1, keepdim=True)
        e_lse = bound["lse"][..., None]
        low = half if dtype != torch.float32 else 0.0                     # the factor's own rounding
        e_P = P * (ds + e_lse + 8 * U + low)
        e_dS = P * (e_dP + e_delta) + dS.abs() * (ds + e_lse + 10 * U + low)
        terms = (H // Hkv) * Sq
        bound["dq"] = back((e_dS + (n + 4) * U * dS.abs()) @ K.abs() * scale) + half * out["dq"].abs()
        bound["dk"] = fold((e_dS + (terms + 4) * U * dS.abs()).transpose(-1, -2) @ Q.abs() * scale) + half * out["dk"].abs()
        bound["dv"] = fold((e_P + (terms + 4) * U * P).transpose(-1, -2) @ dO.abs()) + half * out["dv"].abs()
    out["bound"] = {k: b * 1.01 + 1e-30 for k, b in bound.items()}        # 1 %: products of the errors
    return out


# ---- embedding --------------------------------------------------------------------------------------
def embedding(tokens, table, scale):
    known = (tokens >= 0) & (tokens < table.shape[0])
    return torch.where(known[:, None], table[torch.where(known, tokens, 0).long()] * scale, 0.0)


def embedding_grad(tokens, dout, V, scale, before=None):
    """-> (gradient, bound): sums of fp32 numbers in any order, one scaling, one addition to what was there."""
    known = (tokens >= 0) & (tokens < V)
    ids = tokens[known].long()
    rows = dout[known]
    g = torch.zeros(V, dout.shape[1], dtype=torch.float64).index_add_(0, ids, rows) * scale
    mags = torch.zeros_like(g).index_add_(0, ids, rows.abs()) * abs(scale)
    n = torch.bincount(ids, minlength=V).double()[:, None]
    if before is not None:
        g = g + before
    return g, ((n + 2) * mags + 2 * g.abs()) * U * 1.01


# ---- AdamW ------------------------------------------------------------------------------------------
BLOCK, E4M3_MAX = 256, 448.0


def _hash(x):
    x &= 0xFFFFFFFF
    x ^= x >> 16
    x = x * 0x9E3779B1 & 0xFFFFFFFF
    x ^= x >> 15
    x = x * 0x2545F491 & 0xFFFFFFFF
    return x ^ x >> 16


def random20(seed, step, tensor, n):
    """The random bits of a tensor's elements, as fractions in [0, 1)."""
    key = _hash(_hash(seed + step * 0x9E3779B1) + tensor * 0x9E3779B1)
    x = (torch.arange(n, dtype=torch.int64) * 0x9E3779B1 + key) & 0xFFFFFFFF
    x = ((x ^ (x >> 16)) * 0x9E3779B1) & 0xFFFFFFFF
    x = ((x ^ (x >> 15)) * 0x2545F491) & 0xFFFFFFFF
    return ((x ^ (x >> 16)) >> 12).double() / 2.0 ** 20


def _step_of(x):
    """Distance of e4m3 numbers around x."""
    return torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3.0)


def e4m3_nearest(x):
    s = _step_of(x)
    return (torch.round(x / s) * s).clamp(-E4M3_MAX, E4M3_MAX)


def e4m3_random(x, u):
    s = _step_of(x)
    return torch.where(x > 0, (torch.floor(x / s + u) * s).clamp(2.0 ** -9, E4M3_MAX), 0.0)


def per_block(x, n):
    return x.repeat_interleave(BLOCK)[:n]


def block_max(x):
    pad = torch.zeros(-len(x) % BLOCK, dtype=x.dtype)
    return torch.cat([x.abs(), pad]).view(-1, BLOCK).amax(1)


def adamw(p, m, v, g, hp, step, decay=True):
    """-> new p, m, v and how far fp32 arithmetic may be off each: five roundings in a moment and its factors, twelve in the update."""
    lr, b1, b2, eps, wd = hp
    m1 = b1 * m + (1 - b1) * g
    v1 = b2 * v + (1 - b2) * g * g
    e_m = 5 * U * ((b1 * m).abs() + ((1 - b1) * g).abs())
    e_v = 6 * U * v1
    root = torch.sqrt(v1 / (1 - b2 ** step)) + eps
    up = m1 / (1 - b1 ** step) / root
    p1 = p * (1 - lr * wd if decay else 1.0) - lr * up
    e_p = 3 * U * p.abs() + lr * (e_m / (1 - b1 ** step) / root + 12 * U * up.abs())
    return p1, m1, v1, e_p * 1.01, e_m * 1.01, e_v * 1.01
