"""The operators for programs that drive their own layers, as a list of measurable cases: the way into a model (embedding lookup and its
gradient), attention in a sliding window with sinks (a training pass, a chunk of a prompt, single tokens), and the update of many tensors.

listed() names twelve of them, draw() gives others of the same ranges.  run() computes a case through the library where `own` is set,
and in elementary torch operations otherwise; exact() says in 64 bits what comes out.
"""
import math

import torch

own = False

DEVICE = "cuda"
EMBEDDING, WINDOW, ADAMW = "embedding", "window", "adamw"
# Hyper-parameters of a run late in its schedule, so that a pass repeated on one state leaves it the distribution it started with.
LR, BETA1, BETA2, EPS, WD, FIRST_STEP = 1e-5, 0.9, 0.999, 1e-8, 0.01, 1000
BLOCK = 256          # elements of an 8-bit state that share a scale
E4M3_MAX = 448.0
M_FLOOR = 2.0 ** -100  # a block whose first moments are all smaller is kept as zeros


def listed():
    return [
        # the gradient of a small fp32 embedding added to what is there (unit tests, numerics studies), with padding ids
        dict(name="embedding_grad_small", op=EMBEDDING, what="grad", N=128, V=1003, D=128, dtype="f32", scale=1.0, accumulate=True, pad=True),
        # the way into the 124M-parameter model at batch 32 x 2048, rows scaled by sqrt(D)
        dict(name="embedding_lookup_124m", op=EMBEDDING, what="lookup", N=65536, V=50304, D=768, dtype="bf16", scale=math.sqrt(768.0), pad=False),
        # and the gradient of its table
        dict(name="embedding_grad_124m", op=EMBEDDING, what="grad", N=65536, V=50304, D=768, dtype="bf16", scale=math.sqrt(768.0), accumulate=False, pad=False),
        # the tiny fp32 configuration with a window: launches and latency are all there is
        dict(name="window_train_tiny", op=WINDOW, what="train", B=2, Sq=64, Sk=64, H=4, Hkv=4, dh=32, window=16, sinks=2, dtype="f32", padded=False),
        # a padded batch of texts, head width 80, three query heads to a key head, nothing a multiple of anything large
        dict(name="window_train_ragged", op=WINDOW, what="train", B=3, Sq=1000, Sk=1000, H=15, Hkv=5, dh=80, window=300, sinks=3, dtype="bf16", padded=True),
        # a local layer of the 124M-parameter model
        dict(name="window_train_124m", op=WINDOW, what="train", B=8, Sq=2048, Sk=2048, H=12, Hkv=12, dh=64, window=512, sinks=4, dtype="bf16", padded=False),
        # a local layer of the 4096-wide block on one long text, four query heads to a key head
        dict(name="window_train_long", op=WINDOW, what="train", B=1, Sq=8192, Sk=8192, H=32, Hkv=8, dh=128, window=1024, sinks=4, dtype="bf16", padded=False),
        # a chunk of the prompts over what is in their caches already
        dict(name="window_prompt_chunk", op=WINDOW, what="forward", B=4, Sq=512, Sk=8192, H=16, Hkv=4, dh=128, window=2048, sinks=4, dtype="bf16", padded=True),
        # single tokens over long caches
        dict(name="window_token", op=WINDOW, what="forward", B=8, Sq=1, Sk=16384, H=32, Hkv=8, dh=128, window=4096, sinks=4, dtype="bf16", padded=True),
        # a few tensors of odd sizes (adapters, a probe), bf16 gradients, states in 8 bits
        dict(name="adamw_ragged_8bit", op=ADAMW, layers=2, D=333, Hd=320, F=1001, V=0, state=8, grad="bf16", lowp=True),
        # the 148 tensors of the 124M-parameter model, states in 32 bits and in 8
        dict(name="adamw_124m_32bit", op=ADAMW, layers=12, D=768, Hd=768, F=3072, V=50304, state=32, grad="f32", lowp=True),
        dict(name="adamw_124m_8bit", op=ADAMW, layers=12, D=768, Hd=768, F=3072, V=50304, state=8, grad="f32", lowp=True),
    ]


# ---- drawn cases ------------------------------------------------------------------------------------
def _spread(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw_embedding(rng):
    what = rng.choice(["lookup", "grad", "grad"])
    c = dict(op=EMBEDDING, what=what, N=_spread(rng, 1, 65536), V=_spread(rng, 100, 51200), D=8 * _spread(rng, 8, 256) if rng.random() < 0.6 else _spread(rng, 33, 2048),
             dtype=rng.choice(["bf16", "bf16", "f32"]), pad=rng.random() < 0.3)
    while c["N"] * c["D"] > 65536 * 768:
        c["N"] = (c["N"] + 1) // 2
    while c["V"] * c["D"] > 50304 * 768:
        c["V"] = c["V"] * 3 // 4
    c["scale"] = rng.choice([1.0, math.sqrt(c["D"])])
    if what == "grad":
        c["accumulate"] = rng.random() < 0.5
    return c


def _draw_window(rng):
    what = rng.choice(["train", "train", "train", "forward", "forward"])
    Hkv = _spread(rng, 1, 12)
    c = dict(op=WINDOW, what=what, B=_spread(rng, 1, 8), H=Hkv * rng.choice([1, 1, 2, 3, 4, 8]), Hkv=Hkv, dh=rng.choice([32, 64, 64, 80, 96, 128, 128]),
             dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]), sinks=rng.choice([0, 1, 4, 4, 64, 100]), padded=rng.random() < 0.4)
    if what == "train":
        c["Sq"] = c["Sk"] = _spread(rng, 17, 8192) if rng.random() < 0.6 else 128 * _spread(rng, 1, 32)
    else:
        c["Sk"] = _spread(rng, 64, 16384)
        c["Sq"] = rng.choice([1, 1, 1, 2, _spread(rng, 3, 512)])
        c["Sq"] = min(c["Sq"], c["Sk"])
    c["window"] = _spread(rng, 8, 4096)
    most = 1.5e9 if c["dtype"] == "bf16" else 3e8  # pairs of the whole square: what the plain form computes
    while c["B"] > 1 and c["B"] * c["H"] * c["Sq"] * c["Sk"] > most:
        c["B"] -= 1
    while c["B"] * c["H"] * c["Sq"] * c["Sk"] > most:
        c["Sk"] = c["Sk"] * 3 // 4
        c["Sq"] = c["Sk"] if what == "train" else min(c["Sq"], c["Sk"])
    return c


def _draw_adamw(rng):
    D = _spread(rng, 32, 1024)
    c = dict(op=ADAMW, layers=_spread(rng, 1, 16), D=D, Hd=rng.choice([D, _spread(rng, 32, 1024)]), F=_spread(rng, 64, 4096), V=rng.choice([0, _spread(rng, 100, 51200)]),
             state=rng.choice([8, 8, 32]), grad=rng.choice(["f32", "f32", "bf16"]), lowp=rng.random() < 0.7)
    while sum(math.prod(s) for s, _ in _tensors(c)) > 120_000_000:
        if c["layers"] > 1:
            c["layers"] -= 1
        else:
            c["V"] //= 2
    return c


def draw(rng):
    return rng.choice([_draw_embedding, _draw_window, _draw_window, _draw_adamw])(rng)


# ---- what the parts have in common ------------------------------------------------------------------
class _State:
    pass


def _torch_dtype(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _fax():
    import paper_2204_06514_amd as fax
    return fax


def _workspace(n):
    return torch.empty(max(n, 16), dtype=torch.uint8, device=DEVICE)


# ---- embedding --------------------------------------------------------------------------------------
def _embedding_inputs(c, gen):
    """Ids as a text has them (the share of the r-th most frequent one falls like 1 / r), a table of N(0, 0.02^2), upstream gradients."""
    td = _torch_dtype(c["dtype"])
    N, V, D = c["N"], c["V"], c["D"]
    u = torch.rand(N, generator=gen, device=DEVICE, dtype=torch.float64)
    rank = torch.exp(u * math.log(V + 1.0)).long().clamp(1, V) - 1
    tokens = torch.randperm(V, generator=gen, device=DEVICE)[rank].to(torch.int32)
    if c["pad"]:
        tokens[N - N // 8:] = -1
    i = dict(tokens=tokens)
    if c["what"] == "lookup":
        i["table"] = (0.02 * torch.randn(V, D, generator=gen, device=DEVICE)).to(td)
    else:
        i["dout"] = (1e-3 * torch.randn(N, D, generator=gen, device=DEVICE)).to(td)
        i["before"] = 1e-3 * torch.randn(V, D, generator=gen, device=DEVICE) if c["accumulate"] else None
    return i


def _prepare_embedding(c, gen, s):
    i = _embedding_inputs(c, gen)
    s.tokens, s.td = i["tokens"], _torch_dtype(c["dtype"])
    if c["what"] == "lookup":
        s.table = i["table"]
        s.out = torch.empty(c["N"], c["D"], dtype=s.td, device=DEVICE)
        return
    s.dout, s.dtable = i["dout"], i["before"] if c["accumulate"] else torch.empty(c["V"], c["D"], device=DEVICE)
    if own:
        s.ws_bytes = _fax().fax_embedding_bwd_workspace_bytes(c["N"], c["V"], c["D"])
        s.ws = _workspace(s.ws_bytes)


def _run_embedding(s):
    c = s.case
    if own:
        fax = _fax()
        code = fax.dtype_code(s.td)
        if c["what"] == "lookup":
            fax.fax_embedding_fwd(code, c["N"], c["V"], c["D"], s.tokens, s.table, c["scale"], s.out)
            return {"out": s.out}
        fax.fax_embedding_bwd(code, c["N"], c["V"], c["D"], s.tokens, s.dout, c["scale"], s.dtable, c["accumulate"], s.ws, s.ws_bytes)
        return {"dtable": s.dtable}
    known = (s.tokens >= 0) & (s.tokens < c["V"])
    ids = torch.where(known, s.tokens, 0).long()
    if c["what"] == "lookup":
        s.out.copy_(torch.where(known[:, None], s.table[ids].float() * c["scale"], 0.0))
        return {"out": s.out}
    # sums over up to all positions of a text, in the order the additions happen to come: in 64 bits
    rows = torch.where(known[:, None], s.dout.double(), 0.0) * c["scale"]
    total = torch.zeros(c["V"], c["D"], dtype=torch.float64, device=DEVICE).index_add_(0, ids, rows)
    if c["accumulate"]:
        total += s.dtable
    s.dtable.copy_(total)
    return {"dtable": s.dtable}


def _exact_embedding(c, gen):
    i = _embedding_inputs(c, gen)
    t = i["tokens"].long()
    if c["what"] == "lookup":
        padded = torch.cat([i["table"].double(), torch.zeros(1, c["D"], dtype=torch.float64, device=DEVICE)])
        return {"out": padded[torch.where((t < 0) | (t >= c["V"]), c["V"], t)] * c["scale"]}
    order = torch.argsort(t, stable=True)
    t, rows = t[order], i["dout"].double()[order]
    out = torch.zeros(c["V"], c["D"], dtype=torch.float64, device=DEVICE)
    ids, counts = torch.unique_consecutive(t, return_counts=True)
    ends = torch.cumsum(counts, 0)
    sums = torch.zeros(len(t) + 1, c["D"], dtype=torch.float64, device=DEVICE)
    torch.cumsum(rows, 0, out=sums[1:])
    per_id = sums[ends] - sums[ends - counts]
    keep = (ids >= 0) & (ids < c["V"])
    out[ids[keep]] = per_id[keep] * c["scale"]
    return {"dtable": out + i["before"].double() if c["accumulate"] else out}


def _work_embedding(c):
    es = 4 if c["dtype"] == "f32" else 2
    N, V, D = c["N"], c["V"], c["D"]
    if c["what"] == "lookup":
        distinct = min(N, V)
        return {"bytes": 4.0 * N + es * D * (distinct + N), "flops": float(N * D)}
    return {"bytes": 4.0 * N + es * N * D + (8.0 * D * min(N, V) if c["accumulate"] else 4.0 * V * D), "flops": 2.0 * N * D}


# ---- attention in a window --------------------------------------------------------------------------
def _lengths(c):
    """Keys of each sequence: from a quarter of the room to all of it."""
    B, S = c["B"], c["Sk"]
    return [max(1, S - (S * 3 // 4) * b // B) for b in range(B)] if c["padded"] else [S] * B


def _positions(c):
    """Of each sequence's first query: training starts at zero, a chunk or a token is the last of the keys."""
    return [0] * c["B"] if c["what"] == "train" else [n - c["Sq"] for n in _lengths(c)]


def _window_inputs(c, gen):
    td = _torch_dtype(c["dtype"])
    B, Sq, Sk, H, Hkv, dh = (c[k] for k in ("B", "Sq", "Sk", "H", "Hkv", "dh"))
    i = dict(k_len=torch.tensor(_lengths(c), dtype=torch.int32, device=DEVICE), q_pos=torch.tensor(_positions(c), dtype=torch.int32, device=DEVICE))
    # queries and keys that give some keys a good share of a row
    if c["what"] == "train":
        qkv = torch.randn(B, Sq, H + 2 * Hkv, dh, generator=gen, device=DEVICE)
        qkv[:, :, :H] *= 1.5
        i["qkv"] = qkv.to(td)
        dctx = torch.randn(B, Sq, H, dh, generator=gen, device=DEVICE)
        behind = torch.arange(Sq, device=DEVICE)[None] >= i["k_len"][:, None]
        i["dctx"] = torch.where(behind[:, :, None, None], 0.0, dctx).to(td)  # the loss does not count padding
    else:
        i["q"] = (1.5 * torch.randn(B, Sq, H, dh, generator=gen, device=DEVICE)).to(td)
        i["k"] = torch.randn(B, Sk, Hkv, dh, generator=gen, device=DEVICE).to(td)
        i["v"] = torch.randn(B, Sk, Hkv, dh, generator=gen, device=DEVICE).to(td)
    return i


def _prepare_window(c, gen, s):
    i = _window_inputs(c, gen)
    s.td, s.k_len, s.q_pos = _torch_dtype(c["dtype"]), i["k_len"], i["q_pos"]
    B, Sq, H, Hkv, dh = (c[k] for k in ("B", "Sq", "H", "Hkv", "dh"))
    if c["what"] == "train":
        s.qkv, s.dctx = i["qkv"], i["dctx"]
        s.q, s.k, s.v = s.qkv.split([H, Hkv, Hkv], 2)
        s.dqkv = torch.empty_like(s.qkv)
        s.dq, s.dk, s.dv = s.dqkv.split([H, Hkv, Hkv], 2)
    else:
        s.q, s.k, s.v = i["q"], i["k"], i["v"]
    s.ctx = torch.empty(B, Sq, H, dh, dtype=s.td, device=DEVICE)
    s.lse = torch.empty(B, H, Sq, device=DEVICE)
    if own:
        fax = _fax()
        s.dims = fax.window_dims(s.q, s.k, c["window"], c["sinks"])
        s.ws_bytes = fax.fax_window_attention_workspace_bytes(s.dims)
        s.ws = _workspace(s.ws_bytes)


def _grouped(t, Hkv):
    """[B, S, heads, dh] -> fp32 [B, Hkv, heads / Hkv * S, dh]"""
    B, S, H, dh = t.shape
    return t.float().reshape(B, S, Hkv, H // Hkv, dh).permute(0, 2, 3, 1, 4).reshape(B, Hkv, -1, dh)


def _ungrouped(t, S):
    B, Hkv, n, dh = t.shape
    return t.reshape(B, Hkv, n // S, S, dh).permute(0, 3, 1, 2, 4).reshape(B, S, Hkv * (n // S), dh)


def _plain_window(s):
    c = s.case
    G, Hkv, Sq, scale = c["H"] // c["Hkv"], c["Hkv"], c["Sq"], 1.0 / math.sqrt(c["dh"])
    p = (s.q_pos.long()[:, None] + torch.arange(Sq, device=DEVICE))[:, :, None]
    j = torch.arange(c["Sk"], device=DEVICE)[None, None]
    seen = (j < s.k_len[:, None, None]) & (j <= p) & ((j > p - c["window"]) | (j < c["sinks"]))
    hidden = ~seen.repeat(1, G, 1)[:, None]
    q, k, v = _grouped(s.q, Hkv), _grouped(s.k, Hkv), _grouped(s.v, Hkv)
    x = torch.matmul(q, k.transpose(-1, -2).contiguous()).mul_(scale).masked_fill_(hidden, -math.inf)
    top = x.amax(-1, keepdim=True)
    x = x.sub_(torch.where(top > -math.inf, top, 0.0)).exp_()
    l = x.sum(-1, keepdim=True)
    x.div_(torch.where(l > 0, l, 1.0))
    o = torch.matmul(x, v)
    s.ctx.copy_(_ungrouped(o, Sq))
    s.lse.copy_((top + l.log()).reshape(s.lse.shape))
    if c["what"] != "train":
        return {"ctx": s.ctx, "lse": s.lse}
    do = _grouped(s.dctx, Hkv)
    delta = (do * o).sum(-1, keepdim=True)
    s.dv.copy_(_ungrouped(torch.matmul(x.transpose(-1, -2).contiguous(), do), c["Sk"]))
    x.mul_(torch.matmul(do, v.transpose(-1, -2).contiguous()).sub_(delta)).mul_(scale)
    s.dq.copy_(_ungrouped(torch.matmul(x, k), Sq))
    s.dk.copy_(_ungrouped(torch.matmul(x.transpose(-1, -2).contiguous(), q), c["Sk"]))
    return {"ctx": s.ctx, "lse": s.lse, "dqkv": s.dqkv}


def _run_window(s):
    if not own:
        return _plain_window(s)
    fax = _fax()
    fax.fax_window_attention_fwd(s.dims, s.q, s.k, s.v, s.q_pos, s.k_len, s.ctx, s.lse, s.ws, s.ws_bytes)
    if s.case["what"] != "train":
        return {"ctx": s.ctx, "lse": s.lse}
    fax.fax_window_attention_bwd(s.dims, s.q, s.k, s.v, s.q_pos, s.k_len, s.ctx, s.lse, s.dctx, s.dq, s.dk, s.dv, s.ws, s.ws_bytes)
    return {"ctx": s.ctx, "lse": s.lse, "dqkv": s.dqkv}


def _exact_window(c, gen):
    """Head by head, and in runs of queries against the keys from the first one that any of the run may see in its window, the sinks before them."""
    i = _window_inputs(c, gen)
    B, Sq, Sk, H, Hkv, dh, W = (c[k] for k in ("B", "Sq", "Sk", "H", "Hkv", "dh", "window"))
    train = c["what"] == "train"
    if train:
        q, k, v = i["qkv"].split([H, Hkv, Hkv], 2)
    else:
        q, k, v = i["q"], i["k"], i["v"]
    ctx = torch.zeros(B, Sq, H, dh, dtype=torch.float64, device=DEVICE)
    lse = torch.full((B, H, Sq), -math.inf, dtype=torch.float64, device=DEVICE)
    dqkv = torch.zeros(B, Sq, H + 2 * Hkv, dh, dtype=torch.float64, device=DEVICE) if train else None
    run = 1024
    for b, (n, first) in enumerate(zip(_lengths(c), _positions(c))):
        for r0 in range(0, Sq, run):
            r1 = min(Sq, r0 + run)
            near = max(0, min(n, first + r0 - W + 1))
            some = torch.cat([torch.arange(min(c["sinks"], near), device=DEVICE), torch.arange(near, max(near, min(n, first + r1)), device=DEVICE)])
            if not len(some):
                continue
            at = torch.arange(first + r0, first + r1, device=DEVICE)[:, None]
            far = (some[None] > at) | ((at - some[None] >= W) & (some[None] >= c["sinks"]))
            for h in range(H):
                g = h // (H // Hkv)
                qh, kh, vh = q[b, r0:r1, h].double(), k[b, some, g].double(), v[b, some, g].double()
                z = (qh @ kh.T / math.sqrt(dh)).masked_fill(far, -math.inf)
                ls = torch.logsumexp(z, 1)
                P = torch.exp(z - ls[:, None]).nan_to_num(0.0)
                ctx[b, r0:r1, h], lse[b, h, r0:r1] = P @ vh, ls
                if train:
                    d = i["dctx"][b, r0:r1, h].double()
                    dS = P * (d @ vh.T - (d * (P @ vh)).sum(1, keepdim=True)) / math.sqrt(dh)
                    dqkv[b, r0:r1, h] = dS @ kh
                    dqkv[b, :, H + g].index_add_(0, some, dS.T @ qh)
                    dqkv[b, :, H + Hkv + g].index_add_(0, some, P.T @ d)
    return {"ctx": ctx, "lse": lse, "dqkv": dqkv} if train else {"ctx": ctx, "lse": lse}


def _work_window(c):
    es = 4 if c["dtype"] == "f32" else 2
    B, Sq, H, Hkv, dh = (c[k] for k in ("B", "Sq", "H", "Hkv", "dh"))
    pairs = keys = 0
    for n, first in zip(_lengths(c), _positions(c)):
        p = torch.arange(Sq, dtype=torch.int64) + first
        inside = (torch.clamp(p + 1, max=n) - torch.clamp(p - c["window"] + 1, min=0)).clamp(min=0)
        sinks = torch.minimum(torch.clamp(p - c["window"] + 1, min=0), torch.tensor(min(c["sinks"], n))).clamp(min=0)
        pairs += int((inside + sinks).sum())
        near = max(0, first - c["window"] + 1)
        keys += max(0, min(n, first + Sq) - near) + min(c["sinks"], near)
    rows = B * Sq * H * dh * es
    if c["what"] == "train":
        return {"bytes": 4.0 * rows + 4.0 * keys * Hkv * dh * es + 8.0 * B * H * Sq, "flops": 14.0 * dh * H * pairs}
    return {"bytes": 2.0 * rows + 2.0 * keys * Hkv * dh * es + 4.0 * B * H * Sq, "flops": 4.0 * dh * H * pairs}


# ---- AdamW over many tensors ------------------------------------------------------------------------
def _tensors(c):
    """(shape, whether weights decay) of each."""
    D, Hd, F = c["D"], c["Hd"], c["F"]
    layer = [((D,), False), ((D,), False), ((D, 3 * Hd), True), ((3 * Hd,), False), ((Hd, D), True), ((D,), False),
             ((D,), False), ((D,), False), ((D, F), True), ((F,), False), ((F, D), True), ((D,), False)]
    top = [((c["V"], D), True), ((2048, D), True), ((D,), False), ((D,), False)] if c["V"] else []
    return top + c["layers"] * layer


def _round_up(n, to):
    return (n + to - 1) // to * to


def _adamw_inputs(c, gen):
    """Flat buffers in which every tensor starts a block of its own: gradients of a mean loss (about 1e-4, rows of different size), established moments."""
    counts = [math.prod(t) for t, _ in _tensors(c)]
    starts, at = [], 0
    for n in counts:
        starts.append(at)
        at += _round_up(n, BLOCK)
    real = torch.zeros(at, dtype=torch.bool, device=DEVICE)
    decay = torch.ones(at // BLOCK, 1, device=DEVICE)
    first = torch.zeros(at // BLOCK, 1, dtype=torch.int64, device=DEVICE)  # a block's first element in its tensor
    owner = torch.zeros(at // BLOCK, 1, dtype=torch.int64, device=DEVICE)  # and which tensor that is
    for k, (o, n, (_, weights)) in enumerate(zip(starts, counts, _tensors(c))):
        real[o:o + n] = True
        b0, b1 = o // BLOCK, (o + _round_up(n, BLOCK)) // BLOCK
        decay[b0:b1] = 1.0 - LR * WD if weights else 1.0
        owner[b0:b1] = k
        first[b0:b1, 0] = torch.arange(b1 - b0, device=DEVICE) * BLOCK
    randn = lambda: torch.where(real, torch.randn(at, generator=gen, device=DEVICE), 0.0)  # noqa: E731
    size = (1e-4 * torch.exp(torch.randn(at // 64, 1, generator=gen, device=DEVICE))).expand(-1, 64).reshape(-1)
    i = dict(counts=counts, starts=starts, decay=decay, first=first, owner=owner, seed=int(torch.randint(0, 2 ** 31, (1,), generator=gen, device=DEVICE)))
    i["p"] = 0.02 * randn()
    i["g"] = (size * randn()).to(_torch_dtype(c["grad"]))
    m = 0.2 * size * randn()
    v = torch.where(real, size * size * (0.5 + torch.rand(at, generator=gen, device=DEVICE)), 0.0)
    if c["state"] == 32:
        i["m"], i["v"] = m, v
    else:
        for name, x in (("m", m), ("v", v.sqrt())):
            scale = x.view(-1, BLOCK).abs().amax(1, keepdim=True) / E4M3_MAX
            i[name + "_scale"] = scale.reshape(-1)
            i[name] = (x.view(-1, BLOCK) / scale).to(torch.float8_e4m3fn).reshape(-1)
    return i


def _prepare_adamw(c, gen, s):
    s.__dict__.update(_adamw_inputs(c, gen))
    s.step = FIRST_STEP
    s.lowp = s.p.to(torch.bfloat16) if c["lowp"] else None
    if own:
        fax = _fax()
        s.hp = fax.FaxAdamW(lr=LR, beta1=BETA1, beta2=BETA2, eps=EPS, wd=WD)
        s.state = fax.FAX_STATE_F32 if c["state"] == 32 else fax.FAX_STATE_E4M3
        cut = lambda t, o, n: None if t is None else t[o:o + n]  # noqa: E731
        tensors = []
        for o, n, (_, weights) in zip(s.starts, s.counts, _tensors(c)):
            t = dict(master=cut(s.p, o, n), m=cut(s.m, o, n), v=cut(s.v, o, n), grad=cut(s.g, o, n), lowp=cut(s.lowp, o, n), decay=weights)
            if c["state"] == 8:
                t.update(m_scale=s.m_scale[o // BLOCK:], v_scale=s.v_scale[o // BLOCK:])
            tensors.append(t)
        s.table = fax.adamw_tensors(tensors)


def _mix(x):
    """32 bits of a hash, in int64."""
    x = x & 0xFFFFFFFF
    x = ((x ^ (x >> 16)) * 0x9E3779B1) & 0xFFFFFFFF
    x = ((x ^ (x >> 15)) * 0x2545F491) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _random20(seed, step, owner, first):
    """The twenty random bits with which sqrt(v) of each element is rounded."""
    key = _mix(_mix(torch.tensor(seed + step * 0x9E3779B1, device=DEVICE)) + owner * 0x9E3779B1)
    return _mix((first + torch.arange(BLOCK, device=DEVICE)) * 0x9E3779B1 + key) >> 12


def _plain_adamw(s):
    c = s.case
    s.step += 1
    p, g = s.p.view(-1, BLOCK), s.g.view(-1, BLOCK).float()
    m, v = s.m.view(-1, BLOCK).float(), s.v.view(-1, BLOCK).float()
    if c["state"] == 8:
        m, v = m * s.m_scale[:, None], (v * s.v_scale[:, None]).square()
    m = BETA1 * m + (1.0 - BETA1) * g
    v = BETA2 * v + (1.0 - BETA2) * g * g
    up = (m * (1.0 / (1.0 - BETA1 ** s.step))) / ((v * (1.0 / (1.0 - BETA2 ** s.step))).sqrt() + EPS)
    p.copy_(p * s.decay - LR * up)
    if c["lowp"]:
        s.lowp.copy_(s.p)
    if c["state"] == 32:
        s.m.copy_(m.reshape(-1))
        s.v.copy_(v.reshape(-1))
        return _adamw_outputs(s)
    top = m.abs().amax(1, keepdim=True)
    top = torch.where(top < M_FLOOR, 0.0, top)
    s.m.copy_(torch.where(top > 0, m * (E4M3_MAX / top), 0.0).to(torch.float8_e4m3fn).reshape(-1))
    s.m_scale.copy_((top / E4M3_MAX).reshape(-1))
    r = v.sqrt()
    top = r.amax(1, keepdim=True)
    x = torch.where(top > 0, r * (E4M3_MAX / top), 0.0)
    low = x < 2.0 ** -6  # below, numbers are whole multiples of 2^-9, as they are from 2^-6 to 2^-5
    y = torch.where(low, x + 2.0 ** -6, x).view(torch.int32) + _random20(s.seed, s.step, s.owner, s.first).to(torch.int32)
    y = torch.bitwise_and(y, -1 << 20).view(torch.float32)
    y = torch.where(low, y - 2.0 ** -6, y).clamp(max=E4M3_MAX)
    y = torch.where(r > 0, y.clamp(min=2.0 ** -9), 0.0)
    s.v.copy_(y.to(torch.float8_e4m3fn).reshape(-1))
    s.v_scale.copy_((top / E4M3_MAX).reshape(-1))
    return _adamw_outputs(s)


def _adamw_outputs(s):
    out = {"master": s.p, "m": s.m, "v": s.v}
    if s.case["lowp"]:
        out["lowp"] = s.lowp
    if s.case["state"] == 8:
        out.update(m_scale=s.m_scale, v_scale=s.v_scale)
    return out


def _run_adamw(s):
    if not own:
        return _plain_adamw(s)
    fax = _fax()
    s.step += 1
    fax.fax_adamw_multi_step(s.state, s.table, s.hp, s.step, s.seed)
    return _adamw_outputs(s)


def _exact_adamw(c, gen):
    i = _adamw_inputs(c, gen)
    t = FIRST_STEP + 1
    d = lambda name: i[name].to(torch.float32).double().view(-1, BLOCK)  # noqa: E731
    m, r = d("m"), d("v")
    if c["state"] == 8:
        m = m * i["m_scale"].double()[:, None]
        v = (r * i["v_scale"].double()[:, None]) ** 2
    else:
        v = r
    g = d("g")
    m = m * BETA1 + g * (1.0 - BETA1)
    v = v * BETA2 + g ** 2 * (1.0 - BETA2)
    decay = torch.where(i["decay"] < 1.0, 1.0 - LR * WD, 1.0).double()
    p = d("p") * decay - LR * (m / (1.0 - BETA1 ** t)) / (torch.sqrt(v / (1.0 - BETA2 ** t)) + EPS)
    out = {"master": p.reshape(-1)}
    if c["lowp"]:
        out["lowp"] = out["master"]
    if c["state"] == 32:
        return dict(out, m=m.reshape(-1), v=v.reshape(-1))
    spacing = lambda x: torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3.0)  # noqa: E731
    for name, x in (("m", m), ("v", v.sqrt())):
        scale = x.abs().amax(1, keepdim=True) / E4M3_MAX
        x = torch.where(scale > 0, x / torch.where(scale > 0, scale, 1.0), 0.0)
        step = spacing(x)
        if name == "m":
            x = torch.round(x / step) * step
        else:
            u = _random20(i["seed"], t, i["owner"], i["first"]).double() / 2.0 ** 20
            x = torch.where(x > 0, torch.clamp(torch.floor(x / step + u) * step, 2.0 ** -9, E4M3_MAX), 0.0)
        out[name], out[name + "_scale"] = x.reshape(-1), scale.reshape(-1)
    return out


def _work_adamw(c):
    n = sum(math.prod(t) for t, _ in _tensors(c))
    each = 8 + (4 if c["grad"] == "f32" else 2) + (2 if c["lowp"] else 0) + (16 if c["state"] == 32 else 4 + 16 / BLOCK)
    return {"bytes": float(each * n), "flops": 16.0 * n}


# ---- the six functions ------------------------------------------------------------------------------
_PREPARE = {EMBEDDING: _prepare_embedding, WINDOW: _prepare_window, ADAMW: _prepare_adamw}
_RUN = {EMBEDDING: _run_embedding, WINDOW: _run_window, ADAMW: _run_adamw}
_EXACT = {EMBEDDING: _exact_embedding, WINDOW: _exact_window, ADAMW: _exact_adamw}
_WORK = {EMBEDDING: _work_embedding, WINDOW: _work_window, ADAMW: _work_adamw}


def _generator(seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    return gen


def prepare(case, seed):
    s = _State()
    s.case = dict(case)
    _PREPARE[case["op"]](s.case, _generator(seed), s)
    return s


def run(state):
    return _RUN[state.case["op"]](state)


def exact(case, seed):
    return _EXACT[case["op"]](dict(case), _generator(seed))


def work(case):
    return _WORK[case["op"]](case)
