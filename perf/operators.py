"""Performance cases of the local stream's attention operators.

``listed()`` names the measured calls, ``draw(rng)`` gives more of the same ranges, ``prepare`` makes what a program
holds before the call, ``run`` is one pass (in plain torch, or through the library where ``own`` is true), ``work``
the bytes and FLOPs the pass cannot do without and ``exact`` the same pass from the definition in float64.

Kinds:
  "rope"    norm of every query and key head and its position rotation, forward, or backward with the gradients of
            the norms' weights; positions along one axis (the row of the sequence, or given) or several
  "window"  causal attention in a sliding window with sinks, forward, or a training step (forward and backward)
  "append"  keys (normed and rotated on the way) and values of prompts, or of one token a sequence, into a paged
            cache; the queries get the same norm and rotation
  "attend"  attention of one new token a sequence over its pages
"""
import math

import torch

own = False

F32, F64, BF, I32 = torch.float32, torch.float64, torch.bfloat16, torch.int32
EPS = 1e-6
THETA = 10000.0


def _case(name, **c):
    return dict(c, name=name) if name else c


def _rope(name, batch, L, heads, kv, dh, axes=1, norm=True, offset=0, backward=False, dtype="bf16"):
    """axes > 1: a grid of about L ** (1 / axes) a side, positions given; offset: given positions from there on."""
    return _case(name, kind="rope", batch=batch, L=L, heads=heads, kv=kv, dh=dh, axes=axes, norm=norm, offset=offset,
                 backward=backward, dtype=dtype)


def _window(name, batch, L, heads, kv, window, sinks, train):
    """window 0: every earlier key."""
    return _case(name, kind="window", batch=batch, L=L, heads=heads, kv=kv, window=window, sinks=sinks, train=train)


def _append(name, batch, tokens, before, heads, kv, dh, page, norm=True):
    """tokens 0: one token a sequence; else prompts of up to that many; before: rows up to which caches are filled."""
    return _case(name, kind="append", batch=batch, tokens=tokens, before=before, heads=heads, kv=kv, dh=dh, page=page,
                 norm=norm)


def _attend(name, batch, rows, ragged, heads, kv, dh, page, window=0, sinks=0):
    """rows: of the longest sequence; ragged: the others hold anything from none to that."""
    return _case(name, kind="attend", batch=batch, rows=rows, ragged=ragged, heads=heads, kv=kv, dh=dh, page=page,
                 window=window, sinks=sinks)


def listed():
    return [
        # two short sequences of a small layer: latency
        _rope("rope_fwd_small", 2, 33, 8, 2, 64),
        # training of 64K tokens with 16 query and 4 key heads
        _rope("rope_bwd_64k", 1, 65536, 16, 4, 64, backward=True),
        # four 512 x 512 images, positions along two axes
        _rope("rope_image_fwd", 4, 262144, 8, 8, 64, axes=2),
        # three prompts of about a thousand tokens
        _window("window_fwd_1k", 3, 1021, 8, 2, 256, 4, False),
        # training step of a small ragged layer: latency and launches
        _window("window_train_small", 2, 1000, 2, 2, 128, 1, True),
        # training step of 64K tokens
        _window("window_train_64k", 1, 65536, 16, 16, 1024, 4, True),
        # a prompt of 256K tokens with a wide window and grouped heads
        _window("window_fwd_256k", 1, 262144, 16, 4, 4096, 64, False),
        # one token of each of 8 sequences
        _append("append_b8", 8, 0, 1000, 16, 16, 128, 64),
        # eight prompts of up to 2500 tokens, some of them on a filled cache
        _append("append_prompts", 8, 2500, 700, 16, 2, 128, 64),
        # one token over a short cache
        _attend("attend_b1_1k", 1, 1000, False, 16, 4, 64, 16),
        # one token of each of 8 sequences of up to 16384 cached rows, a key head for every query head
        _attend("attend_b8_16k", 8, 16384, True, 16, 16, 128, 64),
        # one token over a million cached rows with grouped heads
        _attend("attend_b1_1m", 1, 1048576, False, 16, 2, 128, 64),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _heads(rng, most=16):
    """Query heads and key heads: up to `most` query heads for a key head."""
    kv = rng.choice([1, 2, 3, 4, 8, 16])
    return kv * rng.choice([g for g in (1, 2, 4, 5, 8, 16) if g <= most and kv * g <= 32 and kv * g != 24]), kv


def draw(rng):
    kind = rng.choice(["rope", "rope", "window", "window", "window", "append", "append", "attend", "attend", "attend"])
    heads, kv = _heads(rng)
    dh = rng.choice([64, 128])
    page = rng.choice([16, 32, 64, 128])
    if kind == "rope":
        batch = rng.choice([1, 1, 2, 3, 4])
        L = _log(rng, 1, min(262144, 2 ** 29 // (batch * (heads + kv) * dh)))
        return _rope("", batch, L, heads, kv, dh, rng.choice([1, 1, 2, 3]), rng.random() < 0.8,
                     rng.choice([0, 0, _log(rng, 1, 2 ** 20)]), rng.random() < 0.5, rng.choice(["bf16", "bf16", "f32"]))
    if kind == "window":
        while True:
            batch, L = rng.choice([1, 1, 2, 3]), _log(rng, 1, 65536)
            window = rng.choice([0, _log(rng, 1, 4096), _log(rng, 1, 4096)])
            sinks = rng.choice([0, rng.randint(1, 8), _log(rng, 1, 300)])
            train = rng.random() < 0.6
            cost = batch * heads * L * min(L, (window or L) + sinks) * (3.5 if train else 1.0)
            if cost <= 2 ** 34 and batch * L * heads <= 2 ** 21:
                return _window("", batch, L, heads, kv, window, sinks, train)
    if kind == "append":
        tokens = rng.choice([0, _log(rng, 1, 4000)])
        return _append("", _log(rng, 1, 64) if tokens < 600 else _log(rng, 1, 8), tokens, _log(rng, 1, 2000), heads, kv,
                       dh, page, rng.random() < 0.8)
    while True:
        batch, rows = _log(rng, 1, 64), _log(rng, 1, 262144)
        if batch * rows * kv * dh <= 2 ** 28:
            window = rng.choice([0, 0, _log(rng, 1, 8192)])
            return _attend("", batch, rows, rng.random() < 0.7, heads, kv, dh, page, window,
                           _log(rng, 1, 100) if window else 0)


# ------------------------------------------------------------------ inputs
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(g, *shape, dtype=BF, scale=1.0):
    """Normal values, made in pieces of whole rows so that the float32 values never exist all at once."""
    out = torch.empty(shape, dtype=dtype, device="cuda")
    for part in out.view(-1).split(1 << 27):
        part.copy_(torch.randn(part.shape, generator=g, device="cuda").mul_(scale))
    return out


def _norm_weights(c, g):
    """Weights of the norms, about 1 as after training, or none."""
    if not c["norm"]:
        return None, None
    return tuple(1.0 + 0.2 * torch.randn(c["dh"], generator=g, device="cuda") for _ in range(2))


def _pairs(dh, axes):
    """Pairs of a head that each axis turns (the first axes take what does not divide)."""
    n = dh // 2
    return tuple(n // axes + (1 if a < n % axes else 0) for a in range(axes))


def _positions(c):
    """[rows, axes] positions, or None where a token's position is its row in the sequence."""
    if c["axes"] == 1 and not c["offset"]:
        return None
    i = torch.arange(c["L"], device="cuda")
    side = max(1, round(c["L"] ** (1.0 / c["axes"])))
    cols = []
    for a in range(c["axes"] - 1, 0, -1):  # the first axis is the slowest
        cols.insert(0, i % side)
        i = i // side
    cols.insert(0, i)
    return (torch.stack(cols, 1) + c["offset"]).to(I32).repeat(c["batch"], 1).contiguous()


def _spread(n, top):
    """n whole numbers from 0 to top, the first of them top: multiples of the golden section of it."""
    return [top - int((top + 1) * (0.6180339887498949 * i % 1.0)) for i in range(n)]


def _lengths(c):
    """Rows of every sequence before the call and tokens that the call brings (append), or cached rows (attend)."""
    if c["kind"] == "append":
        return _spread(c["batch"], c["before"])[::-1], [max(1, t) for t in _spread(c["batch"], c["tokens"])]
    return _spread(c["batch"], c["rows"]) if c["ragged"] else [c["rows"]] * c["batch"]


def _table(rows, page, g):
    """Page table [batch, pages] for sequences of so many rows, pages in random order, -1 where there is none."""
    need = [-(-r // page) for r in rows]
    n = max(1, sum(need))
    order = torch.randperm(n, generator=g, device="cuda").tolist()
    table = [[-1] * max(1, max(need)) for _ in rows]
    for b, k in enumerate(need):
        for j in range(k):
            table[b][j] = order.pop()
    return torch.tensor(table, dtype=I32, device="cuda"), n


def _inputs(c, seed):
    """The tensors of a case."""
    g = _gen(seed)
    s = {"case": c}
    H, KV, dh = c["heads"], c["kv"], c.get("dh", 64)
    if c["kind"] == "rope":
        n, dt = c["batch"] * c["L"], F32 if c["dtype"] == "f32" else BF
        s.update(q=_randn(g, n, H * dh, dtype=dt, scale=1.5), k=_randn(g, n, KV * dh, dtype=dt, scale=1.5))
        s["w_q"], s["w_k"] = _norm_weights(c, g)
        s["pos"] = _positions(c)
        if c["backward"]:
            s.update(dq=_randn(g, n, H * dh, dtype=dt), dk=_randn(g, n, KV * dh, dtype=dt))
    elif c["kind"] == "window":
        n = c["batch"] * c["L"]
        s.update(q=_randn(g, n, H * dh), k=_randn(g, n, KV * dh), v=_randn(g, n, KV * dh))
        if c["train"]:
            s["do"] = _randn(g, n, H * dh)
    elif c["kind"] == "append":
        before, new = _lengths(c)
        n = sum(new)
        s.update(q=_randn(g, n, H * dh, scale=1.5), k=_randn(g, n, KV * dh, scale=1.5), v=_randn(g, n, KV * dh))
        s["w_q"], s["w_k"] = _norm_weights(c, g)
        rows = [a + b for a, b in zip(before, new)]
        s["table"], pages = _table(rows, c["page"], g)
        s["len"] = torch.tensor(rows, dtype=I32, device="cuda")
        first = [0]
        for t in new:
            first.append(first[-1] + t)
        s["start"] = torch.tensor(first, dtype=I32, device="cuda") if c["tokens"] else None
        s["K"], s["V"] = (_randn(g, pages, KV, c["page"], dh) for _ in range(2))
    else:
        rows = _lengths(c)
        s["q"] = _randn(g, c["batch"], H * dh)
        s["table"], pages = _table(rows, c["page"], g)
        s["len"] = torch.tensor(rows, dtype=I32, device="cuda")
        s["K"], s["V"] = (_randn(g, pages, KV, c["page"], dh) for _ in range(2))
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    c = case
    if own:
        from paper_2608_23463_gb300.local import PagedKVCache, QKRope, WindowAttention
        H, KV, dh = c["heads"], c["kv"], c.get("dh", 64)
        rope = None
        if c["kind"] in ("rope", "append"):
            rope = QKRope(H, KV, dh, s["w_q"], s["w_k"], pairs=_pairs(dh, c.get("axes", 1)), theta=THETA, eps=EPS,
                          dtype=s["q"].dtype)
        if c["kind"] == "rope":
            s["op"] = rope
        elif c["kind"] == "window":
            s["op"] = WindowAttention(c["batch"], c["L"], H, KV, dh, window=c["window"], n_sink=c["sinks"])
        else:
            s["op"] = PagedKVCache(c["batch"], H, KV, dh, c["page"], s["K"].shape[0], s["table"].shape[1], rope=rope,
                                   window=c.get("window", 0), n_sink=c.get("sinks", 0), K=s.pop("K"), V=s.pop("V"),
                                   table=s["table"], len=s["len"])
    elif c["kind"] == "attend":
        # the plain form's plan: which rows of the pools a sequence sees, and the lengths on the host
        s["lens"] = s["len"].tolist()
    return s


# -------------------------------------------------------------- plain forms
def _turns(pos, n):
    """cos and sin [rows, n] of pos * THETA ** (-i / n): whole turns of 2 ** 64 steps, so that far positions lose
    nothing to rounding."""
    f = [int(THETA ** (-i / n) / (2 * math.pi) * 2.0 ** 64) for i in range(n)]
    f = torch.tensor([x - 2 ** 64 if x >= 2 ** 63 else x for x in f], dtype=torch.int64, device=pos.device)
    a = ((pos.long()[:, None] * f) >> 32).to(F32) * (math.pi / 2.0 ** 31)
    return a.cos(), a.sin()


def _angles(c, pos, dh):
    """cos, sin [rows, 1, dh / 2] of the given positions [rows, axes]."""
    cs = [_turns(pos[:, a], n) for a, n in enumerate(_pairs(dh, pos.shape[1]))]
    return tuple(torch.cat([x[i] for x in cs], 1)[:, None] for i in range(2))


def _turn(y, cos, sin):
    a, b = y[..., 0::2], y[..., 1::2]
    return torch.stack((a * cos - b * sin, a * sin + b * cos), -1).flatten(-2)


def _plain_rope(x, w, cos, sin, dh):
    y = x.to(F32).view(x.shape[0], -1, dh)
    if w is not None:
        y = y * (y.square().mean(-1, keepdim=True) + EPS).rsqrt() * w
    return _turn(y, cos, sin).view(x.shape).to(x.dtype)


def _plain_rope_bwd(x, w, dz, cos, sin, dh):
    dy = _turn(dz.to(F32).view(x.shape[0], -1, dh), cos, -sin)
    if w is None:
        return dy.view(x.shape).to(x.dtype), None
    x32 = x.to(F32).view(dy.shape)
    r = (x32.square().mean(-1, keepdim=True) + EPS).rsqrt()
    xh = x32 * r
    dw = (dy * xh).sum((0, 1))
    g = dy * w
    dx = r * (g - xh * (g * xh).mean(-1, keepdim=True))
    return dx.view(x.shape).to(x.dtype), dw


def _run_rope(s):
    c = s["case"]
    if own:
        if c["backward"]:
            return s["op"].backward(s["q"], s["k"], s["dq"], s["dk"], L=c["L"], pos=s["pos"])
        return s["op"].forward(s["q"], s["k"], L=c["L"], pos=s["pos"])
    pos = s["pos"]
    if pos is None:
        pos = torch.arange(c["L"], device="cuda").repeat(c["batch"])[:, None]
    cos, sin = _angles(c, pos, c["dh"])
    if not c["backward"]:
        return tuple(_plain_rope(s[n], s["w_" + n], cos, sin, c["dh"]) for n in "qk")
    (dq, wq), (dk, wk) = (_plain_rope_bwd(s[n], s["w_" + n], s["d" + n], cos, sin, c["dh"]) for n in "qk")
    return dq, dk, wq, wk


def _blocks(c, step):
    """Blocks of queries [i0, i1) and the keys that any of them sees: the sinks [0, s) and [j0, i1)."""
    L, W, S = c["L"], c["window"] or c["L"], c["sinks"]
    for i0 in range(0, L, step):
        i1 = min(L, i0 + step)
        j0 = max(0, i0 - W + 1)
        yield i0, i1, min(S, j0), j0


def _seen(i0, i1, s, j0, W, S):
    """[queries, keys] truth values of what the queries [i0, i1) see of the keys [0, s) and [j0, i1)."""
    i = torch.arange(i0, i1, device="cuda")[:, None]
    j = torch.cat((torch.arange(s, device="cuda"), torch.arange(j0, i1, device="cuda")))
    return (j <= i) & ((i - j < W) | (j < S))


def _run_window(s):
    c = s["case"]
    if own:
        o = s["op"].forward(s["q"], s["k"], s["v"], train=c["train"])
        if not c["train"]:
            return o
        return (o,) + tuple(s["op"].backward(s["q"], s["k"], s["v"], o, s["do"]))
    B, L, H, KV, dh = c["batch"], c["L"], c["heads"], c["kv"], 64
    W, S, scale = c["window"] or L, c["sinks"], dh ** -0.5
    grouped = lambda t: t.to(F32).view(B, L, KV, H // KV, dh).permute(0, 2, 3, 1, 4)  # [B, KV, g, L, dh]
    shared = lambda t: t.to(F32).view(B, L, KV, 1, dh).permute(0, 2, 3, 1, 4)
    q, k, v = grouped(s["q"]), shared(s["k"]), shared(s["v"])
    rows = lambda t: t.permute(0, 3, 1, 2, 4).reshape(B * L, -1).to(BF)
    out = torch.empty_like(q)
    if c["train"]:
        do, dq, dk, dv = grouped(s["do"]), torch.empty_like(q), torch.zeros_like(k), torch.zeros_like(v)
    step = max(256, min(2048, 2 ** 24 // (B * H * 256)))
    for i0, i1, ns, j0 in _blocks(c, step):
        kb, vb = (torch.cat((t[..., :ns, :], t[..., j0:i1, :]), -2) for t in (k, v))
        seen = _seen(i0, i1, ns, j0, W, S)
        p = ((q[..., i0:i1, :] @ kb.mT) * scale).masked_fill_(~seen, -math.inf)
        p = (p - p.amax(-1, keepdim=True)).exp_()
        p /= p.sum(-1, keepdim=True)
        ob = p @ vb
        out[..., i0:i1, :] = ob
        if not c["train"]:
            continue
        gb = do[..., i0:i1, :]
        ds = p * (gb @ vb.mT - (gb * ob).sum(-1, keepdim=True)) * scale
        dq[..., i0:i1, :] = ds @ kb
        for acc, part in ((dk, ds.mT @ q[..., i0:i1, :]), (dv, p.mT @ gb)):
            part = part.sum(2, keepdim=True)
            acc[..., :ns, :] += part[..., :ns, :]
            acc[..., j0:i1, :] += part[..., ns:, :]
    return (rows(out), rows(dq), rows(dk), rows(dv)) if c["train"] else rows(out)


def _run_append(s):
    c = s["case"]
    if own:
        op = s["op"]
        return op.append(s["q"], s["k"], s["v"], start=s["start"]), op.K, op.V
    dh, page = c["dh"], c["page"]
    n, lens = s["q"].shape[0], s["len"].long()
    start = s["start"].long() if s["start"] is not None else torch.arange(c["batch"] + 1, device="cuda")
    i = torch.arange(n, device="cuda")
    b = (i[:, None] >= start[None, 1:]).sum(1)  # the sequence of every token
    row = lens[b] - start[b + 1] + i
    cos, sin = _angles(c, row[:, None], dh)
    q, k = (_plain_rope(s[x], s["w_" + x], cos, sin, dh) for x in "qk")
    pg = s["table"].long()[b, row // page]
    s["K"][pg, :, row % page] = k.view(n, -1, dh)
    s["V"][pg, :, row % page] = s["v"].view(n, -1, dh)
    return q, s["K"], s["V"]


def _visible(c, n):
    """Rows of a cache of n that the newest token sees, as ranges."""
    if not c["window"] or c["window"] >= n:
        return [(0, n)]
    j0 = n - c["window"]
    return [(0, min(c["sinks"], j0)), (j0, n)]


def _run_attend(s):
    c = s["case"]
    if own:
        return s["op"].attend(s["q"])
    H, KV, dh, page = c["heads"], c["kv"], c["dh"], c["page"]
    out = torch.zeros(c["batch"], KV, H // KV, dh, device="cuda")
    q = s["q"].to(F32).view(c["batch"], KV, H // KV, dh) * dh ** -0.5
    for b, n in enumerate(s["lens"]):
        if n == 0:
            continue
        j = torch.cat([torch.arange(*r, device="cuda") for r in _visible(c, n)])
        pg = s["table"][b, j // page].long()
        kb, vb = (s[x][pg, :, j % page].to(F32).transpose(0, 1) for x in "KV")  # [KV, rows, dh]
        p = q[b] @ kb.mT
        p = (p - p.amax(-1, keepdim=True)).exp()
        out[b] = (p / p.sum(-1, keepdim=True)) @ vb
    return out.view(c["batch"], -1).to(BF)


def run(state):
    return {"rope": _run_rope, "window": _run_window, "append": _run_append, "attend": _run_attend}[
        state["case"]["kind"]](state)


# ---------------------------------------------------------------------- work
def _pairs_seen(c):
    """Visible (query, key) pairs of a head and sequence."""
    L, W, S = c["L"], c["window"] or c["L"], c["sinks"]
    full = min(W, L)
    pairs = full * (full + 1) // 2 + (L - full) * W
    for i in range(W, min(L, W + S)):  # the sinks come into sight below the window one by one
        pairs += min(S, i - W + 1)
    return pairs + max(0, L - W - S) * S


def work(case):
    c = case
    H, KV, dh = c["heads"], c["kv"], c.get("dh", 64)
    if c["kind"] == "rope":
        n = c["batch"] * c["L"] * (H + KV) * dh
        size = 4 if c["dtype"] == "f32" else 2
        b = n * size * (3 if c["backward"] else 2)
        if c["axes"] > 1 or c["offset"]:
            b += c["batch"] * c["L"] * c["axes"] * 4
        if c["norm"]:
            b += (4 if c["backward"] else 2) * dh * 4
        return {"bytes": b, "flops": n * (16 if c["backward"] else 8)}
    if c["kind"] == "window":
        n = c["batch"] * c["L"] * dh * 2
        b = n * (2 * H + 2 * KV) + (n * (2 * H + 2 * KV) if c["train"] else 0)
        return {"bytes": b, "flops": (14 if c["train"] else 4) * dh * H * c["batch"] * _pairs_seen(c)}
    if c["kind"] == "append":
        n = sum(_lengths(c)[1])
        return {"bytes": n * dh * 2 * (2 * H + 4 * KV), "flops": n * (H + KV) * dh * 8}
    rows = sum(min(r, c["window"] + c["sinks"]) if c["window"] else r for r in _lengths(c))
    return {"bytes": rows * KV * dh * 4 + c["batch"] * H * dh * 4, "flops": 4 * rows * H * dh}


# --------------------------------------------------------------------- exact
def _exact_rotation(pos, dh, axes):
    """Complex numbers [rows, dh / 2] that turn the pairs."""
    ang = [pos[:, a:a + 1].to(F64) * THETA ** (-torch.arange(n, device="cuda", dtype=F64) / n)
           for a, n in enumerate(_pairs(dh, axes))]
    return torch.polar(torch.ones((), dtype=F64, device="cuda"), torch.cat(ang, 1))


def _exact_normed(x, w, turn, dh):
    y = x.unflatten(-1, (-1, dh))
    if w is not None:
        y = w * y / (y.pow(2).mean(-1, keepdim=True) + EPS).sqrt()
    z = torch.view_as_complex(y.unflatten(-1, (-1, 2)).contiguous()) * turn[:, None]
    return torch.view_as_real(z).flatten(-3)


def _exact_rope(c, s):
    n, dh = c["batch"] * c["L"], c["dh"]
    res = {}
    for name in "qk":
        x, w = s[name], s["w_" + name]
        w = w.to(F64).requires_grad_() if w is not None else None
        z, dw = torch.empty(x.shape, dtype=F64, device="cuda"), None
        for i in range(0, n, 16384):
            j = min(n, i + 16384)
            pos = s["pos"][i:j] if s["pos"] is not None else (torch.arange(i, j, device="cuda") % c["L"])[:, None]
            xi = x[i:j].to(F64).requires_grad_()
            zi = _exact_normed(xi, w, _exact_rotation(pos, dh, c["axes"]), dh)
            if not c["backward"]:
                z[i:j] = zi.detach()
                continue
            gr = torch.autograd.grad(zi, (xi,) if w is None else (xi, w), s["d" + name][i:j].to(F64))
            z[i:j] = gr[0]
            if w is not None:
                dw = gr[1] if dw is None else dw + gr[1]
        res[name] = z
        res["w" + name] = dw
    return (res["q"], res["k"], res["wq"], res["wk"]) if c["backward"] else (res["q"], res["k"])


def _exact_window(c, s):
    B, L, H, KV, dh = c["batch"], c["L"], c["heads"], c["kv"], 64
    if work(c)["flops"] > 1.3e12:
        return None
    outs = [torch.zeros(B * L, h * dh, dtype=F64, device="cuda") for h in (H, H, KV, KV)]
    o, dq, dk, dv = (t.view(B, L, -1, dh) for t in outs)
    W, S, g = c["window"] or L, c["sinks"], H // KV
    for b in range(B):
        for h in range(KV):
            q, k, v = (s[n].view(B, L, -1, dh)[b, :, a].to(F64) for n, a in (("q", slice(h * g, h * g + g)),
                                                                            ("k", h), ("v", h)))
            for i0 in range(0, L, 2048):
                i = torch.arange(i0, min(L, i0 + 2048), device="cuda")
                j = torch.arange(int(i[-1]) + 1, device="cuda")
                j = j[(j < S) | (j > i0 - W)]
                leaf = [t.requires_grad_(c["train"]) for t in (q[i], k[j], v[j])]
                sc = torch.einsum("ihd,jd->hij", leaf[0], leaf[1]) / math.sqrt(dh)
                off = (j[None] > i[:, None]) | ((i[:, None] - j[None] >= W) & (j[None] >= S))
                ob = torch.einsum("hij,jd->ihd", torch.softmax(sc.masked_fill(off, -math.inf), -1), leaf[2])
                o[b, i, h * g:h * g + g] = ob.detach()
                if c["train"]:
                    up = s["do"].view(B, L, -1, dh)[b, i, h * g:h * g + g].to(F64)
                    gq, gk, gv = torch.autograd.grad(ob, leaf, up)
                    dq[b, i, h * g:h * g + g] = gq
                    dk[b, j, h] += gk
                    dv[b, j, h] += gv
    return tuple(outs) if c["train"] else outs[0]


def _exact_append(c, s):
    dh, page = c["dh"], c["page"]
    K, V = s["K"].to(F64), s["V"].to(F64)
    lens, table = s["len"].tolist(), s["table"].tolist()
    start = s["start"].tolist() if s["start"] is not None else list(range(c["batch"] + 1))
    q = []
    for b, n in enumerate(lens):
        t0, t1 = start[b], start[b + 1]
        pos = torch.arange(n - (t1 - t0), n, device="cuda")
        turn = _exact_rotation(pos[:, None], dh, 1)
        wq, wk = (None if w is None else w.to(F64) for w in (s["w_q"], s["w_k"]))
        q.append(_exact_normed(s["q"][t0:t1].to(F64), wq, turn, dh))
        k = _exact_normed(s["k"][t0:t1].to(F64), wk, turn, dh).view(t1 - t0, -1, dh)
        v = s["v"][t0:t1].to(F64).view(t1 - t0, -1, dh)
        for p0 in range((n - (t1 - t0)) // page * page, n, page):  # page by page
            sel = (pos >= p0) & (pos < p0 + page)
            pg = table[b][p0 // page]
            K[pg][:, pos[sel] - p0] = k[sel].transpose(0, 1)
            V[pg][:, pos[sel] - p0] = v[sel].transpose(0, 1)
    return torch.cat(q), K, V


def _exact_attend(c, s):
    H, KV, dh, page = c["heads"], c["kv"], c["dh"], c["page"]
    out = torch.zeros(c["batch"], H * dh, dtype=F64, device="cuda")
    for b, n in enumerate(s["len"].tolist()):
        if n == 0:
            continue
        pg = s["table"][b, :-(-n // page)].long()
        j = torch.arange(n, device="cuda")
        hidden = (j < n - c["window"]) & (j >= c["sinks"]) if c["window"] else torch.zeros_like(j, dtype=torch.bool)
        for h in range(KV):
            k, v = (s[x][pg, h].flatten(0, 1)[:n].to(F64) for x in "KV")
            qh = s["q"][b].view(KV, -1, dh)[h].to(F64)
            p = torch.softmax((qh @ k.T / math.sqrt(dh)).masked_fill(hidden, -math.inf), -1)
            out[b].view(KV, -1, dh)[h] = p @ v
    return out


def exact(case, seed):
    s = _inputs(case, seed)
    return {"rope": _exact_rope, "window": _exact_window, "append": _exact_append, "attend": _exact_attend}[
        case["kind"]](case, s)
