"""What the operators around the streaming step are measured on, with their plain forms.

Five operators: the norm of queries and keys per head with the position rotation in the same pass (`xsv.norm_rotate`) and its
gradient (`xsv.norm_rotate_grad`); attention inside sequences with the row sums that a gradient needs (`xsv.seq_attend`) and its
gradient, which recomputes the probabilities (`xsv.seq_attend_grad`); and attention of a few query rows over a layer's
quantized cache (`Context.query_attend`).  Tensors are bf16 `[heads][tokens][64]`, strided views of what a projection wrote
where a model has them so.
"""
import math

import torch

own = False   # False: plain torch operations; True: this package's operators

DEV = "cuda:0"
D = 64        # channels per head: the one head dimension the library is built for

_ROTATE = dict(tokens=1374, heads=16, kv_heads=16, norm="layer", affine=True, eps=1e-5, axes=2, base=100.0, interleaved=False,
               first=0, packed=True)
_SEQ = dict(q_lengths="1374", k_lengths="", heads=16, kv_heads=16, causal=0, behind=0, packed=True)
_QUERY = dict(rows=1, tokens=4096, heads=16, bits=4, group=64, frame=1374)


def _rotate(kind, name, **kw):
    return dict(_ROTATE, kind=kind, name=name, **kw)


def _seq(kind, name, **kw):
    return dict(_SEQ, kind=kind, name=name, **kw)


def _query(name, **kw):
    return dict(_QUERY, kind="query", name=name, **kw)


def listed():
    return [
        # One token, 16 heads: the smallest call there is; launch and host time.
        _rotate("rotate", "rotate-one-token", tokens=1),
        # One frame of the benchmark's model out of the packed projection: layer norm with weights, rows and columns as positions.
        _rotate("rotate", "rotate-frame"),
        # A long sequence with shared key heads at far positions: RMS norm, one position per token.
        _rotate("rotate", "rotate-long", tokens=40000, heads=32, kv_heads=8, norm="rms", axes=1, base=500000.0, first=1000000),
        # Gradient for one frame of a non-square input and an odd head count, pairs side by side.
        _rotate("rotate_grad", "rotate-grad-ragged", tokens=1041, heads=5, kv_heads=5, interleaved=True, packed=False),
        # Gradient for a clip of 24 frames, weights' and biases' gradients among the outputs.
        _rotate("rotate_grad", "rotate-grad-clip", tokens=24 * 1374),
        # Sequences from nothing and one token to a frame in one call, causal by token, three query heads to a key head, rows
        # behind the last sequence.
        _seq("attend", "attend-ragged", q_lengths="1,63,64,0,200,777,1374", heads=12, kv_heads=4, causal=1, behind=37),
        # A training clip of six frames through global attention: a token sees its own frame and those before it.
        _seq("attend", "attend-frame-causal", q_lengths="8244", causal=1374),
        # The ragged call's gradient; queries begin behind cached keys in two of the sequences.
        _seq("attend_grad", "attend-grad-ragged", q_lengths="1,63,64,0,200,777,1374", k_lengths="1,100,64,9,200,1001,1374", heads=12,
             kv_heads=4, causal=1, behind=37),
        # Frame-wise attention of eight frames: the other half of the alternating backbone, in training.
        _seq("attend_grad", "attend-grad-frames", q_lengths=",".join(["1374"] * 8)),
        # The six-frame clip's gradient: the largest.
        _seq("attend_grad", "attend-grad-frame-causal", q_lengths="8244", causal=1374),
        # A single token over the cache of the benchmark's layer (4 bits, groups of 64).
        _query("query-one-token"),
        # A frame's five special tokens over the unpruned cache of a long video.
        _query("query-long-cache", rows=5, tokens=65536),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_one(rng):
    kind = rng.choice(["rotate", "rotate_grad", "attend", "attend_grad", "attend_grad", "query"])
    kv = rng.choice([1, 2, 4, 5, 8, 12, 16])
    heads = kv * rng.choice([1, 1, 1, 2, 3, 4])
    if kind.startswith("rotate"):
        axes = rng.choice([0, 1, 2, 2])
        return dict(_ROTATE, kind=kind, tokens=_log_int(rng, 1, 40000), heads=heads, kv_heads=kv, norm=rng.choice(["layer", "layer", "rms", "none"]),
                    affine=rng.random() < 0.8, eps=rng.choice([1e-5, 1e-6]), axes=axes, base=rng.choice([100.0, 10000.0, 500000.0]),
                    interleaved=rng.random() < 0.3, first=rng.choice([0, 0, 4097, 1000000]), packed=rng.random() < 0.7)
    if kind == "query":
        return dict(_QUERY, kind=kind, rows=_log_int(rng, 1, 200), tokens=_log_int(rng, 64, 65536), heads=rng.randint(1, 16),
                    bits=rng.choice([4, 4, 4, 2, 16]), group=rng.choice([64, 64, 32]), frame=rng.choice([1, 59, 64]))
    if rng.random() < 0.5:      # a clip: frames alone, or behind each other
        n, frames = _log_int(rng, 33, 1374), rng.randint(1, 6)
        if rng.random() < 0.5:
            q, causal = [n] * frames, 0
        else:
            q, causal = [n * frames], n
        k = list(q)
    else:                       # sequences of any length, some behind cached keys
        q = [0 if rng.random() < 0.1 else _log_int(rng, 1, 2000) for _ in range(rng.randint(1, 8))]
        k = [x if rng.random() < 0.6 else x + _log_int(rng, 1, 2000) for x in q]
        causal = rng.choice([0, 1, 1, 59, 777])
        if rng.random() < 0.2:  # more queries than keys: the first of them see nothing
            k[0] = q[0] // 2
    return dict(_SEQ, kind=kind, q_lengths=",".join(map(str, q)), k_lengths=",".join(map(str, k)), heads=heads, kv_heads=kv,
                causal=causal, behind=rng.choice([0, 0, 5, 130]), packed=rng.random() < 0.7)


def draw(rng):
    most = {k: max(max(work(c)["flops"] / 1e3, work(c)["bytes"]) for c in listed() if c["kind"] == k)
            for k in ("rotate", "rotate_grad", "attend", "attend_grad", "query")}
    while True:
        c = _draw_one(rng)
        w = work(c)
        if w["bytes"] > 0 and max(w["flops"] / 1e3, w["bytes"]) <= most[c["kind"]]:
            return c


# ---- what a pass cannot do without ---------------------------------------------------------------------------------

def _lengths(c):
    q = [int(x) for x in c["q_lengths"].split(",")]
    k = [int(x) for x in c["k_lengths"].split(",")] if c["k_lengths"] else list(q)
    return q, k


def _visible(n, m, causal):
    """Pairs of n queries and m keys that see each other; query i stands at key position i + m - n."""
    if not causal:
        return n * m
    pairs = 0
    for pos in range(max(m - n, 0), m):
        pairs += min(m, (pos // causal + 1) * causal)
    return pairs


def work(case):
    c = case
    if c["kind"].startswith("rotate"):
        rows = c["tokens"] * (c["heads"] + c["kv_heads"])
        grad = c["kind"] == "rotate_grad"
        weights = 4 * 4 * D if c["affine"] and c["norm"] != "none" else 0
        return {"bytes": rows * D * 2 * (3 if grad else 2) + 4 * c["axes"] * c["tokens"] + weights * (2 if grad else 1),
                "flops": rows * D * (24 if grad else 12)}
    if c["kind"] == "query":
        H, T, m = c["heads"], c["tokens"], c["rows"]
        row = 2.0 if c["bits"] == 16 else c["bits"] / 8.0 + 8.0 / c["group"]
        return {"bytes": 2 * row * H * T * D + 2 * 2 * H * m * D + 4 * H * m, "flops": 4 * D * H * m * T}
    q, k = _lengths(c)
    pairs = sum(_visible(a, b, c["causal"]) for a, b in zip(q, k))
    nq, nk, H, Hk = sum(q), sum(k), c["heads"], c["kv_heads"]
    if c["kind"] == "attend":
        return {"bytes": 2 * D * (2 * nq * H + 2 * nk * Hk) + 4 * nq * H, "flops": 4 * D * H * pairs}
    return {"bytes": 2 * D * (4 * nq * H + 4 * nk * Hk) + 4 * nq * H, "flops": 10 * D * H * pairs}


# ---- inputs ---------------------------------------------------------------------------------------------------------

class _Source:
    def __init__(self, seed):
        self.g = torch.Generator(device=DEV).manual_seed(seed)

    def normal(self, *shape, scale=1.0):
        return torch.randn(shape, generator=self.g, device=DEV) * scale

    def heads(self, tokens, counts, packed, scales):
        """One bf16 `[heads][tokens][64]` tensor per count: views of one projection's output, or tensors of their own."""
        if packed:
            x = self.normal(tokens, sum(counts), D)
            at = 0
            for n, s in zip(counts, scales):
                x[:, at:at + n] *= s
                at += n
            x = x.to(torch.bfloat16).transpose(0, 1)
            return list(x.split(counts))
        return [(self.normal(n, tokens, D) * s).to(torch.bfloat16) for n, s in zip(counts, scales)]


def _outliers(src):
    """Gains per channel: keys carry a few channels of larger values."""
    g = torch.ones(D, device=DEV)
    g[torch.randperm(D, generator=src.g, device=DEV)[:6]] = 3.0
    return g


def prepare(case, seed):
    c, src = case, _Source(seed)
    if c["kind"].startswith("rotate"):
        n, axes = c["tokens"], c["axes"]
        one = torch.ones(D, device=DEV)
        q, k = src.heads(n, [c["heads"], c["kv_heads"]], c["packed"], [one, _outliers(src)])
        positions = None
        if axes == 1:
            positions = (torch.arange(n, device=DEV) + c["first"]).to(torch.int32).view(n, 1)
        elif axes == 2:   # rows and columns of patches, 37 to a row
            t = torch.arange(n, device=DEV) + c["first"]
            positions = torch.stack([t // 37, t % 37], 1).to(torch.int32).contiguous()
        weights = [None] * 4
        if c["affine"] and c["norm"] != "none":
            w = [1.0 + src.normal(D, scale=0.2), src.normal(D, scale=0.1), 1.0 + src.normal(D, scale=0.2), src.normal(D, scale=0.1)]
            weights = w if c["norm"] == "layer" else [w[0], None, w[2], None]
        st = dict(case=c, q=q, k=k, positions=positions, weights=weights)
        st["out"] = [torch.empty(q.shape, dtype=q.dtype, device=DEV), torch.empty(k.shape, dtype=k.dtype, device=DEV)]
        if c["kind"] == "rotate_grad":
            st["dq_out"], st["dk_out"] = src.heads(n, [c["heads"], c["kv_heads"]], False, [0.1, 0.1])
        return st
    if c["kind"] == "query":
        return _prepare_query(c, src)
    lq, lk = _lengths(c)
    nq, nk = sum(lq) + c["behind"], sum(lk) + c["behind"]
    H, Hk = c["heads"], c["kv_heads"]
    one = torch.ones(D, device=DEV)
    if nq == nk and c["packed"]:
        q, k, v = src.heads(nq, [H, Hk, Hk], True, [one, _outliers(src), one])
    else:
        q, = src.heads(nq, [H], c["packed"], [one])
        k, v = src.heads(nk, [Hk, Hk], c["packed"], [_outliers(src), one])
    begin = lambda ls: torch.tensor([sum(ls[:i]) for i in range(len(ls) + 1)], dtype=torch.int32, device=DEV)
    st = dict(case=c, q=q, k=k, v=v, q_begin=begin(lq), k_begin=begin(lk), lengths=(lq, lk), longest=(max(lq), max(lk)))
    st["out"] = torch.zeros((H, nq, D), dtype=torch.bfloat16, device=DEV)
    st["lse"] = torch.zeros((H, nq), dtype=torch.float32, device=DEV)
    if c["kind"] == "attend_grad":
        out, lse = _attend_plain(q, k, v, lq, lk, c["causal"])
        st["out"].copy_(out)
        st["lse"].copy_(lse)
        st["dout"], = src.heads(nq, [H], False, [0.1])
        st["grads"] = [torch.zeros((h, n, D), dtype=torch.bfloat16, device=DEV) for h, n in ((H, nq), (Hk, nk), (Hk, nk))]
    return st


def _quantize(x, bits, G, axis):
    """Codes, scales and zero points of bf16 rows [H][T][64]: groups of G tokens per channel (axis 1) or of G channels per
    token (axis 2)."""
    H, T, _ = x.shape
    x = x.float()
    pad = (-x.shape[axis]) % G
    if pad:   # a short last group by itself: repeat its last row, which changes neither extreme
        x = torch.cat([x, x[:, -1:].expand(H, pad, D)], 1)
    shape = (H, x.shape[1] // G, G, D) if axis == 1 else (H, T, D // G, G)
    g = x.view(shape)
    dim = 2 if axis == 1 else 3
    lo, hi = g.amin(dim, keepdim=True), g.amax(dim, keepdim=True)
    s = (hi - lo) / float((1 << bits) - 1)
    s = torch.where(s == 0, torch.ones_like(s), s)
    z = torch.round(-lo / s)
    codes = (torch.round(g / s) + z).clamp_(0, (1 << bits) - 1).to(torch.uint8)
    codes = codes.view(H, -1, D)[:, :T].contiguous()
    return codes, s.squeeze(dim).contiguous(), z.squeeze(dim).contiguous()


def _prepare_query(c, src):
    H, T, m, G = c["heads"], c["tokens"], c["rows"], c["group"]
    q = src.normal(H, m, D).to(torch.bfloat16)
    k = (src.normal(H, T, D) * _outliers(src)).to(torch.bfloat16)
    v = src.normal(H, T, D).to(torch.bfloat16)
    st = dict(case=c, q=q, out=torch.empty((H, m, D), dtype=torch.bfloat16, device=DEV), lse=torch.empty((H, m), device=DEV))
    if c["bits"] == 16:
        st["rows"] = (k, v)
    else:
        st["keys"], st["values"] = _quantize(k, c["bits"], G, 1), _quantize(v, c["bits"], G, 2)
    if own:
        import numpy as np
        from paper_2602_21780_amd import xsv
        n = min(c["frame"], T)
        ctx = xsv.Context(1, H, D, n, 0, 0, c["bits"], G, max_frames=-(-T // n))
        host = lambda t: t.cpu().numpy()
        ids = np.arange(T, dtype=np.int32)
        if c["bits"] == 16:
            raw = [t.view(torch.int16).cpu().numpy().view(np.uint16) for t in (k, v)]
            dump = xsv.CacheDump(T, None, None, None, None, None, None, raw[0], raw[1], ids // n, ids % n)
        else:
            dump = xsv.CacheDump(T, *[host(t) for t in st["keys"]], *[host(t) for t in st["values"]], None, None, ids // n, ids % n)
        ctx.cache_import(0, dump, -(-T // n))
        st["ctx"] = ctx
    return st


# ---- the plain forms ------------------------------------------------------------------------------------------------

def _angles(positions, base):
    """cos and sin, fp32 [tokens][64 / (2 axes)] per axis; angles in 64 bits."""
    axes = positions.shape[1]
    half = D // (2 * axes)
    freq = base ** (-torch.arange(half, dtype=torch.float64, device=DEV) / half)
    a = positions.double()[:, :, None] * freq
    return a.cos().float(), a.sin().float()


def _turn(x, cos, sin, interleaved):
    """Rotates fp32 [heads][tokens][64] by [tokens][axes][half]."""
    H, n, _ = x.shape
    axes, half = cos.shape[1], cos.shape[2]
    if interleaved:
        x = x.view(H, n, axes, half, 2)
        a, b = x[..., 0], x[..., 1]
        return torch.stack([a * cos - b * sin, b * cos + a * sin], -1).view(H, n, D)
    x = x.view(H, n, axes, 2, half)
    a, b = x[..., 0, :], x[..., 1, :]
    return torch.stack([a * cos - b * sin, b * cos + a * sin], -2).view(H, n, D)


def _norm(x, norm, eps):
    """(x normalized, 1 / its deviation)."""
    if norm == "none":
        return x, None
    if norm == "layer":
        x = x - x.mean(-1, keepdim=True)
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + eps)
    return x * r, r


def _rotate_plain(st):
    c, outs = st["case"], []
    turn = _angles(st["positions"], c["base"]) if c["axes"] else None
    for x, w, b in ((st["q"], *st["weights"][:2]), (st["k"], *st["weights"][2:])):
        y, _ = _norm(x.float(), c["norm"], c["eps"])
        if w is not None:
            y = y * w
        if b is not None:
            y = y + b
        if turn is not None:
            y = _turn(y.contiguous(), *turn, c["interleaved"])
        outs.append(y.to(torch.bfloat16))
    return outs


def _rotate_grad_plain(st):
    c, grads, weights = st["case"], [], []
    turn = _angles(st["positions"], c["base"]) if c["axes"] else None
    for x, dy, w in ((st["q"], st["dq_out"], st["weights"][0]), (st["k"], st["dk_out"], st["weights"][2])):
        g = dy.float()
        if turn is not None:
            g = _turn(g.contiguous(), turn[0], -turn[1], c["interleaved"])
        xhat, r = _norm(x.float(), c["norm"], c["eps"])
        weights += [(g * xhat).sum((0, 1)), g.sum((0, 1))]
        if w is not None:
            g = g * w
        if c["norm"] == "layer":
            g = g - g.mean(-1, keepdim=True)
        if r is not None:
            g = r * (g - xhat * (g * xhat).mean(-1, keepdim=True))
        grads.append(g.to(torch.bfloat16))
    return grads + [torch.stack(weights)]


def _mask(n, m, causal):
    """True where query i (key position i + m - n) sees key j."""
    if not causal:
        return None
    pos = torch.arange(n, device=DEV) + (m - n)
    limit = torch.where(pos < 0, torch.zeros_like(pos), (torch.div(pos, causal, rounding_mode="floor") + 1) * causal)
    return torch.arange(m, device=DEV)[None, :] < limit[:, None]


def _head_runs(H, n, m):
    """Runs of heads whose logits stay under a few GB."""
    step = max(1, min(H, (1 << 29) // max(n * m, 1)))
    return [(h, min(H, h + step)) for h in range(0, H, step)]


def _attend_plain(q, k, v, lq, lk, causal):
    H, rep = q.shape[0], q.shape[0] // k.shape[0]
    out = torch.zeros((H, q.shape[1], D), dtype=torch.bfloat16, device=DEV)
    lse = torch.zeros((H, q.shape[1]), device=DEV)
    a = b = 0
    for n, m in zip(lq, lk):
        mask = _mask(n, m, causal)
        for h0, h1 in _head_runs(H, n, m) if n else ():
            if m == 0:
                lse[h0:h1, a:a + n] = -math.inf
                continue
            kv = [h // rep for h in range(h0, h1)]
            s = (q[h0:h1, a:a + n].float() @ k[kv, b:b + m].float().transpose(1, 2).contiguous()) * 0.125
            if mask is not None:
                s = s.masked_fill(~mask, -math.inf)
            top = s.amax(-1, keepdim=True)
            top = torch.where(top == -math.inf, torch.zeros_like(top), top)
            p = torch.exp(s - top)
            total = p.sum(-1, keepdim=True)
            o = (p @ v[kv, b:b + m].float()) / torch.where(total == 0, torch.ones_like(total), total)
            out[h0:h1, a:a + n] = o.to(torch.bfloat16)
            lse[h0:h1, a:a + n] = (top + torch.log(total))[..., 0]
        a, b = a + n, b + m
    return out, lse


def _attend_grad_plain(st):
    c = st["case"]
    q, k, v, out, lse, dout = (st[x] for x in ("q", "k", "v", "out", "lse", "dout"))
    H, Hk = c["heads"], c["kv_heads"]
    rep = H // Hk
    dq = torch.zeros((H, q.shape[1], D), dtype=torch.bfloat16, device=DEV)
    dk = torch.zeros((Hk, k.shape[1], D), device=DEV)
    dv = torch.zeros((Hk, k.shape[1], D), device=DEV)
    a = b = 0
    for n, m in zip(*st["lengths"]):
        mask = _mask(n, m, c["causal"])
        for h0, h1 in _head_runs(H, n, m) if n and m else ():
            kv = [h // rep for h in range(h0, h1)]
            qs, ks, vs = q[h0:h1, a:a + n].float(), k[kv, b:b + m].float(), v[kv, b:b + m].float()
            do = dout[h0:h1, a:a + n].float()
            p = torch.exp((qs @ ks.transpose(1, 2).contiguous()) * 0.125 - lse[h0:h1, a:a + n, None])
            if mask is not None:
                p = p.masked_fill(~mask, 0.0)
            delta = (do * out[h0:h1, a:a + n].float()).sum(-1, keepdim=True)
            ds = p * (do @ vs.transpose(1, 2).contiguous() - delta) * 0.125
            dq[h0:h1, a:a + n] = (ds @ ks).to(torch.bfloat16)
            pv, pk = p.transpose(1, 2).contiguous() @ do, ds.transpose(1, 2).contiguous() @ qs
            for i, g in enumerate(kv):
                dv[g, b:b + m] += pv[i]
                dk[g, b:b + m] += pk[i]
        a, b = a + n, b + m
    return [dq, dk.to(torch.bfloat16), dv.to(torch.bfloat16)]


def _view(codes, scale, zero, G, axis):
    """The cache's dequantized rows: an exact difference, one product in 32 bits, one rounding to bf16."""
    rep = lambda t: t.repeat_interleave(G, axis)[:, :codes.shape[1]]
    return ((codes.float() - rep(zero)) * rep(scale)).to(torch.bfloat16)


def _cache_rows(st):
    if "rows" in st:
        return st["rows"]
    G = st["case"]["group"]
    return _view(*st["keys"], G, 1), _view(*st["values"], G, 2)


def _query_plain(st):
    k, v = _cache_rows(st)
    s = (st["q"].float() @ k.float().transpose(1, 2).contiguous()) * 0.125
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - top)
    total = p.sum(-1, keepdim=True)
    return [((p @ v.float()) / total).to(torch.bfloat16), (top + torch.log(total))[..., 0]]


# ---- one pass -------------------------------------------------------------------------------------------------------

def run(state):
    c = state["case"]
    if not own:
        if c["kind"] == "rotate":
            return _rotate_plain(state)
        if c["kind"] == "rotate_grad":
            return _rotate_grad_plain(state)
        if c["kind"] == "attend":
            return list(_attend_plain(state["q"], state["k"], state["v"], *state["lengths"], c["causal"]))
        if c["kind"] == "attend_grad":
            return _attend_grad_plain(state)
        return _query_plain(state)
    from paper_2602_21780_amd import xsv
    if c["kind"].startswith("rotate"):
        qw, qb, kw, kb = state["weights"]
        form = dict(norm=c["norm"], eps=c["eps"], q_weight=qw, q_bias=qb, k_weight=kw, k_bias=kb, positions=state["positions"],
                    base=c["base"], interleaved=c["interleaved"])
        if c["kind"] == "rotate":
            return list(xsv.norm_rotate(state["q"], state["k"], out=state["out"], **form))
        return list(xsv.norm_rotate_grad(state["dq_out"], state["dk_out"], state["q"], state["k"], out=state["out"], **form))
    if c["kind"] == "query":
        return list(state["ctx"].query_attend(0, state["q"], out=state["out"], lse=state["lse"]))
    form = dict(q_begin=state["q_begin"], k_begin=state["k_begin"], longest_q=state["longest"][0], longest_k=state["longest"][1],
                causal=c["causal"])
    if c["kind"] == "attend":
        return list(xsv.seq_attend(state["q"], state["k"], state["v"], out=state["out"], lse=state["lse"], **form))
    return list(xsv.seq_attend_grad(state["dout"], state["q"], state["k"], state["v"], state["out"], state["lse"],
                                    grads=state["grads"], **form))


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------

def _turn_matrix(position, axes, base, interleaved):
    """The rotations of tokens as [tokens][64][64]: y = R x."""
    n, width = position.shape[0], D // axes
    R = torch.zeros((n, D, D), dtype=torch.float64, device=DEV)
    for ax in range(axes):
        for i in range(width // 2):
            a = position[:, ax].double() * base ** (-2.0 * i / width)
            u = ax * width + (2 * i if interleaved else i)
            w = u + (1 if interleaved else width // 2)
            R[:, u, u] = R[:, w, w] = torch.cos(a)
            R[:, u, w], R[:, w, u] = -torch.sin(a), torch.sin(a)
    return R


def _exact_rotate(st):
    c = st["case"]
    n, chunk = c["tokens"], 4096
    grad = c["kind"] == "rotate_grad"
    parts, wsum = [[], []], torch.zeros((4, D), dtype=torch.float64, device=DEV)
    for t0 in range(0, n, chunk):
        t = slice(t0, min(n, t0 + chunk))
        R = _turn_matrix(st["positions"][t], c["axes"], c["base"], c["interleaved"]) if c["axes"] else None
        for i, x in enumerate((st["q"], st["k"])):
            w, b = st["weights"][2 * i], st["weights"][2 * i + 1]
            x = x[:, t].double()
            mean = x.mean(-1, keepdim=True) if c["norm"] == "layer" else torch.zeros_like(x[..., :1])
            dev = torch.sqrt(((x - mean) ** 2).mean(-1, keepdim=True) + c["eps"]) if c["norm"] != "none" else torch.ones_like(x[..., :1])
            hat = (x - mean) / dev
            scale = w.double() if w is not None else torch.ones(D, dtype=torch.float64, device=DEV)
            if not grad:
                y = hat * scale + (b.double() if b is not None else 0.0)
                if R is not None:
                    y = torch.matmul(y.transpose(0, 1), R.transpose(1, 2).contiguous()).transpose(0, 1)
                parts[i].append(y)
                continue
            g = (st["dq_out"], st["dk_out"])[i][:, t].double()
            if R is not None:   # the transposed rotation
                g = torch.matmul(g.transpose(0, 1).contiguous(), R).transpose(0, 1)
            wsum[2 * i] += (g * hat).sum((0, 1))
            wsum[2 * i + 1] += g.sum((0, 1))
            g = g * scale
            if c["norm"] != "none":
                dot = (g * hat).sum(-1, keepdim=True) / D
                g = (g - (g.sum(-1, keepdim=True) / D if c["norm"] == "layer" else 0.0) - hat * dot) / dev
            parts[i].append(g)
    outs = [torch.cat(p, 1) for p in parts]
    return outs + [wsum] if grad else outs


def _exact_attend(st):
    c = st["case"]
    grad = c["kind"] == "attend_grad"
    H, Hk, causal = c["heads"], c["kv_heads"], c["causal"]
    q, k, v = st["q"], st["k"], st["v"]
    f64 = dict(dtype=torch.float64, device=DEV)
    out, lse = torch.zeros((H, q.shape[1], D), **f64), torch.zeros((H, q.shape[1]), **f64)
    dq, dk, dv = torch.zeros_like(out), torch.zeros((Hk, k.shape[1], D), **f64), torch.zeros((Hk, k.shape[1], D), **f64)
    starts_q, starts_k = st["q_begin"].tolist(), st["k_begin"].tolist()
    for a, a1, b, b1 in zip(starts_q, starts_q[1:], starts_k, starts_k[1:]):
        n, m = a1 - a, b1 - b
        for h in range(H if n else 0):
            g = h * Hk // H
            if m == 0:
                lse[h, a:a1] = -math.inf
                continue
            Q, K, V = q[h, a:a1].double(), k[g, b:b1].double(), v[g, b:b1].double()
            S = torch.mm(Q, K.t()) / math.sqrt(D)
            if causal:
                place = torch.arange(m - n, m, device=DEV)
                frame_q, frame_k = torch.floor(place / causal), torch.arange(m, device=DEV) // causal
                S[(frame_k[None, :] > frame_q[:, None]) | (place < 0)[:, None]] = -math.inf
            L = torch.logsumexp(S, -1)
            empty = L == -math.inf
            P = torch.exp(S - torch.where(empty, torch.zeros_like(L), L)[:, None])
            O = torch.mm(P, V)
            if not grad:
                out[h, a:a1], lse[h, a:a1] = O, L
                continue
            dO = st["dout"][h, a:a1].double()
            dP = torch.mm(dO, V.t())
            dS = P * (dP - (dO * O).sum(-1, keepdim=True)) / math.sqrt(D)
            dq[h, a:a1] = torch.mm(dS, K)
            dk[g, b:b1] += torch.mm(dS.t(), Q)
            dv[g, b:b1] += torch.mm(P.t(), dO)
    return [dq, dk, dv] if grad else [out, lse]


def _exact_query(st):
    q, (k, v) = st["q"].double(), _cache_rows(st)
    outs, sums = [], []
    for h in range(q.shape[0]):
        S = torch.mm(q[h], k[h].double().t()) / math.sqrt(D)
        L = torch.logsumexp(S, -1)
        outs.append(torch.mm(torch.exp(S - L[:, None]), v[h].double()))
        sums.append(L)
    return [torch.stack(outs), torch.stack(sums)]


def exact(case, seed):
    global own
    was, own = own, False     # the inputs alone
    try:
        st = prepare(case, seed)
    finally:
        own = was
    if case["kind"].startswith("rotate"):
        return _exact_rotate(st)
    return _exact_query(st) if case["kind"] == "query" else _exact_attend(st)
