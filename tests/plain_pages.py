"""The paged cache in 64 bits on the CPU, from its definition (test infrastructure)."""
import math

import torch

import plain_operators as plain

PAGE, D, TOP = 64, 64, 448.0


def nearest(x):
    """The e4m3 numbers nearest to x, ties to even, |x| <= 448."""
    step = torch.exp2((torch.frexp(x)[1] - 1).clamp(min=-6).double() - 3)
    return torch.round(x / step) * step


def exponent(x):
    """The smallest e in -100 .. 120 with 448 2^e >= |x| for the finite elements."""
    x = x[torch.isfinite(x)].abs()
    top = float(x.max()) if x.numel() else 0.0
    e = -100
    while e < 120 and TOP * 2.0 ** e < top:
        e += 1
    return e


class Pool:
    """What every page and key head stands for: codes (token-major), exponents, bounds."""

    def __init__(self, pages, heads):
        self.k, self.v = (torch.zeros((pages, heads, PAGE, D), dtype=torch.float64) for _ in range(2))
        self.ke, self.ve = (torch.full((pages, heads), -100, dtype=torch.long) for _ in range(2))
        self.bounds = torch.zeros((pages, heads, 2, D), dtype=torch.float64)
        self.written = torch.zeros(pages, dtype=torch.bool)

    def write(self, k, v, begin, table, lengths):
        """k, v [heads][rows][64]; begin, lengths lists, table a list of lists."""
        k, v = k.double(), v.double()
        for s, m in enumerate(lengths):
            n = begin[s + 1] - begin[s]
            t = max(m - n, 0)
            while t < m:
                j, o = t // PAGE, t % PAGE
                end = min(m, (j + 1) * PAGE) - j * PAGE
                p, a = table[s][j], begin[s] + t - (m - n)
                t += end - o
                if not 0 <= p < self.k.shape[0]:
                    continue
                self.written[p] = True
                for h in range(self.k.shape[1]):
                    for x, codes, e in ((k, self.k, self.ke), (v, self.v, self.ve)):
                        x = x[h, a:a + end - o]
                        to = exponent(x)
                        if o:
                            to = max(to, int(e[p, h]))
                            codes[p, h, :o] = nearest(codes[p, h, :o] * 2.0 ** (int(e[p, h]) - to))
                        else:
                            codes[p, h] = 0.0
                        y = nearest(torch.where(torch.isfinite(x), x, 0.0) / 2.0 ** to)
                        codes[p, h, o:end] = torch.where(torch.isfinite(x), y, math.nan)
                        e[p, h] = to
                    c = self.k[p, h, :end]
                    hi = torch.where(torch.isnan(c), -math.inf, c).amax(0)
                    lo = torch.where(torch.isnan(c), math.inf, c).amin(0)
                    self.bounds[p, h, 0] = torch.where(hi < lo, 0.0, torch.ceil(2 * hi))
                    self.bounds[p, h, 1] = torch.where(hi < lo, 0.0, torch.floor(2 * lo))

    def tokens(self, table, m, h):
        """(keys, values, page number) of a sequence's first m tokens; pages that are none are left out, with the tokens' places."""
        at = [t for t in range(m) if 0 <= table[t // PAGE] < self.k.shape[0]]
        p = torch.tensor([table[t // PAGE] for t in at], dtype=torch.long)
        o = torch.tensor([t % PAGE for t in at], dtype=torch.long)
        two = lambda e: torch.exp2(e.double())[:, None]
        return self.k[p, h, o] * two(self.ke[p, h]), self.v[p, h, o] * two(self.ve[p, h]), torch.tensor(at, dtype=torch.long)


def of(pages):
    """The Pool that a pool of the library stands for."""
    pool = Pool(pages.count, pages.kv_heads)
    value = lambda x: x.cpu().float().double()
    pool.k, pool.v = value(pages.k), value(pages.v).transpose(2, 3).contiguous()
    for name, x in (("ke", pages.k_scale), ("ve", pages.v_scale)):
        f, e = torch.frexp(x.cpu())
        setattr(pool, name, e.long() - 1)
    if pages.k_bounds is not None:
        pool.bounds = pages.k_bounds.cpu().double()
    return pool


def limit(i, n, m, causal):
    at = i + m - n
    if at < 0:
        return 0
    return m if causal == 0 else min(m, (at // causal + 1) * causal)


def check_attend(pool, q, got, begin, table, lengths, causal=0, scale=0.125, chosen=None, heads=None):
    """Every row of every sequence against attention in 64 bits, within plain_operators' bounds."""
    out, lse = (x.cpu().double() for x in got)
    q = q.cpu()
    H, rep = q.shape[0], q.shape[0] // pool.k.shape[1]
    for s, m in enumerate(lengths):
        a, n = begin[s], begin[s + 1] - begin[s]
        for h in range(H) if heads is None else heads:
            k, v, at = pool.tokens(table[s], m, h // rep)
            rows = [range(n)] if causal == 0 and chosen is None and n <= m else [[i] for i in range(n)]
            for r in rows:
                if len(r) == 0:
                    continue
                seen = at < limit(r[0], n, m, causal)
                ks, vs = k[seen], v[seen]
                if chosen is not None:
                    parts = [(at[seen] // PAGE == j).nonzero()[:, 0] for j in sorted(set(chosen[a + r[0], h // rep].tolist())) if j >= 0]
                    pick = torch.cat(parts) if parts else torch.zeros(0, dtype=torch.long)
                    ks, vs = ks[pick], vs[pick]
                e = plain.Attention(q[h, a + r[0]:a + r[-1] + 1], ks, vs, 0, scale)
                o, l = out[h, a + r[0]:a + r[-1] + 1], lse[h, a + r[0]:a + r[-1] + 1]
                if not torch.isfinite(e.out).all() or not torch.isfinite(e.lse).all():
                    assert torch.equal(torch.isnan(o), torch.isnan(e.out)), (s, h, list(r))
                    assert torch.equal(torch.isnan(l), torch.isnan(e.lse)) and torch.equal(l == -math.inf, e.lse == -math.inf), (s, h, list(r))
                    fine = ~torch.isnan(e.out)
                    assert bool(((o - e.out).abs()[fine] <= e.out_tol[fine] + 1e-30).all()), (s, h, list(r))
                    continue
                off = (o - e.out).abs()
                assert bool((off <= e.out_tol + 1e-30).all()), (s, h, list(r), float((off / e.out_tol).max()))
                off = (l - e.lse).abs()
                assert bool((off <= e.lse_tol).all()), (s, h, list(r), float((off / e.lse_tol).max()))


def select(pool, q, begin, table, lengths, count, first, last, causal):
    """The choice as lists [rows][kv_heads] of lists."""
    q = q.cpu().double()
    Hk, rep = pool.k.shape[1], q.shape[0] // pool.k.shape[1]
    chosen = {}
    for s, m in enumerate(lengths):
        n = begin[s + 1] - begin[s]
        for i in range(n):
            pages = -(-limit(i, n, m, causal) // PAGE)
            for g in range(Hk):
                ranked = []
                for j in range(pages):
                    p = table[s][j]
                    if not 0 <= p < pool.k.shape[0]:
                        continue
                    if j < first or j >= pages - last:
                        ranked.append((-math.inf, j))
                        continue
                    best = -math.inf
                    for h in range(g * rep, (g + 1) * rep):
                        x = torch.where(torch.isfinite(q[h, begin[s] + i]), q[h, begin[s] + i], 0.0)
                        t = math.floor(math.log2(max(float(x.abs().max()), 2.0 ** -119))) - 7
                        w = torch.round(x / 2.0 ** t)
                        total = float(torch.maximum(w * pool.bounds[p, g, 0], w * pool.bounds[p, g, 1]).sum())
                        best = max(best, total * 2.0 ** min(max(t + int(pool.ke[p, g]) - 1, -100), 100))
                    ranked.append((-best, j))
                kept = sorted(j for _, j in sorted(ranked)[:count])
                chosen[begin[s] + i, g] = kept + [-1] * (count - len(kept))
    return chosen
