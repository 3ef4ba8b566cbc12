"""seq_attend and its gradient against their definition in 64 bits (plain_operators.Attention, which derives the tolerances)."""
import ctypes as C
import math

import pytest
import torch

import plain_operators as plain
from paper_2602_21780_amd import xsv

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _begin(lengths):
    b = [0]
    for n in lengths:
        b.append(b[-1] + n)
    return torch.tensor(b, dtype=torch.int32, device=DEV)


def _inputs(lq, lk, heads, kv, behind=0, seed=0, scale=1.0, packed=True):
    g = torch.Generator().manual_seed(seed)
    nq, nk = sum(lq) + behind, sum(lk) + behind
    make = lambda h, n, s: (torch.randn((n, h, 64), generator=g) * s).to(torch.bfloat16).to(DEV).transpose(0, 1)
    q, k, v, d = make(heads, nq, scale), make(kv, nk, scale), make(kv, nk, 1.0), make(heads, nq, 0.3)
    return [t if packed else t.contiguous() for t in (q, k, v, d)]


def _run(q, k, v, d, lq, lk, causal=0, scale=0.0, longest=True):
    form = dict(q_begin=_begin(lq), k_begin=_begin(lk), causal=causal, softmax_scale=scale)
    if longest:
        form.update(longest_q=max(lq), longest_k=max(lk))
    out, lse = xsv.seq_attend(q, k, v, **form)
    grads = xsv.seq_attend_grad(d, q, k, v, out, lse, **form)
    torch.cuda.synchronize()
    return out, lse, grads


def _close(name, got, want, tol):
    got = got.double()
    assert torch.equal(got.isnan(), want.isnan()), name
    off = torch.where(want.isfinite(), (got - want).abs(), torch.zeros_like(want))
    assert torch.equal(got[~want.isfinite() & ~want.isnan()], want[~want.isfinite() & ~want.isnan()]), name
    worst = (off / (tol + 1e-30)).nan_to_num(0.0).max() if off.numel() else 0.0
    assert float(worst) <= 1.0, (name, float(worst), float(off.max()))


def _check(q, k, v, d, lq, lk, causal, scale, got, sequences=None, heads=None):
    """Every (sequence, key head) against 64 bits."""
    out, lse, (dq, dk, dv) = got
    H, Hk = q.shape[0], k.shape[0]
    rep = H // Hk
    scale = scale or 0.125
    cpu = [t.cpu() for t in (q, k, v, d, out, lse, dq, dk, dv)]
    q, k, v, d, out, lse, dq, dk, dv = cpu
    a = b = 0
    for s, (n, m) in enumerate(zip(lq, lk)):
        for g in range(Hk):
            if (sequences is not None and s not in sequences) or (heads is not None and g not in heads):
                continue
            K, V = k[g, b:b + m], v[g, b:b + m]
            zero = torch.zeros((m, 64), dtype=torch.float64)
            sums = [zero.clone(), zero.clone(), zero.clone(), zero.clone()]
            for h in range(g * rep, (g + 1) * rep):
                e = plain.Attention(q[h, a:a + n], K, V, causal, scale, d[h, a:a + n])
                where = f"sequence {s} ({n}, {m}) head {h}"
                _close("out " + where, out[h, a:a + n], e.out, e.out_tol)
                _close("lse " + where, lse[h, a:a + n], e.lse, e.lse_tol)
                _close("dq " + where, dq[h, a:a + n], e.dq, e.dq_tol)
                for x, y in zip(sums, (e.dk, e.dk_tol, e.dv, e.dv_tol)):
                    x += y
            _close(f"dk sequence {s} ({n}, {m}) key head {g}", dk[g, b:b + m], sums[0], sums[1] + 2.0 ** -8 * sums[0].abs())
            _close(f"dv sequence {s} ({n}, {m}) key head {g}", dv[g, b:b + m], sums[2], sums[3] + 2.0 ** -8 * sums[2].abs())
        a, b = a + n, b + m


LENGTHS = [
    ([1], [1]), ([1], [200]), ([31], [31]), ([64], [64]), ([65], [129]), ([300], [300]), ([70, 1, 0, 129], [70, 1, 0, 129]),
    ([5, 0, 40, 128], [90, 7, 40, 191]), ([50, 130], [20, 130]), ([3, 33], [0, 33]),
]


@pytest.mark.parametrize("causal", [0, 1, 7, 64, 100000])
@pytest.mark.parametrize("lq,lk", LENGTHS)
def test_lengths_and_masks(lq, lk, causal):
    print(f"seq_attend {lq} {lk} causal={causal}", flush=True)
    heads, kv = (4, 2) if sum(lq) < 100 else (2, 1)
    x = _inputs(lq, lk, heads, kv, seed=sum(lq) + causal)
    _check(*x, lq, lk, causal, 0.0, _run(*x, lq, lk, causal))


@pytest.mark.parametrize("heads,kv", [(1, 1), (5, 5), (6, 1), (12, 4)])
@pytest.mark.parametrize("scale", [0.0, 0.02, 1.0])
def test_heads_shared_keys_and_scales(heads, kv, scale):
    lq, lk = [77, 40], [99, 40]
    x = _inputs(lq, lk, heads, kv, seed=heads, packed=False)
    _check(*x, lq, lk, 1, scale, _run(*x, lq, lk, 1, scale))


@pytest.mark.parametrize("causal,n", [(0, 300), (1, 300), (150, 300), (0, 512), (1, 500)])
def test_many_sequences_at_once(causal, n):
    """Launches large enough for the larger blocks of rows; the lengths' bounds left to the library."""
    lq = [n] * 31 + [n - 45]
    x = _inputs(lq, lq, 16, 16, seed=n + causal)
    _check(*x, lq, lq, causal, 0.0, _run(*x, lq, lq, causal), sequences=(0, 31), heads=(0, 9))
    whole = _run(*x, lq, lq, causal)
    loose = _run(*x, lq, lq, causal, longest=False)
    for a, b in zip((*whole[:2], *whole[2]), (*loose[:2], *loose[2])):
        assert torch.equal(a, b)


@pytest.mark.parametrize("lq,lk,heads,kv,causal", [([4500], [4500], 2, 1, 1), ([3600, 4100], [3600, 4203], 2, 2, 0), ([3521], [9000], 1, 1, 1500),
                                                   ([7001], [3500], 1, 1, 1), ([5000], [5000], 4, 4, 1000)])
def test_long_sequences(lq, lk, heads, kv, causal):
    """Lengths at which the gradient takes blocks of 256 rows, and workgroups share the tiles of the forward pass and of both gradients."""
    print(f"seq_attend {lq} {lk} heads={heads} causal={causal}", flush=True)
    x = _inputs(lq, lk, heads, kv, seed=sum(lq) + causal, behind=5)
    _check(*x, lq, lk, causal, 0.0, _run(*x, lq, lk, causal), heads=(heads - 1,) if kv == heads else None)


def test_more_sequences_than_rows():
    """Nearly all of 3000 sequences empty, one long among them; and 700 of one to nine tokens."""
    lq = [0] * 2000 + [400] + [0] * 999
    x = _inputs(lq, lq, 2, 1, seed=2)
    _check(*x, [400], [400], 1, 0.0, _run(*x, lq, lq, 1))
    lq = [1 + i % 9 for i in range(700)]
    lk = [1 + (3 * i) % 11 for i in range(700)]
    x = _inputs(lq, lk, 4, 2, seed=3)
    _check(*x, lq, lk, 1, 0.0, _run(*x, lq, lk, 1), sequences=range(0, 700, 37))


def test_frame_causal_clip():
    lq = [6 * 239]
    x = _inputs(lq, lq, 3, 3, seed=8)
    _check(*x, lq, lq, 239, 0.0, _run(*x, lq, lq, 239), heads=(1,))


def test_long_keys_few_queries():
    lq, lk = [3, 130], [5000, 7001]
    x = _inputs(lq, lk, 2, 1, seed=4)
    _check(*x, lq, lk, 1, 0.0, _run(*x, lq, lk, 1))


def test_rows_in_no_sequence_are_neither_read_nor_written():
    """Rows in front of the first, between and behind the sequences: NaN inside, and as they were outside."""
    lens = [40, 70]
    q, k, v, d = _inputs([160], [160], 2, 2, seed=3)
    q, k, v, d = (t.clone() for t in (q, k, v, d))
    outside = torch.ones(160, dtype=torch.bool, device=DEV)
    outside[10:50] = outside[50:120] = False
    clean = [t.clone() for t in (q, k, v, d)]
    for t in (q, k, v, d):
        t[:, outside] = float("nan")
    begin = torch.tensor([10, 50, 120], dtype=torch.int32, device=DEV)
    form = dict(q_begin=begin, causal=1, longest_q=70, longest_k=70)
    marks = [torch.full((2, 160, 64), 5.0, dtype=torch.bfloat16, device=DEV) for _ in range(4)]
    lse = torch.full((2, 160), 5.0, device=DEV)
    xsv.seq_attend(q, k, v, out=marks[0], lse=lse, **form)
    xsv.seq_attend_grad(d, q, k, v, marks[0], lse, grads=marks[1:], **form)
    want = _run(*[t[:, ~outside] for t in clean], lens, lens, 1)
    for m, w in zip((marks[0], lse, *marks[1:]), (*want[:2], *want[2])):
        assert torch.equal(m[:, ~outside], w) and bool((m[:, outside] == 5.0).all())


def test_offsets_outside_the_tensors_are_cut_off():
    """Offsets are device data: what they name outside the tensors, or backwards, is left out; the rest is as ever."""
    q, k, v, d = _inputs([100], [100], 2, 1, seed=5)
    for begin, lens in (([-50, 60, 1 << 30], ([60, 40], [60, 40])), ([0, 60, 40, 100], None)):
        b = torch.tensor(begin, dtype=torch.int32, device=DEV)
        out, lse = xsv.seq_attend(q, k, v, b, causal=1)
        grads = xsv.seq_attend_grad(d, q, k, v, out, lse, b, causal=1)
        torch.cuda.synchronize()
        assert all(bool(t.isfinite().all()) for t in (out, lse, *grads))
        if lens is not None:
            want = _run(q, k, v, d, *lens, 1)
            for a, w in zip((out, lse, *grads), (*want[:2], *want[2])):
                assert torch.equal(a, w)


@pytest.mark.parametrize("n,at", [(300, 141), (1300, 700), (3700, 1999)])  # (1300: workgroups share the tiles, 3700: blocks of 256 rows)
@pytest.mark.parametrize("what", ["nan", "inf", "-inf"])
def test_values_that_are_not_finite_stay_where_they_are_seen(what, n, at):
    """NaN and infinities in keys, values, queries and dout of a causal sequence, in tiles that the mask cuts: queries in front of
    them, and the gradients of keys behind the last query that sees them, are what they are without them."""
    q, k, v, d = [t.clone() for t in _inputs([n], [n], 2, 2, seed=6)]
    clean = _run(q, k, v, d, [n], [n], 1)
    x = float(what)
    # a value and a key: queries in front of `at` do not see them
    for name in ("v", "k"):
        bad = dict(q=q, k=k, v=v, d=d)
        bad[name] = bad[name].clone()
        bad[name][1, at, 5] = x
        got = _run(*bad.values(), [n], [n], 1)
        for a, b in zip((*got[:2], got[2][0]), (*clean[:2], clean[2][0])):
            assert torch.equal(a[0], b[0]) and torch.equal(a[1, :at], b[1, :at]), name
        if name == "v":   # one channel of every query that sees it
            bad_channel = got[0][1, at:, 5]
            assert bool((bad_channel.isnan() if what == "nan" else bad_channel == x).all())
            rest = torch.arange(64, device=DEV) != 5
            assert torch.equal(got[0][1, at:][:, rest], clean[0][1, at:][:, rest])
    # a query's dout: keys behind it are not seen by it
    bad_d = d.clone()
    bad_d[1, at, 9] = x
    got = _run(q, k, v, bad_d, [n], [n], 1)
    for a, b in zip(got[2][1:], clean[2][1:]):
        assert torch.equal(a[0], b[0]) and torch.equal(a[1, at + 1:], b[1, at + 1:])
        assert bool((~a[1, :at + 1].isfinite()).any(-1).all())
    assert torch.equal(got[2][0][1, :at], clean[2][0][1, :at]) and torch.equal(got[2][0][1, at + 1:], clean[2][0][1, at + 1:])
    # a query: its own row, and the keys that it sees
    bad_q = q.clone()
    bad_q[1, at, 9] = x
    got = _run(bad_q, k, v, d, [n], [n], 1)
    others = torch.arange(n, device=DEV) != at
    for a, b in zip((*got[:2], got[2][0]), (*clean[:2], clean[2][0])):
        assert torch.equal(a[:, others], b[:, others])
    for a, b in zip(got[2][1:], clean[2][1:]):
        assert torch.equal(a[1, at + 1:], b[1, at + 1:])


@pytest.mark.parametrize("n", [400, 1500])
@pytest.mark.parametrize("kind", ["rise", "fall", "jump", "far-below-zero"])
def test_logits_that_move_the_softmax_reference(kind, n):
    q, k, v, d = [t.clone() for t in _inputs([n], [n], 2, 2, seed=7)]
    ramp = torch.linspace(0, 1, n, device=DEV)
    q[..., 0] = 8.0
    k[..., 0] = {"rise": 60 * ramp, "fall": -60 * ramp, "jump": 90.0 * (ramp > 0.6).float(), "far-below-zero": -300 + 20 * ramp}[kind].to(torch.bfloat16)
    _check(q, k, v, d, [n], [n], 0, 0.0, _run(q, k, v, d, [n], [n]))
    _check(q, k, v, d, [n], [n], 1, 0.0, _run(q, k, v, d, [n], [n], 1))


def test_infinite_logits():
    """First keys of -infinity: no reference yet.  Only -infinity, or +infinity: NaN, as 0 / 0 and inf - inf are."""
    n = 200
    q, k, v, d = [t.clone() for t in _inputs([n], [n], 1, 1, seed=9)]
    q[..., 0] = 1.0
    k[0, :100, 0] = -math.inf
    k[0, 100:, 0] = -50.0
    out, lse = xsv.seq_attend(q, k, v, _begin([n]))
    e = plain.Attention(q[0].cpu(), k[0, 100:].cpu(), v[0, 100:].cpu(), 0, 0.125)
    _close("out", out[0].cpu(), e.out, e.out_tol)
    _close("lse", lse[0].cpu(), e.lse, e.lse_tol)
    k[..., 0] = -math.inf
    out, lse = xsv.seq_attend(q, k, v, _begin([n]))
    assert bool(out.isnan().all()) and bool((lse == -math.inf).all())
    k[..., 0] = 0.0
    k[0, 70, 0] = math.inf
    out, lse = xsv.seq_attend(q, k, v, _begin([n]))
    assert bool(out.isnan().all()) and not bool(lse.isfinite().any())


def test_strides_broadcast_heads_and_strided_outputs():
    """One key head given to several through a stride of 0, rows far apart, outputs between other rows."""
    n, H = 150, 4
    q, k, v, d = _inputs([n], [n], H, 1, seed=11)
    want = _run(q, k, v, d, [n], [n], 1)
    wide = torch.zeros((n, 3, 1024), dtype=torch.bfloat16, device=DEV)
    spread = []
    for i, t in enumerate((k, v)):
        wide[:, i, :64] = t[0]
        spread.append(wide[:, i, :64].unsqueeze(0).expand(H, n, 64))
    room = torch.full((n, 2 * H, 64), 3.0, dtype=torch.bfloat16, device=DEV)
    out, lse = xsv.seq_attend(q, *spread, _begin([n]), causal=1, out=room.transpose(0, 1)[:H])
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1]) and bool((room[:, H:] == 3.0).all())
    dq = xsv.seq_attend_grad(d, q, *spread, out, lse, _begin([n]), causal=1)[0]
    assert torch.equal(dq, want[2][0])


def test_the_same_bits_every_time_whatever_the_neighbours_hold():
    """Twice the same call; and with other values, NaN among them, in the sequences beside one."""
    lq = [257, 100, 31]
    q, k, v, d = _inputs(lq, lq, 6, 2, seed=12)
    a, b = _run(q, k, v, d, lq, lq, 1), _run(q, k, v, d, lq, lq, 1)
    others = [t.clone() for t in (q, k, v, d)]
    for t in others:
        t[:, :257] = t[:, :257].flip(1) * 3.0
        t[:, 357:] = float("nan")
    c = _run(*others, lq, lq, 1)
    for x, y, z in zip((*a[:2], *a[2]), (*b[:2], *b[2]), (*c[:2], *c[2])):
        assert torch.equal(x, y) and torch.equal(x[:, 257:357], z[:, 257:357])


def test_gradient_against_differences():
    """Along random directions, of the definition in 64 bits."""
    n, m = 40, 52
    q, k, v, d = _inputs([n], [m], 1, 1, seed=13)
    dq, dk, dv = _run(q, k, v, d, [n], [m], 4)[2]
    Q, K, V, W = (t[0].cpu().double() for t in (q, k, v, d))
    f = lambda a, b, c: float((plain.Attention(a, b, c, 4, 0.125).out * W).sum())
    e = plain.Attention(Q, K, V, 4, 0.125, W)
    h = 1e-5
    for seed in range(3):
        g = torch.Generator().manual_seed(seed)
        for i, (x, grad, tol) in enumerate(((Q, dq, e.dq_tol), (K, dk, e.dk_tol + 2.0 ** -8 * e.dk.abs()), (V, dv, e.dv_tol + 2.0 ** -8 * e.dv.abs()))):
            u = torch.randn(x.shape, generator=g, dtype=torch.float64)
            args = [Q, K, V]
            plus, minus = list(args), list(args)
            plus[i], minus[i] = x + h * u, x - h * u
            diff = (f(*plus) - f(*minus)) / (2 * h)
            assert abs(float((grad[0].cpu().double() * u).sum()) - diff) <= float((tol * u.abs()).sum()) + 1e-6


def test_on_another_stream_and_captured_into_a_graph():
    lq = [200, 57]
    q, k, v, d = _inputs(lq, lq, 4, 2, seed=15)
    b = _begin(lq)
    form = dict(q_begin=b, causal=1, longest_q=200, longest_k=200)
    want = _run(q, k, v, d, lq, lq, 1)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    out, lse = xsv.seq_attend(q, k, v, stream=s, **form)
    grads = xsv.seq_attend_grad(d, q, k, v, out, lse, stream=s, **form)
    s.synchronize()
    for x, y in zip((out, lse, *grads), (*want[:2], *want[2])):
        assert torch.equal(x, y)
    graphs = []
    for _ in range(2):   # two graphs with workspaces of their own
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out, lse = xsv.seq_attend(q, k, v, **form)
            grads = xsv.seq_attend_grad(d, q, k, v, out, lse, **form)
        graphs.append((graph, (out, lse, *grads)))
    for _ in range(3):
        for graph, res in graphs:
            for t in res:
                t.zero_()
            graph.replay()
            torch.cuda.synchronize()
            for x, y in zip(res, (*want[:2], *want[2])):
                assert torch.equal(x, y)
            _run(d, k, v, q, lq, lq, 0)   # the program's own work between replays


def test_nothing_to_do():
    none = torch.empty((4, 0, 64), dtype=torch.bfloat16, device=DEV)
    q, k, v, d = _inputs([9], [9], 4, 2, seed=1)
    out, lse = xsv.seq_attend(none, none[:2], none[:2], _begin([0]))
    assert out.shape == (4, 0, 64) and lse.shape == (4, 0)
    assert all(t.shape[1] == 0 for t in xsv.seq_attend_grad(none, none, none[:2], none[:2], out, lse, _begin([0])))
    out, lse = xsv.seq_attend(q, k, v, torch.zeros(1, dtype=torch.int32, device=DEV))   # no sequence at all
    assert not out.any() and not lse.any()
    out, lse = xsv.seq_attend(q, none[:2], none[:2], _begin([9]), _begin([0]))          # queries without keys
    assert not out.any() and bool((lse == -math.inf).all())
    grads = xsv.seq_attend_grad(d, q, none[:2], none[:2], out, lse, _begin([9]), _begin([0]))
    assert not grads[0].any()
    out, lse = xsv.seq_attend(none, k, v, _begin([0]), _begin([9]))                     # keys without queries: gradients of zero
    marks = [torch.full(t.shape, 2.0, dtype=t.dtype, device=DEV) for t in (none, k, v)]
    xsv.seq_attend_grad(none, none, k, v, out, lse, _begin([0]), _begin([9]), grads=marks)
    assert not marks[1].any() and not marks[2].any()


@pytest.mark.parametrize("causal", [0, 1, 64, 150])
@pytest.mark.parametrize("lq,lk,longest_q,longest_k", [([300, 20, 90], [300, 20, 90], 64, None), ([300, 20, 90], [300, 20, 90], None, 100),
                                                       ([300, 90], [350, 200], 129, 130), ([40, 300], [33, 310], 31, 250), ([4500], [4600], 200, None),
                                                       ([4500], [4600], None, 4200)])
def test_bounds_below_a_sequences_length_leave_rows_out_and_move_no_other(lq, lk, longest_q, longest_k, causal, monkeypatch):
    """The rows within the bounds keep their positions, and so what they see; those behind are in no result and not written."""
    print(f"seq_attend {lq} {lk} bounds {longest_q} {longest_k} causal={causal}", flush=True)
    q, k, v, d = _inputs(lq, lk, 2, 1, seed=sum(lq) + causal)
    form = dict(q_begin=_begin(lq), k_begin=_begin(lk), causal=causal, longest_q=longest_q, longest_k=longest_k)
    out, lse = xsv.seq_attend(q, k, v, **form)
    grads = xsv.seq_attend_grad(d, q, k, v, out, lse, **form)
    torch.cuda.synchronize()
    whole_mask = plain.sees
    a = b = 0
    for n, m in zip(lq, lk):
        kept_q, kept_k = min(n, longest_q or n), min(m, longest_k or m)
        monkeypatch.setattr(plain, "sees", lambda _n, _m, c: whole_mask(n, m, c)[:_n, :_m])
        at = lambda t, start, rows: t[:, start:start + rows]
        kept = [at(t, a, kept_q) for t in (q, d, out, lse, grads[0])], [at(t, b, kept_k) for t in (k, v, *grads[1:])]
        (kq, kd, ko, kl, kdq), (kk, kv, kdk, kdv) = kept
        _check(kq, kk, kv, kd, [kept_q], [kept_k], causal, 0.0, (ko, kl, (kdq, kdk, kdv)))
        for t, start, rows, length in ((out, a, kept_q, n), (lse, a, kept_q, n), (grads[0], a, kept_q, n), (grads[1], b, kept_k, m), (grads[2], b, kept_k, m)):
            assert not t[:, start + rows:start + length].any()     # (as the binding made them)
        a, b = a + n, b + m


@pytest.mark.parametrize("n", [300, 1300, 4300])  # (1300: waves share the tiles, 4300: workgroups do)
@pytest.mark.parametrize("seen,later", [("inf", "nan"), ("inf", "-inf"), ("-inf", "inf"), ("nan", "inf")])
def test_values_that_are_not_finite_in_neighbouring_tiles(seen, later, n):
    """A row that a query sees, and one of the next tile that it does not, both in tiles that the mask cuts for the same wave: keys begin 40
    in front of the queries, so that 32 queries end in two tiles."""
    q, k, v, _ = [t.clone() for t in _inputs([n], [n + 40], 1, 1, seed=17)]
    form = dict(q_begin=_begin([n]), k_begin=_begin([n + 40]), causal=1)
    clean, clean_lse = xsv.seq_attend(q, k, v, **form)
    first, second = 2 * 64 + 43, 3 * 64 + 2
    v[0, first, 5], v[0, second, 5] = float(seen), float(later)
    got, lse = xsv.seq_attend(q, k, v, **form)
    assert torch.equal(lse, clean_lse)
    rest = torch.arange(64, device=DEV) != 5
    assert torch.equal(got[..., rest], clean[..., rest])
    pos = torch.arange(n, device=DEV) + 40
    want = torch.where(pos < first, clean[0, :, 5].float(), torch.where(pos < second, float(seen), float(seen) + float(later)))
    assert torch.equal(got[0, :, 5].float().nan_to_num(nan=12345.0), want.nan_to_num(nan=12345.0))
