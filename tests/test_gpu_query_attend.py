"""Context.query_attend against attention in 64 bits over the cache's exported dequantized view (plain_operators.Attention)."""
import math

import numpy as np
import pytest
import torch

import plain_operators as plain
from paper_2602_21780_amd import xsv
from paper_2602_21780_amd.inputs import CONFIGS, FrameSource

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _queries(H, m, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn((H, m, 64), generator=g) * scale).to(torch.bfloat16).to(DEV)


def _view(dump):
    f = lambda a: torch.from_numpy((a.astype(np.uint32) << 16).view(np.float32))
    return f(dump.k_bf16), f(dump.v_bf16)


def _compare(ctx, q, got, layer=0, heads=None, scale=0.125):
    k, v = _view(ctx.cache_export(layer))
    out, lse = got
    for h in range(q.shape[0]) if heads is None else heads:
        e = plain.Attention(q[h].cpu().float(), k[h], v[h], 0, scale)
        off = (out[h].cpu().double() - e.out).abs()
        assert bool((off <= e.out_tol + 1e-30).all()), (h, float((off / e.out_tol).max()))
        off = (lse[h].cpu().double() - e.lse).abs()
        assert bool((off <= e.lse_tol).all()), (h, float((off / e.lse_tol).max()))


def _filled(H, n, T, bits, G, seed=0, frames_seen=None, **kw):
    """A context whose layer 0 holds T tokens quantized by the library's own kernels (imported, so that T is any number)."""
    g = torch.Generator().manual_seed(seed)
    k = torch.randn((H, T, 64), generator=g)
    k[..., 5] *= 6.0
    k, v = k.to(torch.bfloat16), torch.randn((H, T, 64), generator=g).to(torch.bfloat16)
    ctx = xsv.Context(1, H, 64, n, 0, 0, bits, G, max_frames=-(-T // n) + 1, **kw)
    ids = np.arange(T, dtype=np.int32)
    if bits == 16:
        raw = [t.view(torch.int16).numpy().view(np.uint16) for t in (k, v)]
        dump = xsv.CacheDump(T, None, None, None, None, None, None, raw[0], raw[1], ids // n, ids % n)
    else:
        parts = [t.cpu().numpy() for fn, x in ((xsv.quantize_k, k), (xsv.quantize_v, v)) for t in fn(x.to(DEV), bits, G)]
        dump = xsv.CacheDump(T, *parts, None, None, ids // n, ids % n)
    ctx.cache_import(0, dump, -(-T // n))
    return ctx


@pytest.mark.parametrize("bits,G", [(4, 64), (4, 32), (2, 64), (2, 32), (16, 64)])
@pytest.mark.parametrize("H,T,m", [(1, 1, 1), (2, 63, 3), (3, 64, 16), (2, 65, 17), (5, 300, 64), (1, 4097, 5), (16, 1374, 1), (3, 1000, 130)])
def test_rows_and_cache_lengths(bits, G, H, T, m):
    print(f"query_attend bits={bits} G={G} H={H} T={T} m={m}", flush=True)
    ctx = _filled(H, 1 if T < 64 else 60, T, bits, G, seed=T + m)
    q = _queries(H, m, m)
    _compare(ctx, q, ctx.query_attend(0, q))
    ctx.destroy()


def test_long_cache_is_cut_over_many_workgroups():
    ctx = _filled(2, 1000, 40000, 4, 64, seed=3)
    for m in (1, 20):
        q = _queries(2, m, m, 1.5)
        first = ctx.query_attend(0, q)
        _compare(ctx, q, first)
        for _ in range(3):   # the same bits, whoever ends last
            for a, b in zip(first, ctx.query_attend(0, q)):
                assert torch.equal(a, b)
    ctx.destroy()


@pytest.mark.parametrize("overlap", [0, 1, 2])
def test_between_the_steps_of_a_stream(overlap):
    """Any layer of a running stream, pruned and re-quantized; the stream itself goes on as without the calls."""
    spec = CONFIGS[0].with_(n_layers=3)
    ctx, plain_ctx = (xsv.Context.from_spec(spec) for _ in range(2))
    ctx.set_overlap(overlap)
    plain_ctx.set_overlap(overlap)
    src = FrameSource(spec, DEV)
    probe = _queries(spec.n_heads, 7, 1)
    alive = []
    for f in range(6):
        q, k, v = src.frame(f)
        alive.append((q, k, v))
        for l in range(3):
            a, b = ctx.step(l, q[l], k[l], v[l]), plain_ctx.step(l, q[l], k[l], v[l])
            got = ctx.query_attend(l, probe)
            torch.cuda.synchronize()
            assert torch.equal(a, b)
            _compare(ctx, probe, got, layer=l)
    for l in range(3):
        x, y = ctx.cache_export(l), plain_ctx.cache_export(l)
        assert x.T == y.T and np.array_equal(x.k_codes, y.k_codes) and np.array_equal(x.v_codes, y.v_codes)
    ctx.destroy()
    plain_ctx.destroy()


def test_joined_with_other_keys_it_is_attention_over_both():
    """What lse is for: over the cache and over a token's own keys, joined, against attention over all of them."""
    H, T, m = 3, 500, 9
    ctx = _filled(H, 60, T, 4, 64, seed=2)
    q = _queries(H, m, 3)
    k, v = _queries(H, m, 4), _queries(H, m, 5)
    a, la = ctx.query_attend(0, q)
    begin = torch.tensor([0, m], dtype=torch.int32, device=DEV)
    b, lb = xsv.seq_attend(q, k, v, begin, causal=1)
    total = torch.logaddexp(la, lb)
    out = a.float() * torch.exp(la - total)[..., None] + b.float() * torch.exp(lb - total)[..., None]
    ck, cv = _view(ctx.cache_export(0))
    for h in range(H):
        for i in range(m):
            e = plain.Attention(q[h, i:i + 1].cpu(), torch.cat([ck[h], k[h, :i + 1].cpu().float()]), torch.cat([cv[h], v[h, :i + 1].cpu().float()]), 0, 0.125)
            assert bool(((out[h, i].cpu().double() - e.out[0]).abs() <= 2 * e.out_tol[0]).all())   # (two results, each rounded)
            assert abs(float(total[h, i]) - float(e.lse)) <= 2 * float(e.lse_tol) + 2.0 ** -20 * abs(float(e.lse))
    ctx.destroy()


def test_strided_queries_neighbouring_outputs_and_another_scale():
    H, T, m = 4, 777, 21
    ctx = _filled(H, 50, T, 4, 32, seed=6, softmax_scale=0.3)
    wide = _queries(1, m * H * 3, 7).view(m, 3, H, 64)
    q = wide[:, 1].transpose(0, 1)
    room, sums = torch.full((H * m * 64 + 128,), 3.0, dtype=torch.bfloat16, device=DEV), torch.full((H * m + 8,), 3.0, device=DEV)
    out, lse = room[64:-64].view(H, m, 64), sums[4:-4].view(H, m)
    _compare(ctx, q, ctx.query_attend(0, q, out=out, lse=lse), scale=0.3)
    for t, n in ((room, 64), (sums, 4)):
        assert bool((t[:n] == 3.0).all()) and bool((t[-n:] == 3.0).all())
    ctx.destroy()


def test_empty_cache_stale_rows_and_rows_that_are_not_finite():
    """No cache: zeros and -infinity.  Rows that the cache held before, NaN among them, behind a shorter one's end."""
    H, n = 2, 100
    ctx = xsv.Context(1, H, 64, n, 0, 0, 16, 64, max_frames=4)
    q = _queries(H, 3, 1)
    out, lse = ctx.query_attend(0, q)
    assert not out.any() and bool((lse == -math.inf).all())
    x = _queries(H, n, 2)
    nan = torch.full_like(x, float("nan"))
    ctx.step(0, x, x, x)
    ctx.step(0, x, nan, nan)
    out, lse = ctx.query_attend(0, q)
    assert bool(out.isnan().all()) and bool(lse.isnan().all())
    ctx.reset()
    ctx.step(0, x, x, x)
    _compare(ctx, q, ctx.query_attend(0, q))
    bad = q.clone()
    bad[1, 1, 3] = float("nan")
    got, want = ctx.query_attend(0, bad), ctx.query_attend(0, q)
    assert bool(got[0][1, 1].isnan().all())
    keep = torch.ones((H, 3), dtype=torch.bool, device=DEV)
    keep[1, 1] = False
    assert torch.equal(got[0][keep], want[0][keep]) and torch.equal(got[1][keep], want[1][keep])
    ctx.destroy()


def test_captured_into_a_graph():
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        ctx = _filled(4, 100, 3000, 4, 64, seed=9, stream=s)
        q = _queries(4, 2, 1)
        want = ctx.query_attend(0, q)
        out, lse = torch.empty_like(want[0]), torch.empty_like(want[1])
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            ctx.query_attend(0, q, out=out, lse=lse)
        for _ in range(3):
            out.zero_()
            lse.zero_()
            graph.replay()
            s.synchronize()
            assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
            ctx.query_attend(0, _queries(4, 33, 2))   # the program's own calls in between
    ctx.destroy()


def test_refusals():
    ctx = xsv.Context(2, 2, 64, 64, 5, 256, 4, 32)
    x = _queries(2, 64, 1)
    out, lse = torch.empty((2, 1, 64), dtype=torch.bfloat16, device=DEV), torch.empty((2, 1), device=DEV)
    call = lambda layer=0, t=None, rows=1, o=out.data_ptr(), l=lse.data_ptr(): xsv.lib().xsv_query_attend(
        ctx._h, layer, xsv.as_tensor(x) if t is None else t, rows, o, l)
    assert call() == xsv.XSV_OK and call(rows=0) == xsv.XSV_OK and call(l=None) == xsv.XSV_OK
    for bad in (dict(layer=-1), dict(layer=2), dict(rows=-1), dict(rows=(1 << 20) + 1), dict(o=None), dict(o=out.data_ptr() + 8), dict(l=lse.data_ptr() + 2),
                dict(t=xsv.xsv_tensor(None, 0, 64)), dict(t=xsv.xsv_tensor(x.data_ptr() + 2, 0, 64)), dict(t=xsv.xsv_tensor(x.data_ptr(), 0, 63))):
        assert call(**bad) == xsv.XSV_ERR_ARG, bad
    ctx.dequant_attend(0, x, x, x)          # between the stages of a step
    assert call() == xsv.XSV_ERR_STATE
    ctx.score_prune(0, x)
    assert call() == xsv.XSV_ERR_STATE
    ctx.quantize(0, x, x)
    assert call() == xsv.XSV_OK
    assert xsv.lib().xsv_query_attend(None, 0, xsv.as_tensor(x), 1, out.data_ptr(), None) == xsv.XSV_ERR_ARG
    for wrong in (x[:1], x[..., :32], x.float()):
        with pytest.raises(ValueError):
            ctx.query_attend(0, wrong)
    with pytest.raises(ValueError):
        ctx.query_attend(0, x, out=out)
    torch.cuda.synchronize()
    ctx.destroy()


def test_a_context_called_under_another_stream_than_it_was_made_under():
    """Outputs that the calls make come from the memory of the stream that they run on, not from a block that the current stream may still use."""
    H, T, m = 4, 1000, 40
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        ctx = _filled(H, 100, T, 4, 64, seed=21)       # (no stream= of its own)
    q, x = _queries(H, m, 3), _queries(H, 100, 4)
    torch.cuda.synchronize()
    held = [torch.empty((H, rows, 64), dtype=torch.bfloat16, device=DEV) for rows in (m, 100)] + [torch.empty((H, m), device=DEV)]
    free = {t.data_ptr() for t in held}
    del held                                           # the current stream's next blocks of these sizes
    out, lse = ctx.query_attend(0, q)
    step = ctx.step(0, x, x, x)
    s.synchronize()
    assert not {out.data_ptr(), lse.data_ptr(), step.data_ptr()} & free
    same = _filled(H, 100, T, 4, 64, seed=21)
    want, want_lse = same.query_attend(0, q)
    assert torch.equal(out, want) and torch.equal(lse, want_lse) and torch.equal(step, same.step(0, x, x, x))
    ctx.destroy()
    same.destroy()


@pytest.mark.parametrize("H,T,m", [(1, 300, 1), (16, 1024, 1), (16, 1090, 1), (16, 4096, 1), (16, 4160, 1), (1, 20000, 1), (16, 300, 2), (2, 5000, 3), (16, 500, 64), (16, 500, 65), (16, 1000, 71)])
def test_every_way_of_joining_the_parts(H, T, m):
    """Inside the launch and by a second one, a row to a workgroup and four, on both sides of where one takes over from the other; twice the same bits."""
    print(f"query_attend joins H={H} T={T} m={m}", flush=True)
    ctx = _filled(H, 60, T, 4, 64, seed=T + m)
    q = _queries(H, m, m)
    first = ctx.query_attend(0, q)
    _compare(ctx, q, first, heads=(0, H - 1))
    for _ in range(2):
        for a, b in zip(first, ctx.query_attend(0, q)):
            assert torch.equal(a, b)
    ctx.destroy()
