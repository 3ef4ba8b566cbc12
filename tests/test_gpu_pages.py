"""The paged cache in 8 bits against its definition in 64 bits (plain_pages)."""
import math
import random

import pytest
import torch

import plain_pages as plain
from paper_2602_21780_amd import xsv

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _randn(seed, *shape):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed))


def _begin(new, first=0):
    return [first + sum(new[:s]) for s in range(len(new) + 1)]


def _int(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _table(lengths, total, seed, width=None):
    """Pages dealt in no order, rows padded with -1."""
    order = list(range(total))
    random.Random(seed).shuffle(order)
    rows = []
    for m in lengths:
        n = -(-m // 64)
        rows.append(order[:n])
        order = order[n:]
    width = max([len(r) for r in rows] + [1]) if width is None else width
    return [r + [-1] * (width - len(r)) for r in rows]


def _table_tensor(table):
    return _int(table).view(len(table), -1)


def _filled(lengths, heads, seed, spare=2, scale=1.0, edit=None, width=None):
    """A pool with sequences of such lengths, written in one call; (pages, table, the pool in 64 bits)."""
    total = sum(-(-m // 64) for m in lengths) + spare
    table = _table(lengths, total, seed, width)
    pages = xsv.Pages.empty(total, heads, DEV)
    k, v = _randn(seed, heads, sum(lengths), 64) * scale, _randn(seed + 1, heads, sum(lengths), 64)
    k[..., 7] *= 5.0
    if edit:
        edit(k, v)
    xsv.pages_write(pages, k.to(torch.bfloat16).to(DEV), v.to(torch.bfloat16).to(DEV), _int(_begin(lengths)), _table_tensor(table), _int(lengths))
    return pages, table, plain.of(pages)


def _same(pages, pool, only=None):
    got = plain.of(pages)
    for p in range(pages.count) if only is None else only:
        if not pool.written[p]:
            continue
        for name in ("k", "v", "ke", "ve", "bounds"):
            a, b = getattr(got, name)[p], getattr(pool, name)[p]
            assert torch.equal(torch.nan_to_num(a, 1e9), torch.nan_to_num(b, 1e9)) if a.is_floating_point() else torch.equal(a, b), (p, name)


# ---- writing --------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("heads", [1, 3, 16])
@pytest.mark.parametrize("steps", [[[1], [1], [61], [1], [1], [64], [129]], [[0, 5, 130], [3, 0, 1], [59, 61, 63], [1, 1, 1]], [[200, 64]],
                                   [[63, 64, 65, 1], [1, 1, 1, 1], [1, 64, 63, 127]]])
def test_sequences_that_grow(heads, steps):
    print(f"pages_write heads={heads} steps={steps}", flush=True)
    ends = [sum(s[i] for s in steps) for i in range(len(steps[0]))]
    total = sum(-(-m // 64) for m in ends) + 3
    table = _table(ends, total, heads)
    pages, pool = xsv.Pages.empty(total, heads, DEV), plain.Pool(total, heads)
    held = [0] * len(ends)
    for i, new in enumerate(steps):
        held = [a + b for a, b in zip(held, new)]
        rows = sum(new) + 2                       # two rows of no sequence, one on either side
        k, v = ((_randn(10 * i + j, heads, rows, 64) * (1 + 3 * i)).to(torch.bfloat16) for j in range(2))
        begin = _begin(new, 1)
        before = plain.of(pages)
        xsv.pages_write(pages, k.to(DEV), v.to(DEV), _int(begin), _table_tensor(table), _int(held))
        pool.write(k, v, begin, table, held)
        _same(pages, pool)
        after = plain.of(pages)
        for p in range(total):
            if not pool.written[p]:
                assert torch.equal(before.k[p], after.k[p]) and torch.equal(before.bounds[p], after.bounds[p])


def test_values_of_every_magnitude_and_none():
    """Scales that grow by a little and by everything, zeros, the smallest and largest numbers, infinities and NaN."""
    heads, sizes = 2, [0.0, 1e-38, 2e-30, 1e-30, 3e-12, 1e-4, 0.9, 1.1, 500.0, 1e20, 3e38]
    table, held = [[1, 0]], 0
    pages, pool = xsv.Pages.empty(2, heads, DEV), plain.Pool(2, heads)
    for i, size in enumerate(sizes * 2):
        k, v = ((_randn(50 + 2 * i + j, heads, 5, 64).clamp(-1, 1) * size).to(torch.bfloat16) for j in range(2))
        if i % 4 == 2:
            k[0, 1, 3], v[1, 2, 4] = math.inf, math.nan
            v[0, 0, 0] = -math.inf
        held += 5
        xsv.pages_write(pages, k.to(DEV), v.to(DEV), _int([0, 5]), _int(table), _int([held]))
        pool.write(k, v, [0, 5], table, [held])
        _same(pages, pool)


def test_every_code_and_tie():
    """All bf16 numbers of 14 binades, so that every rounding to e4m3 occurs, halves and subnormal codes among them."""
    bits = torch.arange(0x3000, 0x43e1, dtype=torch.int32)       # 2^-31 .. 448 and all between
    x = torch.cat([bits, bits | 0x8000]).to(torch.int32)
    x = (x << 16).view(torch.float32)
    n = -(-x.numel() // 4096) * 64
    rows = torch.zeros(n * 64)
    rows[:x.numel()] = x
    rows = rows.view(1, n, 64)
    rows[0, ::64, 0] = 448.0                                      # every page's scale is 1
    pages, table = xsv.Pages.empty(n // 64, 1, DEV), [list(range(n // 64))]
    pool = plain.Pool(n // 64, 1)
    r = rows.to(torch.bfloat16)
    assert torch.equal(r.float(), rows)
    xsv.pages_write(pages, r.to(DEV), r.to(DEV), _int([0, n]), _int(table), _int([n]))
    pool.write(r, r, [0, n], table, [n])
    assert bool((pool.ke == 0).all())
    _same(pages, pool)


def test_packed_rows_and_bounds_on_lengths():
    """Keys and values as a projection leaves them; a bound on the rows; offsets and lengths that leave their tensors."""
    x = _randn(3, 300, 2 * 4, 64).to(torch.bfloat16).to(DEV).transpose(0, 1)
    k, v = x[:4], x[4:]
    for begin, lengths, longest, as_if in (([0, 100, 300], [130, 200], None, ([0, 100, 300], [130, 200])),
                                           ([0, 100, 300], [130, 200], 70, ([0, 70, 100, 170], [100, 0, 70])),
                                           ([-5, 100, 900], [130, 200], None, ([0, 100, 300], [130, 200])),
                                           ([200, 100, 50], [130, 200], None, ([0, 0, 0], [130, 200])),
                                           ([0, 300, 300], [100, 0], None, ([200, 300, 300], [100, 0]))):
        table = _table([300, 300], 12, 1)
        pages, pool = xsv.Pages.empty(12, 4, DEV), plain.Pool(12, 4)
        xsv.pages_write(pages, k, v, _int(begin), _int(table), _int(lengths), longest=longest)
        begin, lengths = as_if
        if len(begin) == 4:     # the first 70 rows of 100 behind 30 tokens, of 200 behind none
            pool.write(k.cpu(), v.cpu(), [0, 70], table[:1], [100])
            pool.write(k.cpu(), v.cpu(), [100, 170], table[1:], [70])
        else:
            pool.write(k.cpu(), v.cpu(), begin, table, lengths)
        got = plain.of(pages)
        for p in range(12):
            for h in range(4):
                if pool.written[p]:
                    assert torch.equal(got.k[p, h], pool.k[p, h]) and torch.equal(got.v[p, h], pool.v[p, h]), (begin, p)
                else:
                    assert not got.k[p].any() and not got.v[p].any()


def test_pages_that_are_none_are_not_written_and_others_are():
    pages, pool = xsv.Pages.empty(3, 2, DEV), plain.Pool(3, 2)
    k, v = (_randn(i, 2, 320, 64).to(torch.bfloat16) for i in (1, 2))
    table = [[2, -1, 3, 1 << 30, 0]]
    xsv.pages_write(pages, k.to(DEV), v.to(DEV), _int([0, 320]), _int(table), _int([320]))
    pool.write(k, v, [0, 320], table, [320])
    _same(pages, pool)
    assert pool.written.tolist() == [True, False, True] and not pages.k.view(torch.uint8)[1].any()


# ---- reading --------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("heads", [1, 5])
def test_reading_back_gives_what_the_codes_stand_for(heads):
    lengths, new = [1, 64, 130, 0, 777], [1, 3, 130, 0, 500]
    pages, table, pool = _filled(lengths, heads, 4, scale=30.0)
    begin = _begin(new, 2)
    rows = begin[-1] + 3
    out = [torch.full((heads, rows, 64), 9.0, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    got = xsv.pages_read(pages, _int(begin), _table_tensor(table), _int(lengths), out=out)
    assert got[0] is out[0] and got[1] is out[1]
    made = xsv.pages_read(pages, _int(begin), _table_tensor(table), _int(lengths), rows=rows)
    for s, m in enumerate(lengths):
        for h in range(heads):
            k, v, _ = pool.tokens(table[s], m, h)
            for x, o, z in ((k, out[0], made[0]), (v, out[1], made[1])):
                want = x[m - new[s]:]
                assert torch.equal(o[h, begin[s]:begin[s + 1]].cpu().double(), want)
                assert torch.equal(z[h, begin[s]:begin[s + 1]].cpu().double(), want)
    for o, z in zip(out, made):
        for r in list(range(2)) + list(range(begin[-1], rows)):
            assert bool((o[:, r] == 9.0).all()) and not z[:, r].any()


def test_reading_into_a_packed_tensor_and_past_pages_that_are_none():
    pages, table, pool = _filled([200], 3, 6)
    table[0][1] = -1
    x = torch.full((210, 6, 64), 9.0, dtype=torch.bfloat16, device=DEV).transpose(0, 1)
    xsv.pages_read(pages, _int([0, 205]), _int(table), _int([200]), out=[x[:3], x[3:]])     # five rows in front of the first token
    for h in range(3):
        k, v, at = pool.tokens(table[0], 200, h)
        for want, got in ((k, x[h]), (v, x[3 + h])):
            full = torch.full((210, 64), 9.0, dtype=torch.float64)
            full[5 + at] = want
            assert torch.equal(got.cpu().double(), full)


# ---- attention ------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("causal", [0, 1, 59])
@pytest.mark.parametrize("heads,kv_heads,new,lengths", [
    (1, 1, [1], [1]), (2, 2, [1], [63]), (4, 1, [1, 1, 1], [64, 65, 1]), (12, 4, [1, 63, 64, 0, 130], [1, 100, 64, 9, 300]), (16, 16, [17], [500]),
    (40, 2, [3, 1], [129, 64]), (7, 7, [5, 1], [3, 700]), (33, 1, [2], [70]), (6, 2, [200], [333]), (4, 2, [40, 3, 20], [5, 0, 20])])
def test_attention_over_pages(heads, kv_heads, new, lengths, causal):
    print(f"pages_attend heads={heads}/{kv_heads} new={new} lengths={lengths} causal={causal}", flush=True)
    pages, table, pool = _filled(lengths, kv_heads, sum(lengths) + causal)
    q = (_randn(5, heads, sum(new) + 2, 64) * 1.5).to(torch.bfloat16).to(DEV)
    begin = _begin(new, 1)
    got = xsv.pages_attend(pages, q, _int(begin), _table_tensor(table), _int(lengths), causal=causal)
    plain.check_attend(pool, q, got, begin, table, lengths, causal)
    for r in (0, begin[-1]):     # rows of no sequence
        assert not got[0][:, r].any() and not got[1][:, r].any()


@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (8, 2)])
def test_long_sequences_are_cut_over_workgroups(heads, kv_heads):
    lengths, new = [20000, 70, 9000], [1, 1, 2]
    pages, table, pool = _filled(lengths, kv_heads, 8)
    q = (_randn(9, heads, 4, 64) * 2.0).to(torch.bfloat16).to(DEV)
    call = lambda **kw: xsv.pages_attend(pages, q, _int(_begin(new)), _table_tensor(table), _int(lengths), causal=1, **kw)
    got = call()
    plain.check_attend(pool, q, got, _begin(new), table, lengths, 1)
    for _ in range(3):
        for a, b in zip(got, call()):
            assert torch.equal(a, b)
    # tokens behind a bound are left out, the others keep their places
    got = call(longest_k=5000)
    plain.check_attend(pool, q[:, :1], [x[:, :1] for x in got], [0, 1], [table[0]], [5000], 0)
    plain.check_attend(pool, q[:, 1:2], [x[:, 1:2] for x in got], [0, 1], [table[1]], [70], 1)


def test_a_frame_over_a_cache_and_a_bound_on_rows():
    lengths, new = [1374 + 700], [1374]
    pages, table, pool = _filled(lengths, 2, 21)
    q = _randn(22, 4, 1374, 64).to(torch.bfloat16).to(DEV)
    for causal in (0, 1374, 1):
        out = torch.full((4, 1374, 64), 3.0, dtype=torch.bfloat16, device=DEV)
        lse = torch.full((4, 1374), 3.0, device=DEV)
        got = xsv.pages_attend(pages, q, _int([0, 1374]), _int(table), _int(lengths), causal=causal, out=out, lse=lse, longest_q=1000)
        assert bool((out[:, 1000:] == 3.0).all()) and bool((lse[:, 1000:] == 3.0).all())
        limits = torch.tensor([plain.limit(i, 1374, lengths[0], causal) for i in range(1000)])
        for h in range(4):
            k, v, at = pool.tokens(table[0], lengths[0], h // 2)
            S = q[h, :1000].cpu().double() @ k.T * 0.125
            S[at[None, :] >= limits[:, None]] = -math.inf
            e = torch.softmax(S, 1) @ v
            # 2^-8 of the result for its rounding, and of the weights' for theirs
            bound = 2.0 ** -8 * (e.abs() + torch.softmax(S, 1) @ v.abs()) * 1.1
            assert bool(((out[h, :1000].cpu().double() - e).abs() <= bound).all())
            assert bool(((lse[h, :1000].cpu().double() - torch.logsumexp(S, 1)).abs() <= 2e-5).all())


def test_rows_that_see_nothing():
    pages, table, pool = _filled([5, 0, 64], 2, 31)
    new, begin = [9, 2, 1], [0, 9, 11, 12]
    q = _randn(1, 2, 12, 64).to(torch.bfloat16).to(DEV)
    for causal in (0, 1):
        out, lse = torch.ones((2, 12, 64), dtype=torch.bfloat16, device=DEV), torch.ones((2, 12), device=DEV)
        xsv.pages_attend(pages, q, _int(begin), _int(table), _int([5, 0, 64]), causal=causal, out=out, lse=lse)
        plain.check_attend(pool, q, (out, lse), begin, table, [5, 0, 64], causal)
        for r in (0, 3, 9, 10):
            assert not out[:, r].any() and bool((lse[:, r] == -math.inf).all())
    empty = xsv.Pages.empty(0, 2, DEV)     # a pool of no pages
    out, lse = xsv.pages_attend(empty, q, _int(begin), _int([[0], [0], [0]]), _int([5, 0, 64]))
    assert not out.any() and bool((lse == -math.inf).all())
    chosen = torch.zeros((12, 2, 1), dtype=torch.int32, device=DEV)
    out, lse = xsv.pages_attend(empty, q, _int(begin), _int([[0], [0], [0]]), _int([5, 0, 64]), chosen=chosen)
    assert not out.any() and bool((lse == -math.inf).all())


def test_pages_that_are_none_and_pages_that_sequences_share():
    lengths = [300, 260]
    pages, table, pool = _filled(lengths, 2, 33)
    table[0][1], table[0][3] = -1, 1 << 20
    table[1][:2] = [table[0][0], table[0][2]]       # a common beginning
    q = _randn(2, 4, 5, 64).to(torch.bfloat16).to(DEV)
    for causal in (0, 1):
        got = xsv.pages_attend(pages, q, _int([0, 2, 5]), _table_tensor(table), _int(lengths), causal=causal)
        plain.check_attend(pool, q, got, [0, 2, 5], table, lengths, causal)


@pytest.mark.parametrize("rows", [3, 70])
def test_nan_reaches_the_rows_that_see_its_token(rows):
    def edit(k, v):
        v[0, 150, 3], v[0, 199, 60], v[1, 20, 5] = math.nan, math.inf, math.nan
        k[1, 195, 2] = math.nan
        k[:, 200:], v[:, 200:] = math.nan, math.nan     # tokens that are taken back
    pages, table, pool = _filled([230], 2, 35, edit=edit)
    q = _randn(4, 4, rows, 64).to(torch.bfloat16).to(DEV)
    for causal in (0, 1, 59):
        got = xsv.pages_attend(pages, q, _int([0, rows]), _int(table), _int([200]), causal=causal)
        plain.check_attend(pool, q, got, [0, rows], table, [200], causal)
    lists = torch.tensor([0, 2, 3], dtype=torch.int32, device=DEV).expand(rows, 2, 3).contiguous()
    got = xsv.pages_attend(pages, q, _int([0, rows]), _int(table), _int([200]), causal=1, chosen=lists)
    plain.check_attend(pool, q, got, [0, rows], table, [200], 1, chosen=lists.cpu())


def test_large_logits_and_scales():
    for scale, size in ((0.125, 40.0), (3.0, 4.0), (1e-6, 1.0)):
        pages, table, pool = _filled([700], 1, 41, scale=size)
        q = (_randn(6, 3, 20, 64) * size).to(torch.bfloat16).to(DEV)
        got = xsv.pages_attend(pages, q, _int([0, 20]), _int(table), _int([700]), causal=1, softmax_scale=scale)
        plain.check_attend(pool, q, got, [0, 20], table, [700], 1, scale)


def test_pages_of_very_different_scales():
    """Pages whose values (and keys) are 2^20 apart, so that their scales are."""
    def edit(k, v):
        for i in range(8):
            v[:, 64 * i:64 * i + 64] *= 2.0 ** (20 * (i % 3) - 20)
            k[:, 64 * i:64 * i + 64] *= 2.0 ** (2 * (i % 4) - 6)
    pages, table, pool = _filled([500], 2, 43, edit=edit)
    q = _randn(7, 4, 90, 64).to(torch.bfloat16).to(DEV)
    for causal in (0, 1):
        got = xsv.pages_attend(pages, q, _int([0, 90]), _int(table), _int([500]), causal=causal)
        plain.check_attend(pool, q, got, [0, 90], table, [500], causal)


def test_scales_whose_product_fp32_does_not_hold():
    """Tiny keys and a tiny scale: logits of 0, and what is masked stays masked."""
    pages, table, pool = _filled([130], 1, 42, scale=1e-29)
    for rows in (2, 40):
        q = _randn(6, 2, rows, 64).to(torch.bfloat16).to(DEV)
        got = xsv.pages_attend(pages, q, _int([0, rows]), _int(table), _int([130]), causal=1, softmax_scale=1e-20)
        plain.check_attend(pool, q, got, [0, rows], table, [130], 1, 1e-20)


@pytest.mark.parametrize("rows", [1, 40])
@pytest.mark.parametrize("step", [0.4, 30.0, 400.0])
def test_logits_that_rise_and_fall_along_a_sequence(rows, step):
    """Logits that rise with the page (by 2^24 and by more than fp32 holds), then fall: references that move, weights that vanish."""
    direction = torch.zeros(64)
    direction[:8] = 1.0

    def edit(k, v):
        for i in range(20):
            k[:, 64 * i:64 * i + 64] += direction * step * (min(i, 14) - 2.0 * max(i - 14, 0))
    pages, table, pool = _filled([64 * 20 - 7], 2, 47, edit=edit)
    q = (_randn(9, 4, rows, 64) * 0.3 + direction).to(torch.bfloat16).to(DEV)
    for causal in (0, 1):
        got = xsv.pages_attend(pages, q, _int([0, rows]), _int(table), _int([64 * 20 - 7]), causal=causal)
        plain.check_attend(pool, q, got, [0, rows], table, [64 * 20 - 7], causal)
    lists = torch.tensor([1, 3, 7, 14, 15, 19], dtype=torch.int32).expand(rows, 2, 6).clone()
    lists[:, 1, ::2] = -1
    got = xsv.pages_attend(pages, q, _int([0, rows]), _int(table), _int([64 * 20 - 7]), causal=1, chosen=lists.to(DEV))
    plain.check_attend(pool, q, got, [0, rows], table, [64 * 20 - 7], 1, chosen=lists)


# Launches with many blocks take 64 rows at a time: rows of no sequence behind those of some make one of any call.
MANY = 2048


def _many(q):
    """q behind which rows of no sequence are, NaN."""
    out = torch.full((q.shape[0], MANY, 64), math.nan, dtype=torch.bfloat16)
    out[:, :q.shape[1]] = q
    return out.to(DEV)


def _attend_many(pages, q, begin, table, lengths, **kw):
    got = xsv.pages_attend(pages, _many(q), _int(begin), _table_tensor(table), _int(lengths), **kw)
    assert not got[0][:, q.shape[1]:].any() and not got[1][:, q.shape[1]:].any()
    return [x[:, :q.shape[1]].contiguous() for x in got]


@pytest.mark.parametrize("causal", [0, 1, 59])
@pytest.mark.parametrize("new,lengths", [([1], [1]), ([70], [500]), ([300], [300]), ([33, 0, 64, 129, 5], [33, 9, 300, 128, 700]), ([40, 3, 20], [5, 0, 20])])
def test_many_blocks_of_rows(new, lengths, causal):
    print(f"pages_attend of 64 rows new={new} lengths={lengths} causal={causal}", flush=True)
    pages, table, pool = _filled(lengths, 8, 61 + sum(new))
    q = (_randn(12, 16, sum(new), 64) * 1.5).to(torch.bfloat16)
    got = _attend_many(pages, q, _begin(new), table, lengths, causal=causal)
    plain.check_attend(pool, q, got, _begin(new), table, lengths, causal, heads=[0, 15])


def test_many_blocks_of_rows_over_a_long_sequence():
    """More pages than a wave looks up at once, some of them none."""
    pages, table, pool = _filled([18000], 8, 62)
    table[0][3], table[0][100], table[0][255:262] = -1, 1 << 20, [-1] * 7
    q = (_randn(13, 16, 40, 64) * 1.5).to(torch.bfloat16)
    got = _attend_many(pages, q, [0, 40], table, [18000])
    assert all(torch.equal(a, b) for a, b in zip(got, _attend_many(pages, q, [0, 40], table, [18000])))
    seen = [j for j in range(len(table[0])) if 0 <= table[0][j] < pages.count]      # (check_attend's rows see all: one product a head)
    assert len(seen) == 282 - 9
    plain.check_attend(pool, q, got, [0, 40], table, [18000], 0, heads=[0, 9])


def test_nan_among_many_blocks_of_rows():
    def edit(k, v):
        v[0, 150, 3], v[0, 199, 60], v[1, 20, 5] = math.nan, math.inf, math.nan
        k[1, 195, 2] = math.nan
        k[:, 200:], v[:, 200:] = math.nan, math.nan     # tokens that are taken back
    pages, table, pool = _filled([230], 8, 63, edit=edit)
    q = _randn(14, 16, 70, 64).to(torch.bfloat16)
    for causal in (0, 1, 59):
        got = _attend_many(pages, q, [0, 70], table, [200], causal=causal)
        plain.check_attend(pool, q, got, [0, 70], table, [200], causal, heads=[0, 1, 2, 3, 15])


@pytest.mark.parametrize("step", [0.4, 30.0, 400.0])
@pytest.mark.parametrize("tile", [0, 1])
@pytest.mark.parametrize("half", [0, 1])
def test_logits_that_rise_in_one_of_many_blocks(half, tile, step):
    """In some tokens of a page and for some rows of 64 only, by less and by more than the weights' reference bears."""
    direction = torch.zeros(64)
    direction[:8] = 1.0

    def edit(k, v):
        for i in (3, 4, 9, 10, 13):
            k[:, 64 * i + 32 * half:64 * i + 32 * half + 32] += direction * step * i
    pages, table, pool = _filled([64 * 20 - 7], 8, 64, edit=edit)
    q = _randn(15, 16, 64, 64) * 0.3
    q[:, 16 * tile:16 * tile + 16] += direction     # (two heads a key head: rows 32 tile .. of the first 64)
    q = q.to(torch.bfloat16)
    for causal in (0, 1):
        few = xsv.pages_attend(pages, q.to(DEV), _int([0, 64]), _int(table), _int([64 * 20 - 7]), causal=causal)     # (32 at a time)
        for got in (few, _attend_many(pages, q, [0, 64], table, [64 * 20 - 7], causal=causal)):
            plain.check_attend(pool, q, got, [0, 64], table, [64 * 20 - 7], causal, heads=[0, 7])


@pytest.mark.parametrize("kv_heads", [3, 8])
def test_many_sequences_of_several_blocks(kv_heads):
    """Up to 64 sequences' blocks go by what they see, those of more by their place."""
    rng = random.Random(kv_heads)
    for count in (5, 66):
        new = [rng.choice([0, 1, 3, 20, 37]) for _ in range(count)]
        lengths = [max(n + rng.choice([-2, 0, 0, 5, 200]), 0) for n in new]
        pages, table, pool = _filled(lengths, kv_heads, 48 + count)
        q = _randn(10, 2 * kv_heads, sum(new), 64).to(torch.bfloat16).to(DEV)
        got = xsv.pages_attend(pages, q, _int(_begin(new)), _table_tensor(table), _int(lengths), causal=1, longest_q=max(new), longest_k=max(lengths))
        plain.check_attend(pool, q, got, _begin(new), table, lengths, 1, heads=[0, 2 * kv_heads - 1])


def test_tokens_of_pages_that_were_never_written_are_zeros():
    pages = xsv.Pages.empty(4, 2, DEV)
    for rows in (1, 40):
        q = _randn(11, 4, rows, 64).to(torch.bfloat16).to(DEV)
        out, lse = xsv.pages_attend(pages, q, _int([0, rows]), _int([[2, 0, 1]]), _int([150]))
        assert not out.any() and bool(((lse - math.log(150.0)).abs() <= 1e-5).all())


def test_strided_queries_and_outputs():
    pages, table, pool = _filled([400, 90], 2, 45)
    q = _randn(8, 70, 6, 64).to(torch.bfloat16).to(DEV).transpose(0, 1)
    out = torch.zeros((70, 6, 64), dtype=torch.bfloat16, device=DEV).transpose(0, 1)
    got = xsv.pages_attend(pages, q, _int([0, 66, 70]), _table_tensor(table), _int([400, 90]), causal=1, out=out)
    assert got[0] is out
    plain.check_attend(pool, q, got, [0, 66, 70], table, [400, 90], 1)


# ---- chosen pages ---------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("heads,kv_heads,count", [(2, 2, 1), (8, 2, 5), (34, 2, 7), (16, 1, 70)])
def test_attention_over_listed_pages(heads, kv_heads, count):
    """Lists in any order, with what is no page, what a row does not see, and pages listed twice."""
    print(f"pages_attend chosen heads={heads}/{kv_heads} count={count}", flush=True)
    lengths, new = [900, 64, 130, 3], [5, 1, 130, 4]
    pages, table, pool = _filled(lengths, kv_heads, 50 + count)
    table[0][4] = -1
    rng = random.Random(count)
    begin = _begin(new, 1)
    rows = begin[-1] + 1
    chosen = torch.tensor([[[rng.choice([-1, 0, 1, 2, rng.randint(0, 14), 1 << 29, -7]) for _ in range(count)] for _ in range(kv_heads)] for _ in range(rows)],
                          dtype=torch.int32)
    q = _randn(11, heads, rows, 64).to(torch.bfloat16).to(DEV)
    for causal in (0, 1):
        got = xsv.pages_attend(pages, q, _int(begin), _table_tensor(table), _int(lengths), causal=causal, chosen=chosen.to(DEV))
        plain.check_attend(pool, q, got, begin, table, lengths, causal, chosen=chosen, heads=None if heads <= 8 else [0, heads // 2, heads - 1])


@pytest.mark.parametrize("causal", [0, 1, 59])
@pytest.mark.parametrize("count", [1, 5, 8])
def test_short_lists_of_many_blocks(count, causal):
    """A wave to a block of queries: pages listed twice, by many, by one, none, NaN, holes, sequences of several lengths."""
    def edit(k, v):
        v[0, 500, 3], k[1, 700, 2] = math.nan, math.nan
    new, lengths = [40, 0, 3, 61], [1000, 9, 2, 61]
    pages, table, pool = _filled(lengths, 8, 91 + count, edit=edit)
    table[0][2] = -1
    q = (_randn(19, 16, sum(new), 64) * 1.5).to(torch.bfloat16)
    g = torch.Generator().manual_seed(92)
    lists = torch.randint(-1, 18, (sum(new), 8, count), generator=g, dtype=torch.int32)
    lists[3:20] = lists[3]
    chosen = torch.full((MANY, 8, count), 7, dtype=torch.int32)
    chosen[:sum(new)] = lists
    got = _attend_many(pages, q, _begin(new), table, lengths, causal=causal, chosen=chosen.to(DEV))
    plain.check_attend(pool, q, got, _begin(new), table, lengths, causal, chosen=lists, heads=[0, 1, 2, 15])


def test_lists_over_many_pages_and_shared_by_workgroups():
    """More pages than are listed at a time; lists of one query long enough to be shared."""
    m = 64 * 4200 + 9
    pages, table, pool = _filled([m], 1, 63)
    rng = random.Random(3)
    for rows, count in ((3, 6), (1, 40)):
        lists = torch.tensor([[sorted(rng.sample(range(4201), count), key=lambda _: rng.random())] for _ in range(rows)], dtype=torch.int32)
        lists[0, 0, :4] = torch.tensor([2047, 2048, 4200, 0])
        q = _randn(14, 2, rows, 64).to(torch.bfloat16).to(DEV)
        got = xsv.pages_attend(pages, q, _int([0, rows]), _int(table), _int([m]), causal=1, chosen=lists.to(DEV))
        plain.check_attend(pool, q, got, [0, rows], table, [m], 1, chosen=lists)
        for _ in range(2):
            again = xsv.pages_attend(pages, q, _int([0, rows]), _int(table), _int([m]), causal=1, chosen=lists.flip(2).contiguous().to(DEV))
            assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])     # the order of a list changes nothing


def test_all_pages_listed_is_attention_over_all():
    pages, table, pool = _filled([2000], 2, 61)
    q = _randn(12, 6, 3, 64).to(torch.bfloat16).to(DEV)
    lists = torch.arange(32, dtype=torch.int32, device=DEV).expand(3, 2, 32).contiguous()
    got = xsv.pages_attend(pages, q, _int([0, 3]), _int(table), _int([2000]), causal=1, chosen=lists)
    plain.check_attend(pool, q, got, [0, 3], table, [2000], 1)


# ---- the choice -----------------------------------------------------------------------------------------------------

def _check_select(pages, pool, q, begin, table, lengths, count, first, last, causal, **kw):
    got = xsv.pages_select(pages, q, _int(begin), _table_tensor(table), _int(lengths), count, first=first, last=last, causal=causal, **kw).cpu()
    want = plain.select(pool, q, begin, table, lengths, count, first, last, causal)
    for (r, g), pages_of in want.items():
        assert got[r, g].tolist() == pages_of, (r, g, got[r, g].tolist(), pages_of)
    for r in range(got.shape[0]):
        if not any(begin[s] <= r < begin[s + 1] for s in range(len(lengths))):
            assert bool((got[r] == -1).all())
    return got


@pytest.mark.parametrize("heads,kv_heads,count,first,last", [(1, 1, 1, 0, 0), (1, 1, 1, 0, 1), (4, 2, 4, 1, 1), (6, 2, 8, 0, 2), (20, 1, 16, 2, 3), (5, 5, 40, 1, 1)])
@pytest.mark.parametrize("causal", [0, 1, 59])
def test_choice_of_pages(heads, kv_heads, count, first, last, causal):
    print(f"pages_select heads={heads}/{kv_heads} count={count} first={first} last={last} causal={causal}", flush=True)
    lengths, new = [1, 1500, 64, 0, 700], [1, 3, 1, 0, 40]
    pages, table, pool = _filled(lengths, kv_heads, 70 + count)
    table[1][5] = -1
    q = _randn(13, heads, sum(new) + 2, 64).to(torch.bfloat16).to(DEV)
    _check_select(pages, pool, q, _begin(new, 1), table, lengths, count, first, last, causal)


def test_equal_scores_go_to_the_lower_page():
    pages, table, pool = _filled([64 * 30], 2, 81)
    for x in (pages.k.view(torch.uint8), pages.k_scale, pages.k_bounds):
        src = x[table[0][9]].clone()
        for j in (3, 4, 12, 13, 14, 20, 29):
            x[table[0][j]] = src
    pool = plain.of(pages)
    q = _randn(14, 4, 6, 64).to(torch.bfloat16)
    q[:, 4] = 0.0                                     # every page the same
    for count in (1, 3, 5, 8, 29, 30, 31):
        _check_select(pages, pool, q.to(DEV), [0, 6], table, [64 * 30], count, 0, 0, 0)


def test_queries_of_every_magnitude():
    pages, table, pool = _filled([64 * 12], 1, 83)
    q = _randn(15, 2, 9, 64)
    for i, size in enumerate((1e-38, 1e-36, 1e-20, 1e-3, 1.0, 1e6, 1e30, 1e38)):
        q[:, i] *= size
    q = q.to(torch.bfloat16)
    q[0, 3, 5], q[1, 4, 9], q[0, 8, 1] = math.nan, math.inf, -math.inf
    _check_select(pages, pool, q.to(DEV), [0, 9], table, [64 * 12], 4, 0, 1, 0)


def test_scales_of_every_magnitude():
    def edit(k, v):
        for i in range(12):
            k[:, 64 * i:64 * i + 64] *= 2.0 ** (18 * (i % 7) - 60)
    pages, table, pool = _filled([64 * 12], 2, 85, edit=edit)
    q = _randn(16, 4, 3, 64)
    q[:, 1] *= 2.0 ** 100
    q[:, 2] *= 2.0 ** -100
    _check_select(pages, pool, q.to(torch.bfloat16).to(DEV), [0, 3], table, [64 * 12], 5, 0, 1, 0)


def test_choice_among_many_pages_and_within_a_bound():
    lengths = [64 * 2500 + 3]
    pages, table, pool = _filled(lengths, 1, 87)
    q = _randn(17, 2, 2, 64).to(torch.bfloat16).to(DEV)
    _check_select(pages, pool, q, [0, 2], table, lengths, 64, 2, 2, 1)
    _check_select(pages, pool, q, [0, 2], table, lengths, 9, 1, 2, 1)
    got = xsv.pages_select(pages, q, _int([0, 2]), _int(table), _int(lengths), 8, causal=0, longest_k=1000).cpu()
    want = plain.select(pool, q, [0, 2], table, [1000], 8, 1, 1, 0)
    assert all(got[r, 0].tolist() == want[r, 0] for r in range(2))


@pytest.mark.parametrize("heads", [8, 16, 40, 64])
def test_choice_of_many_workgroups(heads):
    """Rows of no sequence make the launch large: 4 waves to a workgroup, 16 rows of one, two and eight heads to a key head; five go another way."""
    new, lengths = [40, 0, 3, 61], [1000, 9, 2, 61]
    pages, table, pool = _filled(lengths, 8, 93)
    table[0][2] = -1
    q = (_randn(20, heads, sum(new), 64) * 1.5).to(torch.bfloat16)
    for causal, count in ((1, 5), (0, 12)):
        got = xsv.pages_select(pages, _many(q), _int(_begin(new)), _table_tensor(table), _int(lengths), count, first=1, last=2, causal=causal).cpu()
        assert bool((got[sum(new):] == -1).all())
        want = plain.select(pool, q, _begin(new), table, lengths, count, 1, 2, causal)
        assert all(got[r, g].tolist() == want[r, g] for r in range(sum(new)) for g in range(8))


@pytest.mark.parametrize("heads,kv_heads,length", [(2, 2, 64 * 1000 + 5), (5, 1, 2000), (6, 1, 64 * 1100), (4, 1, 64 * 900)])
def test_choice_for_many_queries_of_a_workgroup(heads, kv_heads, length):
    """16 and 32 rows, heads side by side and not, lists of few and of many."""
    pages, table, pool = _filled([length], kv_heads, 88)
    q = _randn(18, heads, 19, 64).to(torch.bfloat16).to(DEV)
    for count in (9, 70):
        _check_select(pages, pool, q, [0, 19], table, [length], count, 1, 2, 1)


def test_choice_within_a_bound_far_above_many_sequences_rows():
    """The launch is sized by groups of rows, not by rows."""
    lengths = [130 + s for s in range(64)]
    pages, table, pool = _filled(lengths, 16, 66)
    q = _randn(16, 16, 4200, 64).to(torch.bfloat16).to(DEV)
    call = lambda **kw: xsv.pages_select(pages, q, _int(_begin([1] * 64)), _table_tensor(table), _int(lengths), 2, causal=1, **kw)
    assert torch.equal(call(), call(longest_q=1))


@pytest.mark.parametrize("count,pages_in_all", [(65, 700), (100, 90), (200, 300), (64, 64)])
def test_choice_of_more_pages_than_lanes(count, pages_in_all):
    pages, table, pool = _filled([64 * pages_in_all - 1], 2, 86)
    q = _randn(19, 4, 2, 64).to(torch.bfloat16).to(DEV)
    _check_select(pages, pool, q, [0, 2], table, [64 * pages_in_all - 1], count, 3, 1, 1)


def test_choice_in_a_graph_with_much_shared_memory():
    lengths = [64 * 600]
    pages, table, pool = _filled(lengths, 1, 88)
    q = _randn(20, 2, 40, 64).to(torch.bfloat16).to(DEV)
    where = (_int([0, 40]), _int(table), _int(lengths))
    out = torch.empty((40, 1, 9), dtype=torch.int32, device=DEV)
    call = lambda: xsv.pages_select(pages, q, *where, 9, first=2, last=1, causal=1, out=out)
    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for i in range(3):
        q.copy_(_randn(21 + i, 2, 40, 64).to(torch.bfloat16))
        want = call().clone()
        out.fill_(7)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    want = plain.select(pool, q, [0, 40], table, lengths, 9, 2, 1, 1)
    assert all(out[r, 0].tolist() == want[r, 0] for r in range(40))


def test_choice_of_a_whole_frame():
    """Enough rows that rows share what they read."""
    lengths = [300, 64 * 20 + 5]
    pages, table, pool = _filled(lengths, 2, 89)
    q = _randn(18, 4, 75, 64).to(torch.bfloat16).to(DEV)
    _check_select(pages, pool, q, [0, 5, 75], table, lengths, 6, 1, 2, 1)
    _check_select(pages, pool, q, [0, 5, 75], table, lengths, 6, 1, 2, 59)


# ---- all of it ------------------------------------------------------------------------------------------------------

def test_a_stream_that_writes_chooses_and_attends():
    """As a model's layer uses it: rotated keys are written, queries choose pages and attend; against attention over what is read back."""
    heads, kv_heads, frames = 6, 2, [59, 200, 1, 1, 59, 1]
    total = -(-sum(frames) // 64) + 1
    pages, table = xsv.Pages.empty(total, kv_heads, DEV), _table([sum(frames)], total, 5)
    held = 0
    for f, n in enumerate(frames):
        x = _randn(90 + f, n, heads + 2 * kv_heads, 64).to(torch.bfloat16).to(DEV).transpose(0, 1)
        q, k, v = x.split([heads, kv_heads, kv_heads])
        positions = torch.arange(held, held + n, dtype=torch.int32, device=DEV)
        q, k = xsv.norm_rotate(q, k, norm="rms", positions=positions, base=10000.0)
        held += n
        where = (_int([0, n]), _int(table), _int([held]))
        xsv.pages_write(pages, k, v, *where)
        whole = xsv.pages_attend(pages, q, *where, causal=1)
        pool = plain.of(pages)
        plain.check_attend(pool, q, whole, [0, n], table, [held], 1)
        kb, vb = xsv.pages_read(pages, _int([0, held]), _int(table), _int([held]), rows=held)
        out, lse = xsv.seq_attend(q, kb, vb, _int([0, n]), _int([0, held]), causal=1)
        # two results within their bounds of the same: each off by at most 2^-8 of itself and of its weights' product
        assert bool(((out.double() - whole[0].double()).abs() <= 2.0 ** -6 * 4.5).all())
        assert bool(((lse - whole[1]).abs() <= 1e-3).all())     # 2 * 2^-17 of sum |q k| / 8, which stays below 60
        chosen = xsv.pages_select(pages, q, *where, 3, first=1, last=1, causal=1)
        want = plain.select(pool, q, [0, n], table, [held], 3, 1, 1, 1)
        assert all(chosen[r, g].tolist() == pages_of for (r, g), pages_of in want.items())
        got = xsv.pages_attend(pages, q, *where, causal=1, chosen=chosen)
        plain.check_attend(pool, q, got, [0, n], table, [held], 1, chosen=chosen.cpu())


def test_captured_calls_replay():
    """A decoding step in a graph: lengths move on between replays, in place; eager work between them; two graphs at once."""
    heads, kv_heads, lengths = 8, 2, [700, 64, 5000]
    pages, table, _ = _filled(lengths, kv_heads, 95, spare=6)
    for row, m in zip(table, lengths):
        free = [p for p in range(pages.count) if not any(p in r for r in table)]
        row[-(-m // 64):] = [free[0]] + [-1] * (len(row) - -(-m // 64) - 1) if len(row) > -(-m // 64) else []
    t, begin, held = _table_tensor(table), _int([0, 1, 2, 3]), _int(lengths)
    x = _randn(96, 3, heads + 2 * kv_heads, 64).to(torch.bfloat16).to(DEV)
    q, k, v = x.transpose(0, 1).split([heads, kv_heads, kv_heads])

    def step():
        xsv.pages_write(pages, k, v, begin, t, held, longest=1)
        chosen = xsv.pages_select(pages, q, begin, t, held, 9, causal=1, longest_q=1)
        return (chosen, *xsv.pages_attend(pages, q, begin, t, held, causal=1, longest_q=1), *xsv.pages_attend(pages, q, begin, t, held, chosen=chosen, causal=1, longest_q=1))

    step()
    graphs, results = [], []
    for _ in range(2):
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            results.append(step())
        graphs.append(g)
    for i in range(3):
        held += 1
        x.copy_(_randn(97 + i, 3, heads + 2 * kv_heads, 64).to(torch.bfloat16))
        want = [y.clone() for y in step()]
        torch.cuda.synchronize()
        for g, got in zip(graphs, results):
            g.replay()
            torch.cuda.synchronize()
            for a, b in zip(got, want):
                assert torch.equal(a, b)
    side = [torch.cuda.Stream(), torch.cuda.Stream()]
    for g, s in zip(graphs, side):
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            g.replay()
    torch.cuda.synchronize()
    for got in results:
        for a, b in zip(got, want):
            assert torch.equal(a, b)


def test_captured_calls_of_many_blocks_replay():
    """Prompts behind caches, in a graph whose launches are sized by bounds: rows and lengths move between replays."""
    pages, table, _ = _filled([1500, 900, 700], 8, 98)
    t, begin, held = _table_tensor(table), _int([0, 0, 0, 0]), _int([0, 0, 0])
    q = _many(_randn(99, 16, 300, 64).to(torch.bfloat16))

    def step():
        form = dict(causal=1, longest_q=300, longest_k=1500)
        chosen = xsv.pages_select(pages, q, begin, t, held, 5, **form)
        return (chosen, *xsv.pages_attend(pages, q, begin, t, held, **form), *xsv.pages_attend(pages, q, begin, t, held, causal=1), *xsv.pages_attend(pages, q, begin, t, held, chosen=chosen, causal=1))

    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = step()
    for rows, lengths in (([100, 1, 60], [1500, 900, 60]), ([0, 300, 0], [64, 900, 3]), ([33, 32, 31], [1400, 800, 700])):
        begin.copy_(_int(_begin(rows)))
        held.copy_(_int(lengths))
        want = [y.clone() for y in step()]
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for x, y in zip(got, want):
            assert torch.equal(x[:sum(rows)] if x.dtype == torch.int32 else x[:, :sum(rows)], y[:sum(rows)] if y.dtype == torch.int32 else y[:, :sum(rows)])


def test_calls_on_another_stream():
    lengths = [3000, 10]
    pages, table, _ = _filled(lengths, 2, 99)
    q = _randn(98, 4, 2, 64).to(torch.bfloat16).to(DEV)
    where = (_int([0, 1, 2]), _table_tensor(table), _int(lengths))
    want = xsv.pages_attend(pages, q, *where), xsv.pages_select(pages, q, *where, 5), xsv.pages_read(pages, *where, rows=2)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = xsv.pages_attend(pages, q, *where, stream=s), xsv.pages_select(pages, q, *where, 5, stream=s), xsv.pages_read(pages, *where, rows=2, stream=s)
    s.synchronize()
    assert torch.equal(got[1], want[1])
    for a, b in zip(got[0] + tuple(got[2]), want[0] + tuple(want[2])):
        assert torch.equal(a, b)


def test_pools_whose_offsets_pass_32_bits():
    """2^20 pages and heads: 4 GiB of keys, as much of values."""
    heads, total = 16, (1 << 16) + 9
    new = lambda *shape, dtype: torch.empty((total, heads) + shape, dtype=dtype, device=DEV)
    pages = xsv.Pages(new(64, 64, dtype=torch.float8_e4m3fn), new(64, 64, dtype=torch.float8_e4m3fn), new(dtype=torch.float32), new(dtype=torch.float32),
                      new(2, 64, dtype=torch.float16))
    at = [total - 1, 3, total - 4, 1 << 15]
    table, m = [at], 250
    k, v = (_randn(i, heads, m, 64).to(torch.bfloat16) for i in (5, 6))
    where = (_int([0, m]), _int(table), _int([m]))
    xsv.pages_write(pages, k.to(DEV), v.to(DEV), *where)
    part = xsv.Pages(*[x.view(torch.uint8)[at].contiguous().view(torch.float8_e4m3fn) for x in (pages.k, pages.v)], pages.k_scale[at].contiguous(),
                     pages.v_scale[at].contiguous(), pages.k_bounds[at].contiguous())
    pool = plain.Pool(4, heads)
    pool.write(k, v, [0, m], [[0, 1, 2, 3]], [m])
    _same(part, pool)
    rk, rv = xsv.pages_read(pages, *where, rows=m)
    q = _randn(7, heads, 2, 64).to(torch.bfloat16).to(DEV)
    ask = (_int([0, 2]), _int(table), _int([m]))
    got = xsv.pages_attend(pages, q, *ask, causal=1)
    plain.check_attend(pool, q, got, [0, 2], [[0, 1, 2, 3]], [m], 1, heads=[0, 9, 15])
    want = plain.select(pool, q, [0, 2], [[0, 1, 2, 3]], [m], 2, 0, 1, 1)
    chosen = xsv.pages_select(pages, q, *ask, 2, first=0, last=1, causal=1)
    assert all(chosen[r, g].tolist() == pages_of for (r, g), pages_of in want.items())
    got = xsv.pages_attend(pages, q, *ask, causal=1, chosen=chosen)
    plain.check_attend(pool, q, got, [0, 2], [[0, 1, 2, 3]], [m], 1, chosen=chosen.cpu(), heads=[0, 9, 15])
    for h in (0, 15):
        kk, vv, _ = pool.tokens([0, 1, 2, 3], m, h)
        assert torch.equal(rk[h].cpu().double(), kk) and torch.equal(rv[h].cpu().double(), vv)
