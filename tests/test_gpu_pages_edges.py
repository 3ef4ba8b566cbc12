"""The paged cache in 8 bits at its limits (plain_pages is the definition in 64 bits)."""
import math
import random

import pytest
import torch

import plain_pages as plain
from paper_2602_21780_amd import xsv
from test_gpu_pages import DEV, MANY, _attend_many, _begin, _check_select, _filled, _int, _randn, _table, _table_tensor

pytestmark = pytest.mark.gpu


# ---- the choice -----------------------------------------------------------------------------------------------------

def _guarded_select(pages, q, begin, table, lengths, count, **kw):
    """The choice into rows of a larger tensor, whose other rows stay as they were."""
    rows, guard = q.shape[1], 64
    room = torch.full((rows + 2 * guard, pages.kv_heads, count), 77777, dtype=torch.int32, device=DEV)
    out = room[guard:guard + rows]
    got = xsv.pages_select(pages, q, _int(begin), _table_tensor(table), _int(lengths), count, out=out, **kw)
    assert got is out and bool((room[:guard] == 77777).all()) and bool((room[guard + rows:] == 77777).all())
    return out.cpu()


@pytest.mark.parametrize("heads", [1, 2, 5])
@pytest.mark.parametrize("pages_in_all", [2100, 2500, 4097])
def test_equal_scores_of_more_pages_than_registers_hold(pages_in_all, heads):
    """More than 64 scores that equal the last chosen one: a row has its `count` lowest pages, and nothing behind them is written."""
    print(f"pages_select equal scores, pages={pages_in_all} heads={heads}", flush=True)
    pages, table, pool = _filled([64 * pages_in_all], 1, 190)
    alike = range(100, pages_in_all - 100)
    for x in (pages.k.view(torch.uint8), pages.k_scale, pages.k_bounds):
        x[[table[0][j] for j in alike]] = x[table[0][50]].clone()
    pool = plain.of(pages)
    q = _randn(191, heads, 4, 64).to(torch.bfloat16)
    q[:, 1:3] = 0.0                                   # every page the same
    for count, first, last in ((20, 0, 0), (70, 2, 3), (1000, 1, 1)):
        got = _guarded_select(pages, q.to(DEV), [0, 4], table, [64 * pages_in_all], count, first=first, last=last)
        want = plain.select(pool, q, [0, 4], table, [64 * pages_in_all], count, first, last, 0)
        assert all(got[r, 0].tolist() == want[r, 0] for r in range(4)), (count, first, last)


def _signed_pages(n, heads, seed):
    """A pool whose page j has keys c_j in channel 0 and zeros elsewhere: a few c_j above zero, some below, most of them 0."""
    rng = random.Random(seed)
    c = [rng.choice([0.5, 1.0, 1.5]) if x < 0.05 else -1.0 if x < 0.25 else 0.0 for x in (rng.random() for _ in range(n))]

    def edit(k, v):
        k[:] = 0.0
        k[..., 0] = torch.tensor(c).repeat_interleave(64)
    return _filled([64 * n], heads, seed, edit=edit)


@pytest.mark.parametrize("pages_in_all,heads", [(60, 1), (100, 1), (100, 5), (300, 2), (700, 1), (1500, 2), (2500, 1)])
def test_scores_of_zero_are_scores(pages_in_all, heads):
    """Zero queries, queries that are not finite, zero keys: many equal scores, 0 among numbers above and below, at every size of the choice."""
    print(f"pages_select scores of 0, pages={pages_in_all} heads={heads}", flush=True)
    pages, table, pool = _signed_pages(pages_in_all, 1, 200 + pages_in_all)
    q = torch.zeros((heads, 5, 64))
    q[:, 1] = math.nan
    q[:, 2, 0], q[:, 3, 0] = 3.0, -3.0        # fewer scores above 0 than are wanted; then more
    q[:, 4] = _randn(201, heads, 64)
    q = q.to(torch.bfloat16).to(DEV)
    for count, first, last in ((20, 0, 0), (32, 1, 1), (70, 2, 3), (pages_in_all - 1, 0, 0)):
        _check_select(pages, pool, q, [0, 5], table, [64 * pages_in_all], count, first, last, 0)


def test_pages_that_were_never_written_are_chosen_in_order():
    pages = xsv.Pages.empty(200, 2, DEV)
    table = [list(range(199, -1, -1))]
    q = _randn(202, 4, 3, 64).to(torch.bfloat16).to(DEV)
    got = xsv.pages_select(pages, q, _int([0, 3]), _int(table), _int([64 * 200]), 90, first=0, last=1)
    assert bool((got.cpu() == torch.tensor(list(range(89)) + [199])).all())


@pytest.mark.parametrize("heads", [1, 2, 5])
@pytest.mark.parametrize("pages_in_all", [50, 100, 300, 700, 1500, 2500])
def test_scores_that_are_no_numbers_count_as_the_lowest(pages_in_all, heads):
    """Bounds that are NaN, in more pages than are wanted and than a wave has lanes: nothing behind a row's entries is written, and pages with numbers come first."""
    print(f"pages_select NaN bounds, pages={pages_in_all} heads={heads}", flush=True)
    pages, table, _ = _filled([64 * pages_in_all], 1, 210)
    rng = random.Random(pages_in_all)
    bad = rng.sample(range(pages_in_all), pages_in_all * 2 // 5)
    pages.k_bounds[[table[0][j] for j in bad], 0, rng.randrange(2)] = math.nan
    pool = plain.of(pages)        # (its ranking leaves NaN at the lowest)
    q = _randn(211, heads, 4, 64).to(torch.bfloat16).to(DEV)
    q[:, 3] = 0.0
    for count, first, last in ((4, 0, 0), (9, 2, 3), (pages_in_all * 4 // 5, 0, 0), (pages_in_all, 1, 0)):
        got = _guarded_select(pages, q, [0, 4], table, [64 * pages_in_all], count, first=first, last=last)
        want = plain.select(pool, q, [0, 4], table, [64 * pages_in_all], count, first, last, 0)
        assert all(got[r, 0].tolist() == want[r, 0] for r in range(4)), (count, first, last)


@pytest.mark.parametrize("heads", [1, 2, 5])
def test_bounds_of_any_bits(heads):
    """What a pool of memory as it came may hold: lists stay lists, and the same ones every time."""
    for n in (50, 400, 2500):
        pages, table, _ = _filled([64 * n], 2, 212)
        g = torch.Generator().manual_seed(n)
        pages.k_bounds.copy_(torch.randint(-32768, 32768, pages.k_bounds.shape, generator=g, dtype=torch.int16).view(torch.float16))
        pages.k_scale.copy_(torch.randint(-2**31, 2**31 - 1, pages.k_scale.shape, generator=g, dtype=torch.int32).view(torch.float32))
        q = _randn(213, 2 * heads, 6, 64).to(torch.bfloat16).to(DEV)
        for count in (4, 70):
            got = _guarded_select(pages, q, [0, 6], table, [64 * n], count, first=1, last=1)
            some = min(count, n)
            assert bool((got[..., 0] == 0).all()) and bool((got[..., some - 1] == n - 1).all()) and bool((got[..., some:] == -1).all())
            assert bool((got[..., 1:some] > got[..., :some - 1]).all())
            assert torch.equal(got, _guarded_select(pages, q, [0, 6], table, [64 * n], count, first=1, last=1))


# ---- lengths behind the table ---------------------------------------------------------------------------------------

@pytest.mark.parametrize("length", [129, 133, 138, 200, 1 << 20, (1 << 31) - 1])
def test_rows_behind_the_table_are_left_out(length):
    """They are not written over what is held, not read from there, and the others keep their places."""
    print(f"pages behind the table: length={length}", flush=True)
    pages, table, pool = _filled([128], 2, 220)
    k, v = (_randn(221 + i, 2, 10, 64).to(torch.bfloat16) for i in range(2))
    xsv.pages_write(pages, k.to(DEV), v.to(DEV), _int([0, 10]), _int(table), _int([length]))
    inside = max(128 - (length - 10), 0)           # rows in front of the table's end
    if inside:
        pool.write(k[:, :inside], v[:, :inside], [0, inside], table, [128])
    got = plain.of(pages)
    for name in ("k", "v", "ke", "ve", "bounds"):
        for p in table[0]:
            assert torch.equal(getattr(got, name)[p], getattr(pool, name)[p]), (name, p)
    out = [torch.full((2, 10, 64), 9.0, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    xsv.pages_read(pages, _int([0, 10]), _int(table), _int([length]), out=out)
    for h in range(2):
        for want, x in zip(pool.tokens(table[0], 128, h), out):
            full = torch.full((10, 64), 9.0, dtype=torch.float64)
            full[:inside] = want[128 - inside:]
            assert torch.equal(x[h].cpu().double(), full)


@pytest.mark.parametrize("causal", [0, 1, 59])
@pytest.mark.parametrize("rows", [10, 70])
def test_rows_keep_their_positions_where_a_length_is_behind_the_table(rows, causal):
    held, length = 64 * 20, 64 * 20 + 25
    pages, table, pool = _filled([held], 2, 222)
    q = (_randn(223, 4, rows, 64) * 1.5).to(torch.bfloat16)
    where = (_int([0, rows]), _int(table), _int([length]))
    sees = [min(plain.limit(i, rows, length, causal), held) for i in range(rows)]
    lists = torch.randint(0, 20, (rows, 2, 5), generator=torch.Generator().manual_seed(7), dtype=torch.int32)
    whole = xsv.pages_attend(pages, q.to(DEV), *where, causal=causal)
    some = xsv.pages_attend(pages, q.to(DEV), *where, causal=causal, chosen=lists.to(DEV))
    choice = xsv.pages_select(pages, q.to(DEV), *where, 6, first=1, last=2, causal=causal).cpu()
    for i in range(rows):
        one = slice(i, i + 1)
        plain.check_attend(pool, q[:, one], [x[:, one] for x in whole], [0, 1], table, [sees[i]], 0)
        plain.check_attend(pool, q[:, one], [x[:, one] for x in some], [0, 1], table, [sees[i]], 0, chosen=lists[one])
        want = plain.select(pool, q[:, one], [0, 1], table, [sees[i]], 6, 1, 2, 0)
        assert [choice[i, g].tolist() for g in range(2)] == [want[0, g] for g in range(2)]
    pages, table, pool = _filled([held], 8, 224)
    q = q.repeat(4, 1, 1)
    many = _attend_many(pages, q, [0, rows], table, [length], causal=causal)
    for i in (0, rows - 26, rows - 25, rows - 1) if rows > 26 else (0, rows - 1):
        one = slice(i, i + 1)
        plain.check_attend(pool, q[:, one], [x[:, one] for x in many], [0, 1], table, [sees[i]], 0, heads=[0, 15])


# ---- the largest numbers --------------------------------------------------------------------------------------------

def test_the_largest_finite_numbers_stay_finite():
    """Above 248 2^120 the nearest code would stand for 2^128, which bf16 does not hold: 240 2^120 is the largest that a page stands for."""
    bits = [0x7f7f, 0x7f7e, 0x7f78, 0x7f77, 0x7f70, 0x7f6f, 0x7f00]      # the largest; 248 2^120 and the one below; 240 2^120 and the one below; 2^127
    x = torch.tensor(bits, dtype=torch.int32)
    x = torch.cat([x, x | 0x8000, torch.tensor([0x3f80, 0x7f80, 0x7fc0], dtype=torch.int32)])
    k = torch.zeros((1, 70, 64))
    k[0, 3, :17] = (x << 16).view(torch.float32)
    k[0, 66, 5], k[0, 69, 6] = k[0, 3, 0], -k[0, 3, 0]
    k, v = k.to(torch.bfloat16), (-k).to(torch.bfloat16)
    pages, pool = xsv.Pages.empty(2, 1, DEV), plain.Pool(2, 1)
    for begin, held in ((0, 65), (65, 70)):      # the second page in two calls, the second of which raises its scale
        a, b = (y[:, begin:held].contiguous() for y in (k, v))
        xsv.pages_write(pages, a.to(DEV), b.to(DEV), _int([0, held - begin]), _int([[1, 0]]), _int([held]))
        pool.write(a, b, [0, held - begin], [[1, 0]], [held])
    top = torch.where(pool.ke == 120, 240.0, 448.0)[:, :, None, None]
    assert bool((pool.ke == 120).all()) and bool((pool.ve == 120).all())
    assert int((pool.k == 256.0).sum()) == 4 and int((pool.k == -256.0).sum()) == 4      # what the definition without the limit gives
    pool.k, pool.v, pool.bounds = (torch.maximum(torch.minimum(y, t), -t) for y, t in ((pool.k, top), (pool.v, top), (pool.bounds, 2 * top)))
    got = plain.of(pages)
    for name in ("k", "v", "ke", "ve", "bounds"):
        assert torch.equal(torch.nan_to_num(getattr(got, name), 1e9), torch.nan_to_num(getattr(pool, name), 1e9)), name
    rk, rv = xsv.pages_read(pages, _int([0, 70]), _int([[1, 0]]), _int([70]), rows=70)
    for x, r in zip(pool.tokens([1, 0], 70, 0), (rk, rv)):
        assert torch.equal(torch.nan_to_num(r[0].cpu().double(), 1e9), torch.nan_to_num(x, 1e9))
    for x, r in ((k, rk), (v, rv)):
        assert torch.equal(torch.isfinite(r.cpu()), torch.isfinite(x))


def test_attention_over_the_largest_finite_numbers():
    """One token, so that no sum passes what fp32 holds; small queries, so that no logit does."""
    top = torch.tensor([0x7f7f0000], dtype=torch.int32).view(torch.float32)
    k = torch.zeros((1, 1, 64))
    k[0, 0, 0], k[0, 0, 1] = top, -top
    k = k.to(torch.bfloat16).to(DEV)
    pages = xsv.Pages.empty(1, 1, DEV)
    xsv.pages_write(pages, k, -k, _int([0, 1]), _int([[0]]), _int([1]))
    for heads, rows in ((1, 1), (1, 40), (40, 1)):       # (rows in front of the only token see nothing)
        q = torch.zeros((heads, rows, 64))
        q[..., 0] = 2.0 ** -126
        out, lse = xsv.pages_attend(pages, q.to(torch.bfloat16).to(DEV), _int([0, rows]), _int([[0]]), _int([1]))
        assert not out[:, :-1].any() and bool((lse[:, :-1] == -math.inf).all())
        out, lse = out[:, -1], lse[:, -1]
        assert bool((out[:, 0] == -240.0 * 2.0 ** 120).all()) and bool((out[:, 1] == 240.0 * 2.0 ** 120).all()) and not out[:, 2:].any()
        assert bool(((lse.cpu().double() - 240.0 * 2.0 ** -6 / 8).abs() <= 1e-6).all())      # 0.47: a few roundings of 2^-24


# ---- scales of nothing ----------------------------------------------------------------------------------------------

# of a key of channel 0 and a query of it, under a scale of 1/8
LOGITS = {20.0: (20.0, 8.0), 18.703125: (18.0, 8.3125)}


def _one_large(logit, q_rows, heads, kv_heads, page_count):
    """One key with a large logit among page_count pages with logits of 0 whose values are zeros but for its own page's."""
    def edit(k, v):
        k[:] = 0.0
        k[:, 70, 0] = LOGITS[logit][0]
        v[:, :64], v[:, 128:] = 0.0, 0.0
    pages, table, pool = _filled([64 * page_count], kv_heads, 230, edit=edit)
    q = torch.zeros((heads, q_rows, 64))
    q[..., 0] = LOGITS[logit][1]
    return pages, table, pool, q.to(torch.bfloat16)


def _check_one_large(logit, pool, table, got, n):
    heads = got[0].shape[0]
    rep = heads // pool.k.shape[1]
    total = math.exp(logit) + n - 1
    # lse: six roundings of 2^-24 of numbers of at most 20 (of the factor two, the product, the difference from the reference, and two at the end), 7.2e-6;
    # and a wave adds up its pages, at least every fourth, in two halves at most, each time rounding a sum that is near 1 by up to 2^-24
    bound = 7.2e-6 + n / 64 / 4 * 2 * 2.0 ** -24
    for h in (0, heads - 1):
        _, v, _ = pool.tokens(table[0], 192, h // rep)
        want = (v.sum(0) + (math.exp(logit) - 1.0) * v[70]) / total
        off = (got[1][h].cpu().double() - math.log(total)).abs()
        assert bool((off <= bound).all()), (float(off.max()), bound)
        assert bool(((got[0][h].cpu().double() - want).abs() <= 2.0 ** -8 * 2.1 * want.abs() + 1e-6).all())


@pytest.mark.parametrize("logit", list(LOGITS))
@pytest.mark.parametrize("rows", [1, 3, 40])
def test_tokens_without_values_count_in_the_sum(rows, logit):
    """131071 logits of 0 beside one of 20 (19): 3e-4 (1e-3) of the sum, though each weight is below 2^-26 of the largest and its value is 0."""
    pages, table, pool, q = _one_large(logit, rows, 2, 2, 2048)
    got = xsv.pages_attend(pages, q.to(DEV), _int([0, rows]), _int(table), _int([64 * 2048]))
    _check_one_large(logit, pool, table, got, 64 * 2048)
    lists = torch.arange(2047, -1, -1, dtype=torch.int32, device=DEV).expand(rows, 2, 2048).contiguous()
    got = xsv.pages_attend(pages, q.to(DEV), _int([0, rows]), _int(table), _int([64 * 2048]), chosen=lists)
    _check_one_large(logit, pool, table, got, 64 * 2048)


@pytest.mark.parametrize("logit", list(LOGITS))
@pytest.mark.parametrize("form", ["32 rows", "64 rows", "chosen"])
def test_tokens_without_values_count_in_the_sum_of_many_blocks(form, logit):
    """Launches of so many blocks that the wave that has the large logit has many of the other pages, too."""
    if form == "32 rows":
        pages, table, pool, q = _one_large(logit, 1374, 8, 8, 2048)
        got = xsv.pages_attend(pages, q.to(DEV), _int([0, 1374]), _int(table), _int([64 * 2048]))
        _check_one_large(logit, pool, table, got, 64 * 2048)
        return
    pages, table, pool, q = _one_large(logit, 70, 16, 8, 1024)
    lists = torch.arange(1024, dtype=torch.int32, device=DEV).expand(MANY, 8, 1024).contiguous()
    got = _attend_many(pages, q, [0, 70], table, [64 * 1024], chosen=lists if form == "chosen" else None)
    _check_one_large(logit, pool, table, got, 64 * 1024)


@pytest.mark.parametrize("rows", [1, 40, 300])
def test_pages_of_tiny_values(rows):
    """Values of 2^-50 to 2^-90, a page each, some of them NaN, beside zeros: results in their size, and rows that see a NaN."""
    def edit(k, v):
        for i in range(12):
            v[:, 64 * i:64 * i + 64] *= 2.0 ** (-50 - 10 * (i % 5)) if i % 6 else 0.0
        v[0, 64 * 7 + 3, 5] = math.nan
    pages, table, pool = _filled([64 * 12], 8, 231, edit=edit)
    q = (_randn(232, 16, rows, 64) * 1.5).to(torch.bfloat16)
    for causal in (0, 1):
        got = xsv.pages_attend(pages, q.to(DEV), _int([0, rows]), _int(table), _int([64 * 12]), causal=causal)
        plain.check_attend(pool, q, got, [0, rows], table, [64 * 12], causal, heads=[0, 1, 15])
    got = _attend_many(pages, q, [0, rows], table, [64 * 12], causal=1)
    plain.check_attend(pool, q, got, [0, rows], table, [64 * 12], 1, heads=[0, 1, 15])
    for j in range(12):      # one page alone: of its own size
        lists = torch.full((rows, 8, 1), j, dtype=torch.int32)
        got = xsv.pages_attend(pages, q.to(DEV), _int([0, rows]), _int(table), _int([64 * 12]), chosen=lists.to(DEV))
        for h in (0, 15):
            k, v, _ = pool.tokens(table[0], 64 * 12, h // 2)
            P = torch.softmax(q[h].double() @ k[64 * j:64 * j + 64].T * 0.125, 1)
            V = v[64 * j:64 * j + 64]
            want, weight = P @ V, P @ V.abs()
            o = got[0][h].cpu().double()
            assert torch.equal(torch.isnan(o), torch.isnan(want))
            fine = ~torch.isnan(want)
            # weights and results are rounded to 2^-8; logits below 2^-17 of what they add up from
            assert bool(((o - want).abs()[fine] <= 2.0 ** -8 * 1.1 * (want.abs() + weight)[fine]).all()), (j, h)


# ---- many sequences -------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("sequences,rows", [(65, 100000), (200, 40000), (4200, 5000)])
def test_choice_for_any_number_of_sequences_within_a_bound_far_above_their_rows(sequences, rows):
    """The launch is sized by the rows and the sequences, not by their product."""
    lengths = [130 + s % 64 for s in range(sequences)]
    pages, table, pool = _filled(lengths, 16, 240)
    q = torch.zeros((16, rows, 64), dtype=torch.bfloat16, device=DEV)
    q[:, :sequences] = _randn(241, 16, sequences, 64).to(torch.bfloat16).to(DEV)
    call = lambda **kw: xsv.pages_select(pages, q, _int(_begin([1] * sequences)), _table_tensor(table), _int(lengths), 2, causal=1, **kw)
    assert torch.equal(call(), call(longest_q=1))


@pytest.mark.parametrize("sequences,rows", [(1000, 100000), (5000, 20000)])
def test_writes_of_any_number_of_sequences_within_a_bound_far_above_their_rows(sequences, rows):
    lengths = [1 + s % 130 for s in range(sequences)]
    k, v = (torch.zeros((16, rows, 64), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    k[:, :sequences], v[:, :sequences] = (_randn(242 + i, 16, sequences, 64).to(torch.bfloat16).to(DEV) for i in range(2))
    total = sum(-(-m // 64) for m in lengths)
    where = (_int(_begin([1] * sequences)), _table_tensor(_table(lengths, total, 7)), _int(lengths))
    pools, read = [xsv.Pages.empty(total, 16, DEV) for _ in range(2)], []
    for pages, longest in zip(pools, (None, 1)):
        xsv.pages_write(pages, k, v, *where, longest=longest)
        read.append(xsv.pages_read(pages, *where, rows=rows, longest=longest))
        assert bool(read[-1][0][:, :sequences].any(2).all())
    for name in ("k", "v", "k_scale", "v_scale", "k_bounds"):
        a, b = (getattr(p, name) for p in pools)
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), name
    assert torch.equal(read[0][0], read[1][0]) and torch.equal(read[0][1], read[1][1])


def _uneven(sequences, seed, rows):
    """Rows and lengths of many sequences, some of no rows, some of no tokens, one far longer than the others."""
    rng = random.Random(seed)
    new = [rng.choice([0, 1, 1, 2, 5, 37]) for _ in range(sequences)]
    new[sequences // 3] = rows
    lengths = [max(n + rng.choice([-2, 0, 0, 5, 100]), 0) for n in new]
    return new, lengths


@pytest.mark.parametrize("sequences", [65, 200, 4200])
def test_rows_of_many_uneven_sequences(sequences):
    """Written, read, attended to and chosen for within no bound: blocks are found by number among 64 offsets at a time, twice and more."""
    print(f"pages of many sequences {sequences}", flush=True)
    new, lengths = _uneven(sequences, sequences, 700)
    begin = _begin(new, 3)
    total, rows = sum(-(-m // 64) for m in lengths) + 2, sum(new) + 5
    table = _table(lengths, total, 9)
    where = (_int(begin), _table_tensor(table), _int(lengths))
    pages, pool = xsv.Pages.empty(total, 2, DEV), plain.Pool(total, 2)
    k, v = (_randn(250 + i, 2, rows, 64).to(torch.bfloat16) for i in range(2))
    xsv.pages_write(pages, k.to(DEV), v.to(DEV), *where)
    pool.write(k, v, begin, table, lengths)
    got = plain.of(pages)
    for name in ("k", "v", "bounds"):
        assert torch.equal(getattr(got, name)[pool.written], getattr(pool, name)[pool.written]), name
    assert not got.k[~pool.written].any()
    pool = got
    for x, y in zip(xsv.pages_read(pages, *where, rows=rows), xsv.pages_read(pages, *where, rows=rows, longest=max(new))):
        assert torch.equal(x, y)
    q = _randn(252, 4, rows, 64).to(torch.bfloat16).to(DEV)
    lists = torch.randint(-1, 12, (rows, 2, 3), generator=torch.Generator().manual_seed(8), dtype=torch.int32)
    some = range(sequences) if sequences < 1000 else sorted({0, 1, sequences // 3, sequences - 1, *random.Random(1).sample(range(sequences), 400)})
    parts = ([begin[s] for s in some], [begin[s + 1] for s in some])

    def each(check):
        for s, a, b in zip(some, *parts):
            if s == sequences // 3 and sequences > 65:
                b = a + 40                  # (the long one's first rows: its length goes by the cut)
            check([a, b], [table[s]], [lengths[s] - (begin[s + 1] - b)], s)
    whole, chosen = xsv.pages_attend(pages, q, *where, causal=1), xsv.pages_attend(pages, q, *where, causal=1, chosen=lists.to(DEV))
    choice = xsv.pages_select(pages, q, *where, 3, first=0, last=1, causal=1)
    each(lambda be, t, m, s: plain.check_attend(pool, q, whole, be, t, m, 1, heads=[0, 3]))
    each(lambda be, t, m, s: plain.check_attend(pool, q, chosen, be, t, m, 1, chosen=lists, heads=[3]))
    for x in (*whole, *chosen):
        assert not x[:, :3].any() and not x[:, begin[-1]:].any()
    assert torch.equal(choice, xsv.pages_select(pages, q, *where, 3, first=0, last=1, causal=1, longest_q=max(new)))

    def check(be, t, m, s):
        for (r, g), want in plain.select(pool, q, be, t, m, 3, 0, 1, 1).items():
            assert choice[r, g].tolist() == want, (s, r, g)
    choice = choice.cpu()
    each(check)


def test_offsets_that_do_not_ascend_are_within_bounds():
    """Offsets that begin again: what is written is written within the tensors, and the first and last sequences' rows are answered."""
    sequences = 300
    lengths = [70] * sequences
    pages, table, pool = _filled(lengths, 1, 253)
    begin = [min(s * 10, 1500) if s < 150 else max(1500 - 10 * (s - 150), -50) for s in range(sequences + 1)]
    q = _randn(254, 2, 1500, 64).to(torch.bfloat16).to(DEV)
    out = torch.zeros((2, 1564, 64), dtype=torch.bfloat16, device=DEV)
    room = out[:, :1500]
    got = xsv.pages_attend(pages, q, _int(begin), _table_tensor(table), _int(lengths), out=room, causal=1)
    assert not out[:, 1500:].any() and bool(torch.isfinite(got[0]).all())
    plain.check_attend(pool, q, got, begin[:2], table[:1], lengths[:1], 1)
