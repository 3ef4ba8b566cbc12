"""The paged cache in 8 bits at its limits (plain_pages is the definition in 64 bits)."""
import pytest
import torch

import plain_pages as plain
from paper_2602_21780_amd import xsv
from test_gpu_pages import DEV, _filled, _int, _randn, _table_tensor

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
