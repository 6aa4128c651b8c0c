"""What is not finite in an 8-bit pool (sw_kv8_attn_run): pages that no list names, and what blocks with a NaN scale reach in a chunk.

Chunks over the pool (no scratch) and over a 16-bit copy of their prompts (a scratch, and chunks long enough to be worth it)."""
import math

import pytest
import torch

from paper_2609_07883_b200 import binding as B
from tests import op_util as U

pytestmark = pytest.mark.gpu

FLOOR = 2.0 ** -32     # of the row's largest weight, per key: see op_util


def attend(c, codes, scales, scratch):
    pages = sum(-(-(P + C) // U.PAGE) for P, C, _, _ in c.batch.chunks())
    room = torch.full((B.sw_kv8_scratch_bytes(c.ctx.layout, pages),), 0xFF, dtype=torch.uint8, device=c.dev) if scratch and pages else None
    B.sw_kv8_attn_run(c.ctx, codes, scales, c.db, c.q, c.out, c.lse, room)
    c.ok()
    torch.cuda.synchronize()


def leave_page_zero_free(c):
    free = c.free_pages()
    if 0 in free:
        return
    for ids in (c.batch.decode_pages, c.batch.prefill_pages):
        ids[ids == 0] = free[-1]
    c.renew()


@pytest.mark.parametrize("heads", [(8, 2, 64), (32, 8, 128), (8, 1, 128), (4, 4, 64)])
@pytest.mark.parametrize("chunks", [[(0, 1)], [(0, 300)], [(1000, 77)], [(3000, 40), (130, 300), (0, 17)], [(700, 1500)]])
@pytest.mark.parametrize("lens", [[], [100, 1, 700]])
@pytest.mark.parametrize("scratch", [False, True])
def test_pages_that_no_list_names_may_hold_anything(heads, chunks, lens, scratch):
    c = U.Case(heads, lens, chunks, seed=len(chunks))
    leave_page_zero_free(c)
    codes, scales = U.quantise(c.pool)
    want = U.dequantise(codes, scales)
    free = c.free_pages()
    assert 0 in free
    codes.view(torch.uint8)[free] = 0x7F
    scales[free] = math.nan
    attend(c, codes, scales, scratch)
    c.check(want, floor=FLOOR)


@pytest.mark.parametrize("heads,chunk,page", [((8, 2, 64), (1000, 300), 75), ((32, 8, 128), (1000, 300), 80), ((8, 1, 128), (0, 200), 3), ((4, 4, 64), (37, 500), 20),
                                              ((32, 8, 128), (700, 1500), 100)])
@pytest.mark.parametrize("scratch", [False, True])
@pytest.mark.parametrize("how", ["scale", "codes"])
def test_nan_keys_reach_the_rows_that_attend_them(heads, chunk, page, scratch, how):
    """K of one block, some way into the chunk: the rows in front of it do not attend it, and the other heads have nothing to do with it."""
    c = U.Case(heads, [], [chunk], seed=page)
    codes, scales = U.quantise(c.pool)
    want = U.dequantise(codes, scales)
    if how == "scale":
        scales[int(c.batch.prefill_pages[page]), 0, 0] = math.nan
    else:
        codes.view(torch.uint8)[int(c.batch.prefill_pages[page]), 0, 0] = 0x7F
    attend(c, codes, scales, scratch)
    g, (P, C) = c.shape.group, chunk
    behind = (page + 1) * U.PAGE - 1 - P         # the row that attends the whole block
    assert 0 < page * U.PAGE - P < behind < C
    assert bool(torch.isnan(c.out[behind:, :g]).all()) and bool(torch.isnan(c.lse[behind:, :g]).all())
    assert not bool(torch.isnan(c.out[:, g:]).any()) and not bool(torch.isnan(c.lse[:, g:]).any())
    c.check(want, rows=slice(0, page * U.PAGE - P), floor=FLOOR)


@pytest.mark.parametrize("scratch", [False, True])
@pytest.mark.parametrize("how", ["scale", "codes", "one code"])
def test_nan_values_reach_the_rows_that_attend_them(scratch, how):
    """V of one block, or one element of it.  Rows in front whose last 128 keys hold the block may be reached too, as by the V rows of a 16-bit pool; those
    before them are not, nor is any log-sum-exp."""
    heads, (P, C), page = (32, 8, 128), (704, 1500), 100
    c = U.Case(heads, [100], [(P, C)], seed=2)
    codes, scales = U.quantise(c.pool)
    want = U.dequantise(codes, scales)
    at = int(c.batch.prefill_pages[page])
    columns = slice(None)
    if how == "scale":
        scales[at, 1, 0] = math.nan
    elif how == "codes":
        codes.view(torch.uint8)[at, 1, 0] = 0xFF
    else:
        codes.view(torch.uint8)[at, 1, 0, 0, 37] = 0x7F
        columns = slice(37, 38)
    attend(c, codes, scales, scratch)
    assert bool(torch.isnan(c.out[page * U.PAGE - P:C, :4, columns]).all())
    assert not bool(torch.isnan(c.out[:, 4:]).any()) and not bool(torch.isnan(c.lse).any())
    if how == "one code":
        assert not bool(torch.isnan(c.out[:, :, :37]).any()) and not bool(torch.isnan(c.out[:, :, 38:]).any())
    # a tile of 128 rows is 32 tokens; those that reach into the block's 128 keys start at token 1536 - P
    c.check(want, rows=list(range(page * U.PAGE // 128 * 128 - P)) + [C], floor=FLOOR)
