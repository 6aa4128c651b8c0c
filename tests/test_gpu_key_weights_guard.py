"""When sw_decode_attn_weights_run leaves the accumulated weights alone, and batches whose page lists do not start at the first entry."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2609_07883_b200 import binding as B
from tests import op_util as U
from tests.test_gpu_key_weights import check_weights, weigh, weights_of

pytestmark = pytest.mark.gpu


def rows_of(c, rows):
    return torch.tensor(list(rows), dtype=torch.int32, device=c.dev)


def status(c):
    return B.sw_check_status(c.ctx, raise_on_error=False)[0]


def test_expired_wait_behind_another_problem_leaves_the_weights_alone():
    """The status words keep the first problem: one that was reported before and not yet asked for must not hide an expired wait."""
    c = U.Case((32, 8, 128), [3000] * 40, seed=3)     # (enough that some page is still on its way)
    w = weights_of(c, 40, 3000)
    before = w.clone()
    kw = B.KeyWeights(w, rows_of(c, range(40)))
    page = int(c.batch.decode_pages[7])
    c.batch.decode_pages[7] = c.pages
    c.renew()
    B.sw_mixed_attn_run(c.ctx, c.pool, c.db, c.q, c.out, c.lse)      # reports a page outside the pool
    c.batch.decode_pages[7] = page
    c.renew()
    torch.cuda.synchronize()
    B._lib.sw_ctx_set_line_wait(c.ctx.handle, ctypes.c_int64(0))     # what has not arrived at the first look has expired
    weigh(c, kw)
    torch.cuda.synchronize()
    assert torch.equal(w, before)
    assert status(c) == B.SW_ERR_OUT_OF_RANGE and status(c) == B.SW_OK


@pytest.mark.parametrize("heads,lens", [((8, 2, 64), [40, 100, 30]), ((8, 1, 128), [700] * 40), ((8, 2, 64), [90] * 500)])
def test_bad_page_leaves_the_weights_alone(heads, lens):
    """The request's log-sum-exps are those of page 0's keys then.  Once the problem has been asked for, weights are written again."""
    c = U.Case(heads, lens, seed=4)
    n = len(lens)
    w = weights_of(c, n, max(lens))
    before = w.clone()
    kw = B.KeyWeights(w, rows_of(c, range(n)))
    page = int(c.batch.decode_pages[2])
    for bad in (c.pages, -1):
        c.batch.decode_pages[2] = bad
        c.renew()
        weigh(c, kw)
        c.batch.decode_pages[2] = page
        c.renew()
        weigh(c, kw)                          # (not asked for yet)
        torch.cuda.synchronize()
        assert torch.equal(w, before)
        assert status(c) == B.SW_ERR_OUT_OF_RANGE
    weigh(c, kw)
    c.ok()
    check_weights(c, before, w, list(range(n)), c.check(c.pool.double()))


@pytest.mark.parametrize("heads,lens", [((8, 2, 64), [300, 40, 1000, 17]), ((32, 8, 128), [2000, 100]), ((8, 1, 128), [500] * 40)])
def test_lists_that_start_behind_the_first_entry(heads, lens):
    """The later requests of a longer batch: decode_page_indptr starts above zero.  Weights in front of the rows in use stay as they are."""
    c = U.Case(heads, lens, seed=5)
    n, at = len(lens), 70
    c.batch.decode_pages = np.concatenate([np.full(at, -1, dtype=np.int32), c.batch.decode_pages])
    c.batch.decode_page_indptr = c.batch.decode_page_indptr + np.int32(at)
    c.renew()
    w = weights_of(c, n + 2, max(lens) + 3)
    before = w.clone()
    weigh(c, B.KeyWeights(w, rows_of(c, range(2, n + 2))))
    c.ok()
    check_weights(c, before, w, list(range(2, n + 2)), c.check(c.pool.double()))


def test_evict_in_rows_of_the_largest_capacity():
    c = U.Case((8, 1, 64), [100], seed=6)
    budget, capacity = 40, 2 ** 31 - 1
    w = torch.empty(2, 1, capacity, device=c.dev)          # 17 GB, of which the first words of each row are looked at
    w[:, :, :128] = weights_of(c, 2, 128)
    ints = lambda *v: torch.tensor(v, dtype=torch.int32, device=c.dev)  # noqa: E731
    kept, new_len = torch.full((1, 1, budget), -7, dtype=torch.int32, device=c.dev), ints(-7)
    B.sw_kv_evict(c.ctx, c.pool, c.db, B.KeyWeights(w, rows_of(c, [0])), ints(0, 3), ints(*c.free_pages()[:3]), B.KeyWeights(w, rows_of(c, [1])),
                  budget, 4, 7, kept, new_len)
    c.ok()
    want = torch.cat([torch.arange(4, device=c.dev), w[0, 0, 4:93].argsort(descending=True, stable=True)[:29].sort().values + 4, torch.arange(93, 100, device=c.dev)])
    assert new_len.tolist() == [40] and torch.equal(kept[0, 0].long(), want) and torch.equal(w[1, 0, :40], w[0, 0, want])
    del w
    torch.cuda.empty_cache()
