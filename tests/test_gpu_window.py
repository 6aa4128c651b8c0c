"""Attention inside a sliding window with sinks (sw_mixed_attn_window_run, sw_mixed_iteration_window_run) against the plain 64-bit form."""
import math

import numpy as np
import pytest
import torch

from paper_2609_07883_b200 import binding as B
from tests import op_util as U

pytestmark = pytest.mark.gpu

HEADS = [(8, 2, 64), (32, 8, 128), (8, 1, 128), (4, 4, 64), (16, 8, 128), (8, 1, 64)]
LENS = [1, 2, 15, 16, 17, 31, 100, 257, 1000, 2049]


def forget(case, window, sinks):
    """Pages that no row of a request or chunk attends: bad ids for half of them, NaN rows for the others; attended pages keep theirs.  Keys that
    are not attended inside the window's first page become NaN where no chunk row needs them."""
    b = case.batch
    for i in range(b.num_decode):
        n, at = int(b.decode_kv_len[i]), int(b.decode_page_indptr[i])
        for j in range(-(-n // U.PAGE)):
            keys = np.arange(j * U.PAGE, min(n, j * U.PAGE + U.PAGE))
            seen = (keys > n - 1 - window) | (keys < sinks)
            case.pool[int(b.decode_pages[at + j]), :, :, [int(k) % U.PAGE for k in keys[~seen]]] = math.nan
            if not seen.any():
                b.decode_pages[at + j] = -1 - j if j % 2 else b.decode_pages[at + j]
    case.renew()


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("window,sinks", [(1, 0), (5, 4), (16, 0), (17, 16), (100, 1), (130, 300), (5000, 4), (1 << 30, 1 << 30)])
def test_decode(heads, window, sinks):
    c = U.Case(heads, LENS, seed=window % 97 + sinks)
    forget(c, window, sinks)
    B.sw_mixed_attn_window_run(c.ctx, c.pool, c.db, window, sinks, c.q, c.out, c.lse)
    c.ok()
    c.check(c.pool.double(), window, sinks)


@pytest.mark.parametrize("heads,n", [((8, 2, 64), 500), ((8, 1, 128), 40)])   # more than a line takes; groups of eight at head size 128
def test_decode_units(heads, n):
    rng = np.random.default_rng(n)
    c = U.Case(heads, rng.integers(1, 700 if n < 100 else 200, n), seed=n)
    forget(c, 60, 20)
    B.sw_mixed_attn_window_run(c.ctx, c.pool, c.db, 60, 20, c.q, c.out, c.lse)
    c.ok()
    c.check(c.pool.double(), 60, 20)


def test_long_contexts_short_window():
    c = U.Case((32, 8, 128), [20000, 16384, 8191], seed=3)
    forget(c, 1000, 4)
    B.sw_mixed_attn_window_run(c.ctx, c.pool, c.db, 1000, 4, c.q, c.out, c.lse)
    c.ok()
    c.check(c.pool.double(), 1000, 4)


def test_empty_request_is_left_alone():
    c = U.Case((8, 2, 64), [40, 0, 50])
    c.out.fill_(7)
    c.lse.fill_(7)
    B.sw_mixed_attn_window_run(c.ctx, c.pool, c.db, 20, 2, c.q, c.out, c.lse)
    c.ok()
    c.check(c.pool.double(), 20, 2)
    assert bool((c.out[1] == 7).all()) and bool((c.lse[1] == 7).all())


CHUNKS = [([(0, 1)], 3, 0), ([(0, 300)], 64, 4), ([(1000, 77)], 100, 0), ([(1000, 513)], 200, 130), ([(2000, 130)], 1, 1), ([(4111, 300)], 128, 4),
          ([(500, 256)], 5000, 4), ([(3000, 40), (130, 300), (0, 17)], 150, 5), ([(2500, 700), (2500, 700)], 1000, 0), ([(6000, 20)], 2500, 40)]


@pytest.mark.parametrize("heads", [(8, 2, 64), (32, 8, 128), (8, 1, 128), (4, 4, 64)])
@pytest.mark.parametrize("chunks,window,sinks", CHUNKS)
def test_chunks(heads, chunks, window, sinks):
    c = U.Case(heads, [100, 1, 700], chunks, seed=len(chunks) + window)
    # pages in front of every row's window may belong to somebody else
    b = c.batch
    lists = b.chunk_page_indptr if b.chunk_page_indptr is not None else [0]
    for (P, C, _, pages), at in zip(b.chunks(), lists):
        for j in range(len(pages)):
            if j * U.PAGE >= sinks and j * U.PAGE + U.PAGE <= P + 1 - window:
                c.pool[int(pages[j])] = math.nan
                b.prefill_pages[int(at) + j] = -5
    c.renew()
    B.sw_mixed_attn_window_run(c.ctx, c.pool, c.db, window, sinks, c.q, c.out, c.lse)
    c.ok()
    c.check(c.pool.double(), window, sinks)


@pytest.mark.parametrize("heads,lens,chunks", [((32, 8, 128), [300, 17, 4000], [(1500, 200)]), ((8, 2, 64), [33, 64, 1], []), ((8, 1, 128), [500] * 5, []),
                                               ((16, 4, 64), [5], [(40, 300), (16, 33)])])
def test_iteration_appends_and_attends(heads, lens, chunks):
    c = U.Case(heads, lens, chunks, seed=11)
    want = c.pool.clone()
    for row, count, pos, pages in U.entries_of(c.batch):
        for r in range(count):
            page, slot = int(pages[(pos + r) // U.PAGE]), (pos + r) % U.PAGE
            want[page, 0, :, slot], want[page, 1, :, slot] = c.k_new[row + r], c.v_new[row + r]
    B.sw_mixed_iteration_window_run(c.ctx, c.pool, c.db, 70, 3, c.k_new, c.v_new, c.q, c.out, c.lse)
    c.ok()
    assert torch.equal(c.pool, want)
    c.check(want.double(), 70, 3)


def test_full_window_is_the_plain_iteration():
    c = U.Case((32, 8, 128), [300, 5000], seed=5)
    B.sw_mixed_attn_window_run(c.ctx, c.pool, c.db, 6000, 0, c.q, c.out, c.lse)
    out, lse = c.out.clone(), c.lse.clone()
    B.sw_mixed_attn_run(c.ctx, c.pool, c.db, c.q, c.out, c.lse)
    c.ok()
    assert torch.equal(out, c.out) and torch.equal(lse, c.lse)


def test_captured_and_replayed_on_another_stream():
    c = U.Case((32, 8, 128), [300, 5000, 40], [(700, 100)], seed=6)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        B.sw_mixed_attn_window_run(c.ctx, c.pool, c.db, 90, 3, c.q, c.out, c.lse, stream=s)
    for seed in (1, 2):
        c.q.copy_(torch.randn(c.q.shape, generator=torch.Generator().manual_seed(seed)))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        c.ok()
        c.check(c.pool.double(), 90, 3)


def test_refusals():
    c = U.Case((8, 2, 64), [40])
    for window, sinks in [(0, 0), (-1, 0), (5, -1)]:
        with pytest.raises(B.SwError) as e:
            B.sw_mixed_attn_window_run(c.ctx, c.pool, c.db, window, sinks, c.q, c.out)
        assert e.value.status == B.SW_ERR_INVALID_ARG
    with pytest.raises(B.SwError) as e:
        B.sw_mixed_iteration_window_run(c.ctx, c.pool, c.db, 5, 0, None, c.v_new, c.q, c.out)
    assert e.value.status == B.SW_ERR_INVALID_ARG
    with pytest.raises(B.SwError) as e:
        B.sw_mixed_attn_window_run(c.ctx, c.pool, c.db, 5, 0, None, c.out)
    assert e.value.status == B.SW_ERR_INVALID_ARG
