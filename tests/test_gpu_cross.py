"""Cross attention to cached encoder states (sw_cross_attn_run) against the plain 64-bit form."""
import math

import numpy as np
import pytest
import torch

from paper_2609_07883_b200 import binding as B
from tests import more_op_util as M

pytestmark = pytest.mark.gpu

HEADS = [(8, 2, 64), (32, 8, 128), (8, 1, 128), (4, 4, 64), (16, 8, 128), (8, 1, 64)]
LENS = [1, 0, 2, 15, 16, 17, 31, 100, 0, 257, 1000, 2049, 0]


def run(c, rows=slice(None)):
    B.sw_cross_attn_run(c.ctx, c.pool, c.db, c.q, c.out, c.lse)
    c.ok()
    c.check_cross(rows)


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("keys", [1, 15, 16, 17, 127, 128, 129, 500, 1025])
@pytest.mark.parametrize("rows", [1, 33, 128, 200])
def test_one_chunk(heads, keys, rows):
    run(M.CrossCase(heads, [], [(keys, rows)], seed=keys + rows))


@pytest.mark.parametrize("heads", HEADS)
def test_decode(heads):
    run(M.CrossCase(heads, LENS, seed=3))


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("chunks", [[(300, 100), (17, 260), (1, 1)], [(0, 5), (130, 64)], [(130, 64), (0, 70), (40, 3)], [(130, 64), (40, 3), (0, 33)],
                                    [(0, 9), (64, 31), (0, 2)], [(0, 40)], [(0, 3), (0, 4)],
                                    [(2000, 1), (1000, 2), (500, 64), (250, 65), (100, 7), (16, 128), (3, 1), (1, 129)]])
@pytest.mark.parametrize("lens", [[], LENS, [0, 0]])
def test_several_chunks(heads, chunks, lens):
    run(M.CrossCase(heads, lens, chunks, seed=len(chunks) + len(lens)))


def test_only_requests_without_keys():
    run(M.CrossCase((8, 2, 64), [0, 0, 0]))
    run(M.CrossCase((8, 2, 64), [0] * 500))


@pytest.mark.parametrize("heads,n", [((8, 2, 64), 500), ((8, 1, 128), 40)])   # more than a line takes; groups of eight at head size 128
def test_decode_units(heads, n):
    rng = np.random.default_rng(n)
    run(M.CrossCase(heads, rng.integers(0, 300, n) * (rng.random(n) < 0.8), seed=n))


@pytest.mark.parametrize("heads,lens,chunks", [
    ((32, 8, 128), [], [(20000, 40)]),                                  # items cut into pieces
    ((32, 8, 128), [1500] * 64 + [0], [(4111, 448), (1500, 224), (333, 77)]),
    ((32, 8, 128), [], [(700, 4500)]),                                  # whole rounds of items
    ((32, 8, 128), [4000] * 90, [(1500, 4200)]),                        # beside enough pages that CTAs take no entry
    ((16, 16, 64), [1500] * 70, [(1500, 300), (900, 300)]),
])
def test_large(heads, lens, chunks):
    run(M.CrossCase(heads, lens, chunks, seed=len(lens)))


def test_long_chunk_over_one_page_row_by_row():
    """As many rows as keys, more rows than keys and the other way round: no row's place in the chunk matters."""
    c = M.CrossCase((8, 2, 64), [], [(200, 200)], seed=9)
    c.q[:] = c.q[0]
    B.sw_cross_attn_run(c.ctx, c.pool, c.db, c.q, c.out, c.lse)
    c.ok()
    assert bool((c.out == c.out[0]).all()) and bool((c.lse == c.lse[0]).all())
    c.check_cross()


def test_without_lse_and_captured():
    c = M.CrossCase((32, 8, 128), [100, 0, 1500], [(500, 70), (0, 3)], seed=4)
    B.sw_cross_attn_run(c.ctx, c.pool, c.db, c.q, c.out)
    c.ok()
    out = c.out.clone()
    assert bool(torch.isnan(c.lse).all())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            B.sw_cross_attn_run(c.ctx, c.pool, c.db, c.q, c.out, c.lse)
        for _ in range(3):
            c.out.fill_(math.nan)
            c.lse.fill_(math.nan)
            graph.replay()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert torch.equal(c.out, out)
    c.ok()
    c.check_cross()


def test_pages_outside_the_pool_are_reported():
    for where in ("prefill_pages", "decode_pages"):
        c = M.CrossCase((8, 2, 64), [40, 20], [(60, 20)], seed=6)
        getattr(c.batch, where)[1] = c.pages
        c.renew()
        B.sw_cross_attn_run(c.ctx, c.pool, c.db, c.q, c.out, c.lse)
        assert B.sw_check_status(c.ctx, raise_on_error=False)[0] == B.SW_ERR_OUT_OF_RANGE
        c = M.CrossCase((8, 2, 64), [40, 20], [(60, 20)], seed=6)
        run(c)


def test_refusals():
    c = M.CrossCase((8, 2, 64), [40], [(60, 20)], seed=6)
    c.db.struct.num_prefill_pages = 3          # 60 keys lie on four pages
    with pytest.raises(B.SwError) as e:
        B.sw_cross_attn_run(c.ctx, c.pool, c.db, c.q, c.out)
    assert e.value.status == B.SW_ERR_OUT_OF_RANGE
    c.db.struct.num_prefill_pages = 4
    for args in [(None, c.q, c.out), (c.pool, None, c.out), (c.pool, c.q, None)]:
        with pytest.raises(B.SwError) as e:
            B.sw_cross_attn_run(c.ctx, args[0], c.db, args[1], args[2])
        assert e.value.status == B.SW_ERR_INVALID_ARG
    off = torch.empty(c.q.numel() + 1, dtype=torch.bfloat16, device=c.dev)[1:]
    with pytest.raises(B.SwError) as e:
        B.sw_cross_attn_run(c.ctx, c.pool, c.db, c.q, off)
    assert e.value.status == B.SW_ERR_INVALID_ARG
    run(c)
