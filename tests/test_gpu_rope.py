"""Rotary positions (sw_rope_append, sw_rope_run) against the plain 64-bit form; pools are compared whole."""
import numpy as np
import pytest
import torch

from paper_2609_07883_b200 import binding as B
from tests import more_op_util as M
from tests import op_util as U

pytestmark = pytest.mark.gpu

HEADS = [(8, 2, 64), (32, 8, 128), (8, 1, 128), (4, 4, 64), (2, 1, 128), (1, 1, 64), (72, 9, 128)]
LENS = [1, 2, 15, 16, 17, 33, 1000]


def close(got, want, tol, what):
    err = (got.double() - want).abs()
    assert bool((err <= tol).all()), f"{what} off by {float((err / tol.clamp(min=1e-30)).max()):.3g} of its tolerance"


def rope_of(c, rotary, interleaved=False, scaling="plain", positions=None, magnitude=None, base=10000.0):
    turns, m = B.sw_rope_frequencies(rotary, base, scaling, 8.0, 4096, 1.0, 4.0 if scaling == "bands" else 32.0)
    return B.Rope(turns, interleaved, m if magnitude is None else magnitude, positions, device=c.dev), turns


def check_append(c, rope, turns, q, k, v, pos=None):
    """Queries, and the whole pool: the new rows rotated, everything else as it was."""
    pos = M.batch_positions(c.batch) if pos is None else pos
    before = c.pool.clone()
    B.sw_rope_append(c.ctx, c.pool, c.db, rope, q, k, v, c.out)
    c.ok()
    close(c.out, *M.rotate(q, pos, turns, rope.interleaved, rope.magnitude), "q")
    want, tol = M.rotate(k, pos, turns, rope.interleaved, rope.magnitude)
    left = torch.ones(c.pool.shape, dtype=torch.bool, device=c.dev)
    for row, count, first, pages in U.entries_of(c.batch):
        if count == 0:
            continue
        at = torch.arange(first, first + count, device=c.dev)
        ids = torch.from_numpy(np.asarray(pages, dtype=np.int64)).to(c.dev)[at // U.PAGE]
        close(c.pool[ids, 0, :, at % U.PAGE], want[row:row + count], tol[row:row + count], "k")
        assert torch.equal(c.pool[ids, 1, :, at % U.PAGE], v[row:row + count])
        left[ids, :, :, at % U.PAGE] = False
    assert torch.equal(c.pool[left], before[left])


def sliced(c):
    """q, k, v as slices of one projection's rows, with something else behind them."""
    hq, hkv, d = c.shape.num_q_heads, c.shape.num_kv_heads, c.shape.head_dim
    rows = torch.randn(c.batch.num_rows, hq + 2 * hkv + 1, d, device=c.dev).to(torch.bfloat16)
    return rows[:, :hq], rows[:, hq:hq + hkv], rows[:, hq + hkv:hq + 2 * hkv]


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("share", [1, 2, 4])
@pytest.mark.parametrize("interleaved", [False, True])
def test_append(heads, share, interleaved):
    for chunks in ([], [(0, 1)], [(37, 300)], [(100, 33), (15, 2), (0, 16)]):
        c = U.Case(heads, LENS, chunks, seed=share)
        rope, turns = rope_of(c, heads[2] // share, interleaved, "bands")
        check_append(c, rope, turns, c.q, c.k_new, c.v_new)
        c.pool.normal_()
        check_append(c, rope, turns, *sliced(c))


@pytest.mark.parametrize("rotary", [48, 80, 96, 112])
@pytest.mark.parametrize("interleaved", [False, True])
def test_parts_of_a_head(rotary, interleaved):
    c = U.Case((8, 2, 128), LENS, [(40, 70)], seed=rotary)
    rope, turns = rope_of(c, rotary, interleaved, "ramp")
    check_append(c, rope, turns, *sliced(c))


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("heads,chunks,lens", [((32, 8, 128), [(0, 8192)], []), ((16, 4, 64), [(30011, 1777)], [500] * 128), ((8, 1, 64), [(5, 3), (0, 5000)], [1] * 9)])
def test_long_batches(heads, chunks, lens, interleaved):
    c = U.Case(heads, lens, chunks, seed=8)
    rope, turns = rope_of(c, heads[2], interleaved, base=500000.0)
    check_append(c, rope, turns, c.q, c.k_new, c.v_new)


@pytest.mark.parametrize("interleaved", [False, True])
def test_given_and_far_positions(interleaved):
    c = U.Case((8, 2, 128), LENS, [(40, 20)], seed=2)
    pos = np.random.default_rng(3).integers(-2 ** 31, 2 ** 31, c.batch.num_rows)
    pos[:6] = [0, 2 ** 31 - 1, -2 ** 31, 131071, -1, 1 << 20]
    rope, turns = rope_of(c, 128, interleaved, positions=torch.from_numpy(pos.astype(np.int32)).to(c.dev), magnitude=1.25)
    check_append(c, rope, turns, c.q, c.k_new, c.v_new, pos)


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("interleaved", [False, True])
def test_run_beside_and_in_place(heads, interleaved):
    c = U.Case(heads, LENS, [(37, 65), (3, 1)], seed=5)
    rope, turns = rope_of(c, heads[2], interleaved, "linear")
    pos = M.batch_positions(c.batch)
    want = [M.rotate(x, pos, turns, interleaved, rope.magnitude) for x in (c.q, c.k_new)]
    for q, k in ((c.q, c.k_new), sliced(c)[:2]):
        wants = [M.rotate(x, pos, turns, interleaved, rope.magnitude) for x in (q, k)]
        k_out = torch.full_like(c.k_new, 7.0)
        B.sw_rope_run(c.ctx, c.db, rope, q, k, c.out, k_out)
        c.ok()
        close(c.out, *wants[0], "q")
        close(k_out, *wants[1], "k")
    B.sw_rope_run(c.ctx, c.db, rope, c.q, c.k_new, c.q, c.k_new)
    c.ok()
    close(c.q, *want[0], "q in place")
    close(c.k_new, *want[1], "k in place")


def test_rotation_keeps_lengths_and_differences():
    """Products of rotated queries and keys depend on the difference of their positions alone."""
    c = U.Case((2, 1, 128), [], [(0, 64)], seed=11)
    c.q[:], c.k_new[:] = c.q[0], c.k_new[0]
    rope, _ = rope_of(c, 128)
    k_out = torch.empty_like(c.k_new)
    B.sw_rope_run(c.ctx, c.db, rope, c.q, c.k_new, c.out, k_out)
    c.ok()
    q, k = c.out[:, 0].double(), k_out[:, 0].double()
    dots = q @ k.T
    # 128 products of two bf16 roundings each, 2^-8 of |q| |k| for either
    slack = 2 * 2.0 ** -8 * float(q.norm(dim=1).max() * k.norm(dim=1).max()) * 2
    for apart in (0, 1, 5, 40):
        line = torch.diagonal(dots, -apart)
        assert float((line - line[0]).abs().max()) <= slack
    assert float((q.norm(dim=1) - c.q[:, 0].double().norm(dim=1)).abs().max()) <= 2.0 ** -8 * float(q.norm(dim=1).max()) * 1.01


def test_non_finite_values_stay_in_their_pairs():
    c = U.Case((2, 1, 64), [5], [], seed=12)
    c.q[0, 0, 3], c.q[0, 1, 40] = float("nan"), float("inf")
    rope, _ = rope_of(c, 64)
    B.sw_rope_append(c.ctx, c.pool, c.db, rope, c.q, c.k_new, c.v_new, c.out)
    c.ok()
    bad = ~torch.isfinite(c.out[0].float())
    want = torch.zeros_like(bad)
    want[0, [3, 35]] = True
    want[1, [8, 40]] = True
    assert torch.equal(bad, want)


def test_rows_without_a_place_are_reported():
    """A page outside the pool, a list that is too short, a length of zero: no row is written, the queries are rotated all the same."""
    for spoil in ("page", "list", "length", "chunk page"):
        c = U.Case((8, 2, 64), [40, 20, 33], [(20, 20)], seed=6)
        b = c.batch
        if spoil == "page":
            b.decode_pages[int(b.decode_page_indptr[1]) - 1] = c.pages
        elif spoil == "chunk page":
            b.prefill_pages[1] = -1
        elif spoil == "length":
            b.decode_kv_len[0] = 0
        else:
            b.decode_kv_len[0] = 49            # three pages listed
        c.renew()
        rope, turns = rope_of(c, 64)
        before = c.pool.clone()
        B.sw_rope_append(c.ctx, c.pool, c.db, rope, c.q, c.k_new, c.v_new, c.out)
        assert B.sw_check_status(c.ctx, raise_on_error=False)[0] == B.SW_ERR_OUT_OF_RANGE
        close(c.out, *M.rotate(c.q, M.batch_positions(b), turns, False, 1.0), "q")
        pages = (c.pool != before).flatten(1).any(1).nonzero().flatten().tolist()
        want = {int(b.decode_pages[b.decode_page_indptr[i + 1] - 1]) for i in range(3)} | {int(b.prefill_pages[1]), int(b.prefill_pages[2])}
        if spoil in ("length", "list"):
            want -= {int(b.decode_pages[b.decode_page_indptr[1] - 1])}
        assert set(pages) == {p for p in want if 0 <= p < c.pages}


def test_followed_by_the_iteration():
    """Rotated rows of sw_rope_run through the launch that appends by itself: the same pool and output as append and attention apart."""
    for chunks in ([], [(37, 65)]):
        a, b = (U.Case((8, 2, 64), LENS, chunks, seed=21) for _ in range(2))
        rope, _ = rope_of(a, 64)
        qa = torch.empty_like(a.q)
        B.sw_rope_append(a.ctx, a.pool, a.db, rope, a.q, a.k_new, a.v_new, qa)
        B.sw_mixed_attn_run(a.ctx, a.pool, a.db, qa, a.out, a.lse)
        a.ok()
        B.sw_rope_run(b.ctx, b.db, rope, b.q, b.k_new, b.q, b.k_new)
        B.sw_mixed_iteration_run(b.ctx, b.pool, b.db, b.k_new, b.v_new, b.q, b.out, b.lse)
        b.ok()
        assert torch.equal(a.pool, b.pool) and torch.equal(qa, b.q) and torch.equal(a.out, b.out)


def test_captured():
    c = U.Case((32, 8, 128), LENS, [(37, 65)], seed=7)
    rope, turns = rope_of(c, 128)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            B.sw_rope_append(c.ctx, c.pool, c.db, rope, c.q, c.k_new, c.v_new, c.out)
        c.q.normal_()
        graph.replay()
    torch.cuda.synchronize()
    c.ok()
    close(c.out, *M.rotate(c.q, M.batch_positions(c.batch), turns, False, 1.0), "q")


def test_refusals():
    c = U.Case((8, 2, 64), [40], [(60, 20)], seed=6)
    rope, _ = rope_of(c, 64)
    k_out = torch.empty_like(c.k_new)

    def refused(status, call):
        with pytest.raises(B.SwError) as e:
            call()
        assert e.value.status == status

    append = lambda pool=c.pool, r=rope, q=c.q, k=c.k_new, v=c.v_new, out=c.out: B.sw_rope_append(c.ctx, pool, c.db, r, q, k, v, out)  # noqa: E731
    run = lambda r=rope, q=c.q, k=c.k_new, q_out=c.out, to=k_out: B.sw_rope_run(c.ctx, c.db, r, q, k, q_out, to)  # noqa: E731
    refused(B.SW_ERR_INVALID_ARG, lambda: append(pool=None))
    refused(B.SW_ERR_UNSUPPORTED, lambda: append(r=rope_of(c, 128)[0]))          # more than the head size
    one = torch.empty(c.q.numel() * 2, dtype=torch.bfloat16, device=c.dev)
    shifted = lambda t, by: one[by:by + t.numel()].view(t.shape)  # noqa: E731
    refused(B.SW_ERR_INVALID_ARG, lambda: append(q=shifted(c.q, 1)))              # alignment
    refused(B.SW_ERR_INVALID_ARG, lambda: append(q=shifted(c.q, 0), out=shifted(c.q, 8)))
    refused(B.SW_ERR_INVALID_ARG, lambda: append(v=shifted(c.v_new, 0), out=shifted(c.q, 0)))
    refused(B.SW_ERR_INVALID_ARG, lambda: run(q_out=shifted(c.q, 0), to=shifted(k_out, 64)))
    rows = torch.empty(c.batch.num_rows, 12, 64, dtype=torch.bfloat16, device=c.dev)
    refused(B.SW_ERR_INVALID_ARG, lambda: append(q=rows[:, :8], out=rows.flatten()[:c.q.numel()].view(c.q.shape)))   # in place, but not dense
    for bad in (c.q.float(), c.q[:, :4], c.q.transpose(1, 2).contiguous().transpose(1, 2)):
        with pytest.raises(ValueError):
            append(q=bad)
    with pytest.raises(ValueError):
        append(out=rows[:, :8])
    with pytest.raises(ValueError):
        append(r=rope_of(c, 64, positions=torch.zeros(3, dtype=torch.int32, device=c.dev))[0])
    append()
    run()
    c.ok()
