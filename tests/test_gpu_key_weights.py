"""Weights of keys (sw_decode_attn_weights_run) and eviction by them (sw_kv_evict) against the plain 64-bit forms."""
import math

import numpy as np
import pytest
import torch

from paper_2609_07883_b200 import binding as B
from tests import op_util as U

pytestmark = pytest.mark.gpu

HEADS = [(8, 2, 64), (32, 8, 128), (8, 1, 128), (4, 4, 64), (16, 8, 128), (8, 1, 64)]


def weights_of(c, rows, capacity, seed=1):
    gen = torch.Generator(device=c.dev)
    gen.manual_seed(seed)
    return torch.rand(rows, c.shape.num_kv_heads, capacity, device=c.dev, generator=gen)


def weigh(c, kw):
    scratch = torch.full((B.sw_attn_weights_scratch_bytes(c.ctx.layout, len(c.batch.decode_pages)),), 0xFF, dtype=torch.uint8, device=c.dev)
    B.sw_decode_attn_weights_run(c.ctx, c.pool, c.db, c.q, c.out, c.lse, kw, scratch)


def check_weights(c, before, after, rows, got):
    want, tol = before.double().clone(), torch.zeros_like(before, dtype=torch.float64)
    for (i, h), (w, seen, rel) in got.items():
        n = len(w)
        old = want[rows[i], h, :n].clone()
        old[n - 1] = 0
        want[rows[i], h, :n] = old + w
        tol[rows[i], h, :n] = rel * w + 2.0 ** -23 * (old + w)     # exponents' errors; two additions and roundings of fp32
    err = (after.double() - want).abs()
    assert bool((err <= tol).all()), f"weights off by {float((err / tol.clamp(min=1e-30)).max()):.3g} of their tolerance"


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("lens", [[1], [5000], [1, 2, 15, 16, 17, 31, 100, 257, 1000, 2049], [0, 700, 0, 64]])
def test_weights(heads, lens):
    c = U.Case(heads, lens, seed=len(lens))
    rows = np.random.default_rng(0).permutation(len(lens) + 3)[:len(lens)]
    w = weights_of(c, len(lens) + 3, max(lens) + 5)
    before = w.clone()
    weigh(c, B.KeyWeights(w, torch.from_numpy(rows.astype(np.int32)).to(c.dev)))
    c.ok()
    check_weights(c, before, w, rows, c.check(c.pool.double()))


@pytest.mark.parametrize("heads,n", [((8, 2, 64), 500), ((8, 1, 128), 40)])   # units
def test_weights_of_units(heads, n):
    rng = np.random.default_rng(n)
    c = U.Case(heads, rng.integers(0, 3000 if n < 100 else 200, n), seed=n)
    w = weights_of(c, n, 3000)
    before = w.clone()
    weigh(c, B.KeyWeights(w, torch.arange(n, dtype=torch.int32, device=c.dev)))
    c.ok()
    check_weights(c, before, w, list(range(n)), c.check(c.pool.double()))


def test_masked_slots_hold_anything():
    c = U.Case((8, 2, 64), [5, 40], seed=3)
    clean = c.pool.double()
    for i, n in enumerate((5, 40)):
        c.pool[int(c.batch.decode_pages[c.batch.decode_page_indptr[i + 1] - 1]), :, :, n % U.PAGE:] = math.nan
    w = weights_of(c, 2, 64)
    before = w.clone()
    weigh(c, B.KeyWeights(w, torch.arange(2, dtype=torch.int32, device=c.dev)))
    c.ok()
    check_weights(c, before, w, [0, 1], c.check(clean))


def test_expired_wait_leaves_the_weights_alone():
    import ctypes

    c = U.Case((32, 8, 128), [3000] * 40, seed=3)     # (enough that some page is still on its way)
    w = weights_of(c, 40, 3000)
    before = w.clone()
    B._lib.sw_ctx_set_line_wait(c.ctx.handle, ctypes.c_int64(0))     # what has not arrived at the first look has expired
    weigh(c, B.KeyWeights(w, torch.arange(40, dtype=torch.int32, device=c.dev)))
    assert B.sw_check_status(c.ctx, raise_on_error=False)[0] == B.SW_ERR_DEVICE_TIMEOUT
    assert torch.equal(w, before)


def test_what_does_not_fit_is_reported():
    c = U.Case((8, 2, 64), [40, 100, 30], seed=4)
    w = weights_of(c, 3, 60)
    before = w.clone()
    kw = B.KeyWeights(w, torch.tensor([0, 1, 7], dtype=torch.int32, device=c.dev))     # 1 is too long, 2 has no row
    weigh(c, kw)
    assert B.sw_check_status(c.ctx, raise_on_error=False)[0] == B.SW_ERR_OUT_OF_RANGE
    got = c.check(c.pool.double())
    check_weights(c, before, w, [0, 1, 2], {k: v for k, v in got.items() if k[0] == 0})
    # a scratch of four pages: the first request and one page of the second
    w = weights_of(c, 3, 200)
    before = w.clone()
    scratch = torch.empty(B.sw_attn_weights_scratch_bytes(c.ctx.layout, 4), dtype=torch.uint8, device=c.dev)
    B.sw_decode_attn_weights_run(c.ctx, c.pool, c.db, c.q, c.out, c.lse, B.KeyWeights(w, torch.arange(3, dtype=torch.int32, device=c.dev)), scratch)
    assert B.sw_check_status(c.ctx, raise_on_error=False)[0] == B.SW_ERR_WORKSPACE
    c.check(c.pool.double())
    assert torch.equal(w[2], before[2]) and torch.equal(w[1, :, 16:], before[1, :, 16:])
    assert not torch.equal(w[0], before[0]) and not torch.equal(w[1, :, :16], before[1, :, :16])


def evict(c, w, rows, new_rows, budget, sinks, recent, seed=5):
    """The call into free pages; returns what the plain form gives and what the call gave."""
    b, H, n = c.batch, c.shape.num_kv_heads, c.batch.num_decode
    lens = b.decode_kv_len.tolist()
    per = [-(-min(x, budget) // U.PAGE) for x in lens]
    free = c.free_pages()
    assert sum(per) <= len(free)
    new_indptr = np.concatenate([[0], np.cumsum(per)]).astype(np.int32)
    new_pages = np.random.default_rng(seed).permutation(free)[:sum(per)].astype(np.int32)
    kept = torch.full((n, H, budget), -7, dtype=torch.int32, device=c.dev)
    new_len = torch.full((n,), -7, dtype=torch.int32, device=c.dev)
    pool, weights, want_kept = c.pool.clone(), w.clone(), kept.clone()
    for i, x in enumerate(lens):
        m = min(x, budget)
        for h in range(H):
            v = w[rows[i], h, :x].double().cpu()
            order = sorted(range(x), key=lambda t: (0 if (t < sinks or t >= x - recent or x <= budget) else 1,
                                                    -(-math.inf if math.isnan(float(v[t])) else float(v[t])) if not math.isnan(float(v[t])) else math.inf,
                                                    1 if math.isnan(float(v[t])) else 0, t))
            for j, t in enumerate(sorted(order[:m])):
                to, at = int(new_pages[new_indptr[i] + j // U.PAGE]), int(b.decode_pages[b.decode_page_indptr[i] + t // U.PAGE])
                pool[to, :, h, j % U.PAGE] = c.pool[at, :, h, t % U.PAGE]
                weights[new_rows[i], h, j] = w[rows[i], h, t]
                want_kept[i, h, j] = t
    to_dev = lambda a: torch.from_numpy(np.asarray(a, dtype=np.int32)).to(c.dev)  # noqa: E731
    B.sw_kv_evict(c.ctx, c.pool, c.db, B.KeyWeights(w, to_dev(rows)), to_dev(new_indptr), to_dev(new_pages), B.KeyWeights(w, to_dev(new_rows)),
                  budget, sinks, recent, kept, new_len)
    torch.cuda.synchronize()
    return pool, weights, want_kept, kept, new_len


def check_evict(c, w, budget, sinks, recent):
    n = c.batch.num_decode
    rows, new_rows = np.arange(n)[::-1].copy(), n + np.arange(n)
    pool, weights, want_kept, kept, new_len = evict(c, w, rows, new_rows, budget, sinks, recent)
    c.ok()
    assert new_len.tolist() == [min(int(x), budget) for x in c.batch.decode_kv_len]
    assert torch.equal(kept, want_kept)
    assert torch.equal(c.pool.view(torch.int16), pool.view(torch.int16))
    assert torch.equal(w.view(torch.int32), weights.view(torch.int32))


@pytest.mark.parametrize("heads", [(8, 2, 64), (32, 8, 128), (8, 1, 128), (4, 4, 64)])
@pytest.mark.parametrize("budget,sinks,recent", [(1, 0, 0), (1, 1, 0), (1, 0, 1), (16, 4, 4), (33, 0, 33), (100, 3, 17), (257, 200, 57), (4000, 4, 10)])
def test_evict(heads, budget, sinks, recent):
    c = U.Case(heads, [1, 15, 16, 40, 100, 258, 1000], seed=budget, spare=200)
    check_evict(c, weights_of(c, 14, 4000), budget, sinks, recent)


def test_evict_ties_and_special_weights():
    """Equal weights: the lowest positions; NaN after everything, infinities at the ends, -0 like 0, subnormal and negative weights in order."""
    c = U.Case((8, 2, 64), [500, 500, 500, 500, 500], seed=1, spare=200)
    w = weights_of(c, 10, 512)
    w[0] = 0
    w[1] = torch.round(w[1] * 4) / 4
    w[2, :, ::3] = math.nan
    w[2, :, ::7] = math.inf
    w[2, :, ::11] = -math.inf
    w[3] = torch.where(w[3] < 0.5, -0.0, 0.0)
    w[4] = (w[4] - 0.5) * 1e-38
    check_evict(c, w, 101, 2, 5)
    c2 = U.Case((8, 2, 64), [500], seed=2, spare=200)
    w2 = torch.full((2, 2, 512), math.nan, device=c2.dev)
    check_evict(c2, w2, 101, 2, 5)


# keys beyond those held in shared memory; every cluster size; CTAs of both sizes
@pytest.mark.parametrize("lens,budget", [([60000], 1000), ([120000, 3000], 40000), ([20000] * 60, 64), ([150000], 900), ([9000] * 60, 64), ([1900, 40] * 30, 64)])
def test_evict_long(lens, budget):
    c = U.Case((4, 1, 64) if len(lens) < 3 else (8, 8, 64), lens, seed=3, spare=sum(-(-min(n, budget) // U.PAGE) for n in lens) + 8)
    w = weights_of(c, 2 * len(lens), max(lens))
    w[::2] = torch.round(w[::2] * 1000) / 1000     # ties across CTAs
    b = c.batch
    n, H = b.num_decode, c.shape.num_kv_heads
    per = [-(-min(x, budget) // U.PAGE) for x in lens]
    new_indptr = np.concatenate([[0], np.cumsum(per)]).astype(np.int32)
    new_pages = np.array(c.free_pages()[:sum(per)], dtype=np.int32)
    to_dev = lambda a: torch.from_numpy(np.asarray(a, dtype=np.int32)).to(c.dev)  # noqa: E731
    kept, new_len = torch.zeros(n, H, budget, dtype=torch.int32, device=c.dev), torch.zeros(n, dtype=torch.int32, device=c.dev)
    rows, new_rows = np.arange(n), n + np.arange(n)
    B.sw_kv_evict(c.ctx, c.pool, c.db, B.KeyWeights(w, to_dev(rows)), to_dev(new_indptr), to_dev(new_pages), B.KeyWeights(w, to_dev(new_rows)),
                  budget, 4, 7, kept, new_len)
    c.ok()
    for i, x in enumerate(lens):
        m = min(x, budget)
        for h in range(H):
            v = w[i, h, :x].double().clone()
            if x > budget:
                v[:4] = math.inf
                v[x - 7:] = math.inf
            keep = torch.sort(torch.argsort(v, descending=True, stable=True)[:m]).values if x > budget else torch.arange(x, device=c.dev)
            assert torch.equal(kept[i, h, :m].long(), keep)
            assert torch.equal(w[n + i, h, :m], w[i, h, keep])
            src = to_dev(b.decode_pages[b.decode_page_indptr[i]:b.decode_page_indptr[i + 1]]).long()[keep // U.PAGE]
            j = torch.arange(m, device=c.dev)
            to = to_dev(new_pages[new_indptr[i]:new_indptr[i + 1]]).long()[j // U.PAGE]
            assert torch.equal(c.pool[to, :, h, j % U.PAGE].view(torch.int16), c.pool[src, :, h, keep % U.PAGE].view(torch.int16))


@pytest.mark.parametrize("n,capacity", [(1, 300), (1, 9000), (60, 300), (60, 9000)])   # CTAs of both sizes, alone and in clusters
@pytest.mark.parametrize("budget", [17, 101])
def test_evict_special_weights_in_every_form(n, capacity, budget):
    """Thresholds among NaN, infinities, zeros of both signs, numbers one step apart and numbers that share their first 16 bits."""
    c = U.Case((8, 8, 64), [300] * n, seed=n, spare=n * 7 + 8)
    gen = torch.Generator(device=c.dev)
    gen.manual_seed(budget)
    near = torch.randint(0, 9, (2 * n, 8, capacity), device=c.dev, generator=gen, dtype=torch.int32)
    w = (near + 0x3F800000).view(torch.float32).clone()
    w[::5] = torch.tensor([math.nan, math.inf, -math.inf, 0.0, -0.0, 1e-45, -1e-45, 3.0, -3.0], device=c.dev)[near[::5].long()]
    w[1::5] = -w[1::5]
    w[2::5] = math.nan
    w[2::5, :, 40:70] = -math.inf
    check_evict(c, w, budget, 1, 3)


def test_evict_what_does_not_fit_is_reported():
    c = U.Case((8, 2, 64), [100, 100, 100, 100], seed=6, spare=100)
    w = weights_of(c, 8, 100)
    before, pool = w.clone(), c.pool.clone()
    free = c.free_pages()
    to_dev = lambda a: torch.from_numpy(np.asarray(a, dtype=np.int32)).to(c.dev)  # noqa: E731
    kept, new_len = torch.full((4, 2, 40), -7, dtype=torch.int32, device=c.dev), torch.full((4,), -7, dtype=torch.int32, device=c.dev)
    new_pages = free[:12]
    new_pages[11] = c.pages          # request 3: a page outside the pool
    # request 0: too few new pages; 1: no such row; 2: onto itself
    B.sw_kv_evict(c.ctx, c.pool, c.db, B.KeyWeights(w, to_dev([0, 1, 2, 3])), to_dev([0, 2, 5, 8, 11 + 1]), to_dev(new_pages),
                  B.KeyWeights(w, to_dev([4, 9, 2, 7])), 40, 2, 2, kept, new_len)
    assert B.sw_check_status(c.ctx, raise_on_error=False)[0] == B.SW_ERR_OUT_OF_RANGE
    assert new_len.tolist()[:3] == [0, 0, 0] and bool((kept[:3] == -7).all())
    assert torch.equal(w[:7], before[:7])
    torch.cuda.synchronize()
    assert torch.equal(c.pool[c.batch.decode_pages], pool[c.batch.decode_pages])


def test_weigh_evict_and_go_on():
    """A few decode steps that weigh, an eviction, then decode steps over what is left, with the weights that moved along."""
    c = U.Case((16, 4, 64), [90, 130, 40], seed=8, spare=60)
    w = torch.zeros(6, 4, 160, device=c.dev)
    rows = torch.tensor([4, 0, 2], dtype=torch.int32, device=c.dev)
    for step in range(2):
        c.q.copy_(torch.randn(c.q.shape, generator=torch.Generator().manual_seed(step)))
        before = w.clone()
        weigh(c, B.KeyWeights(w, rows))
        c.ok()
        check_weights(c, before, w, rows.tolist(), c.check(c.pool.double()))
    pool, weights, want_kept, kept, new_len = evict(c, w, [4, 0, 2], [1, 3, 5], 48, 2, 8)
    c.ok()
    assert torch.equal(kept, want_kept) and torch.equal(w, weights) and torch.equal(c.pool, pool)
    # the kept rows, one more each, in the new pages
    b = c.batch
    per = [3, 3, 3]
    fresh = [p for p in c.free_pages()]
    new_pages = np.random.default_rng(5).permutation(fresh)[:9].astype(np.int32)
    more = [p for p in fresh if p not in set(new_pages.tolist())][:3]
    b.decode_pages = np.concatenate([np.append(new_pages[3 * i:3 * i + 3], more[i]) for i in range(3)]).astype(np.int32)
    b.decode_page_indptr = np.array([0, 4, 8, 12], dtype=np.int32)
    b.decode_kv_len = np.array([49, 49, 41], dtype=np.int32)
    c.renew()
    B.sw_kv_append(c.ctx, c.pool, c.db, c.k_new, c.v_new)
    before = w.clone()
    weigh(c, B.KeyWeights(w, torch.tensor([1, 3, 5], dtype=torch.int32, device=c.dev)))
    c.ok()
    check_weights(c, before, w, [1, 3, 5], c.check(c.pool.double()))
    assert per == [3, 3, 3]


def test_captured_and_replayed_on_another_stream():
    c = U.Case((32, 8, 128), [300, 5000, 40], seed=6, spare=80)
    w = torch.zeros(6, 8, 5008, device=c.dev)
    to_dev = lambda a: torch.from_numpy(np.asarray(a, dtype=np.int32)).to(c.dev)  # noqa: E731
    old, new = B.KeyWeights(w, to_dev([0, 1, 2])), B.KeyWeights(w, to_dev([3, 4, 5]))
    scratch = torch.empty(B.sw_attn_weights_scratch_bytes(c.ctx.layout, len(c.batch.decode_pages)), dtype=torch.uint8, device=c.dev)
    new_indptr, new_pages = to_dev([0, 8, 16, 19]), to_dev(c.free_pages()[:19])
    kept, new_len = torch.zeros(3, 8, 128, dtype=torch.int32, device=c.dev), torch.zeros(3, dtype=torch.int32, device=c.dev)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        B.sw_decode_attn_weights_run(c.ctx, c.pool, c.db, c.q, c.out, c.lse, old, scratch, stream=s)
        B.sw_kv_evict(c.ctx, c.pool, c.db, old, new_indptr, new_pages, new, 128, 4, 16, kept, new_len, stream=s)
    for seed in (1, 2):
        c.q.copy_(torch.randn(c.q.shape, generator=torch.Generator().manual_seed(seed)))
        before = w.clone()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        c.ok()
        got = c.check(c.pool.double())
        check_weights(c, before[:3], w[:3], [0, 1, 2], got)
        keep = w[1, 3, 4:5000 - 16].argsort(descending=True, stable=True)[:108].sort().values + 4
        assert torch.equal(kept[1, 3, 4:112].long(), keep) and new_len.tolist() == [128, 128, 40]


def test_refusals():
    c = U.Case((8, 2, 64), [40], [(0, 20)])
    w = weights_of(c, 2, 64)
    kw, new = B.KeyWeights(w, torch.zeros(1, dtype=torch.int32, device=c.dev)), B.KeyWeights(w, torch.ones(1, dtype=torch.int32, device=c.dev))
    scratch = torch.empty(1 << 20, dtype=torch.uint8, device=c.dev)
    ints = torch.zeros(256, dtype=torch.int32, device=c.dev)
    with pytest.raises(B.SwError) as e:      # a chunk
        B.sw_decode_attn_weights_run(c.ctx, c.pool, c.db, c.q, c.out, c.lse, kw, scratch)
    assert e.value.status == B.SW_ERR_UNSUPPORTED
    with pytest.raises(B.SwError) as e:
        B.sw_kv_evict(c.ctx, c.pool, c.db, kw, ints, ints, new, 16, 0, 0, ints, ints)
    assert e.value.status == B.SW_ERR_UNSUPPORTED
    d = U.Case((8, 2, 64), [40])
    for lse, s in [(None, scratch), (d.lse, None), (d.lse.view(-1)[1:], scratch)]:
        with pytest.raises(B.SwError) as e:
            B.sw_decode_attn_weights_run(d.ctx, d.pool, d.db, d.q, d.out, lse, kw, s)
        assert e.value.status == B.SW_ERR_INVALID_ARG
    with pytest.raises(B.SwError) as e:
        B.sw_decode_attn_weights_run(d.ctx, d.pool, d.db, d.q, d.out, d.lse, kw, scratch[16:])
    assert e.value.status == B.SW_ERR_WORKSPACE
    for budget, sinks, recent in [(0, 0, 0), (65, 0, 0), (16, 10, 7), (16, -1, 0), (16, 0, -1)]:
        with pytest.raises(B.SwError) as e:
            B.sw_kv_evict(d.ctx, d.pool, d.db, kw, ints, ints, new, budget, sinks, recent, ints, ints)
        assert e.value.status == B.SW_ERR_INVALID_ARG
    for bad in (w.double(), w[:, :, ::2], w[0]):
        with pytest.raises(ValueError):
            B.KeyWeights(bad, torch.zeros(1, dtype=torch.int32, device=c.dev))
    one_head, no_rows = weights_of(c, 2, 64)[:, :1].contiguous(), torch.zeros(0, dtype=torch.int32, device=c.dev)
    for old, fresh, kept in [(kw, B.KeyWeights(w.clone(), new.row_of), ints), (B.KeyWeights(w, no_rows), new, ints), (kw, B.KeyWeights(w, no_rows), ints),
                             (B.KeyWeights(one_head, kw.row_of), B.KeyWeights(one_head, new.row_of), ints), (kw, new, ints[:31])]:
        with pytest.raises(ValueError):
            B.sw_kv_evict(d.ctx, d.pool, d.db, old, ints, ints, fresh, 16, 0, 0, kept, ints)
    with pytest.raises(ValueError):
        B.sw_decode_attn_weights_run(d.ctx, d.pool, d.db, d.q, d.out, d.lse, B.KeyWeights(one_head, kw.row_of), scratch)
