"""The KV pool in 8 bits (sw_kv8_append, sw_kv8_attn_run) against the plain 64-bit form."""
import math

import numpy as np
import pytest
import torch

from paper_2609_07883_b200 import binding as B
from tests import op_util as U

pytestmark = pytest.mark.gpu

HEADS = [(8, 2, 64), (32, 8, 128), (8, 1, 128), (4, 4, 64), (16, 8, 128), (8, 1, 64)]


def same_bits(a, b):
    return torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def pool8(c):
    codes, scales = U.quantise(c.pool)
    return codes, scales


def attend(c, codes, scales, scratch=True):
    """With a scratch long chunks read a 16-bit copy of their prompts, without one the pool."""
    pages = sum(-(-(P + C) // U.PAGE) for P, C, _, _ in c.batch.chunks())
    room = torch.full((B.sw_kv8_scratch_bytes(c.ctx.layout, pages),), 0xFF, dtype=torch.uint8, device=c.dev) if scratch and pages else None
    B.sw_kv8_attn_run(c.ctx, codes, scales, c.db, c.q, c.out, c.lse, room)


def check8(c, want, **kw):
    c.check(want, floor=2.0 ** -32, **kw)


def check_append(c, codes, scales):
    want, want_scales = codes.view(torch.uint8).cpu().clone(), scales.cpu().clone()
    U.append8(want, want_scales, U.entries_of(c.batch), c.k_new.cpu(), c.v_new.cpu())
    B.sw_kv8_append(c.ctx, codes, scales, c.db, c.k_new, c.v_new)
    c.ok()
    torch.cuda.synchronize()
    got_scales = scales.cpu()
    assert torch.equal(torch.isnan(got_scales), torch.isnan(want_scales))
    assert torch.equal(torch.nan_to_num(got_scales), torch.nan_to_num(want_scales))
    assert torch.equal(codes.view(torch.uint8).cpu(), want)


@pytest.mark.parametrize("heads", HEADS)
def test_append_rows(heads):
    c = U.Case(heads, [1, 16, 17, 33, 47, 48], [(5, 60)], seed=2)
    c.k_new *= torch.exp(3 * torch.randn(c.k_new.shape[:2], device=c.dev))[..., None]     # scales that grow, and that do not
    check_append(c, *pool8(c))


@pytest.mark.parametrize("chunks", [[(0, 1)], [(15, 1)], [(15, 2)], [(0, 16)], [(7, 9)], [(3, 300)], [(40, 20), (16, 33), (0, 1)]])
def test_append_chunks(chunks):
    c = U.Case((8, 2, 64), [], chunks, seed=3)
    codes, scales = pool8(c)
    scales.mul_(2.0 ** -6)
    check_append(c, codes, scales)


def test_append_values_at_the_edges():
    """Halves between two codes, subnormal codes, zeros, the largest and smallest bf16, rows of one value; a scale of 2^-100 at least."""
    c = U.Case((8, 8, 64), [1, 2, 3, 18, 35, 100, 1, 1], seed=4)
    half = torch.arange(64, device=c.dev).float()
    rows = [448 - 8 * half, (half - 32) / 1024 + 448 * (half == 0), torch.zeros(64, device=c.dev), half * 0 + 3.3e38, half * 1e-38, half * 2.0 ** -100,
            torch.where(half == 9, 449.0, half), -half * 1e5]
    for i, r in enumerate(rows):
        c.k_new[i] = r.to(torch.bfloat16)
        c.v_new[i] = (-r).to(torch.bfloat16)
    check_append(c, *pool8(c))


def test_append_into_an_uninitialised_pool():
    c = U.Case((8, 2, 64), [1, 17], [(0, 20)], seed=5)
    codes = torch.randint(0, 256, c.pool.shape, device=c.dev, dtype=torch.uint8)
    scales = torch.full(c.pool.shape[:3], math.nan, device=c.dev)
    check_append(c, codes, scales)


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_append_non_finite(bad):
    c = U.Case((8, 2, 64), [5, 20], [(0, 40)], seed=6)
    c.k_new[20, 1, 7] = bad      # chunk, second page
    c.v_new[40, 0, 3] = bad      # request 0, behind other rows
    codes, scales = pool8(c)
    check_append(c, codes, scales)
    assert int(torch.isnan(scales).sum()) == 2
    c.k_new.fill_(1)
    c.v_new.fill_(1)
    check_append(c, codes, scales)     # rows behind others do not mend the block, a row at the first slot does


def test_append_in_steps_equals_append_at_once_up_to_subnormals():
    c = U.Case((8, 2, 64), [], [(0, 64)], seed=7)
    codes, scales = pool8(c)
    B.sw_kv8_append(c.ctx, codes, scales, c.db, c.k_new, c.v_new)
    whole = U.dequantise(codes, scales)[c.batch.prefill_pages[:4]]
    pages = c.batch.prefill_pages
    for t in range(64):
        one = U.Case((8, 2, 64), [t + 1], seed=7, spare=c.pages)
        one.batch.decode_pages[:] = pages[:len(one.batch.decode_pages)]
        one.renew()
        B.sw_kv8_append(one.ctx, codes, scales, one.db, c.k_new[t:t + 1].contiguous(), c.v_new[t:t + 1].contiguous())
        one.ok()
    steps = U.dequantise(codes, scales)[pages[:4]]
    unit = scales[torch.from_numpy(pages[:4]).long().to(c.dev)].double()[..., None, None] * 2.0 ** -9
    # a code that became subnormal was rounded once more at half a subnormal step per growth of the scale
    assert bool(((steps - whole).abs() <= 16 * unit).all()) and bool(((steps != whole) <= (whole.abs() < 16 * unit)).all())


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("lens", [[1], [8192], [1, 2, 15, 16, 17, 31, 100, 257, 1000, 2049], [4000] * 20])
def test_decode(heads, lens):
    c = U.Case(heads, lens, seed=len(lens))
    c.pool[:, 0] *= 3.0
    codes, scales = pool8(c)
    want = U.dequantise(codes, scales)
    raw = codes.view(torch.uint8)
    for i, n in enumerate(lens):     # slots past the context hold anything
        if n % U.PAGE:
            raw[int(c.batch.decode_pages[c.batch.decode_page_indptr[i + 1] - 1]), :, :, n % U.PAGE:] = 0x7F
    attend(c, codes, scales)
    c.ok()
    check8(c, want)


@pytest.mark.parametrize("heads,n", [((8, 2, 64), 500), ((8, 1, 128), 40), ((8, 1, 64), 450)])   # units
def test_decode_units(heads, n):
    rng = np.random.default_rng(n)
    c = U.Case(heads, rng.integers(0, 3000 if n < 100 else 200, n), seed=n)
    codes, scales = pool8(c)
    attend(c, codes, scales)
    c.ok()
    check8(c, U.dequantise(codes, scales))


@pytest.mark.parametrize("heads", [(8, 2, 64), (32, 8, 128), (8, 1, 128), (4, 4, 64)])
@pytest.mark.parametrize("chunks", [[(0, 1)], [(0, 300)], [(1000, 77)], [(3000, 40), (130, 300), (0, 17)], [(700, 1500)], [(2000, 900), (2000, 900)]])
@pytest.mark.parametrize("lens,scratch", [([], True), ([100, 1, 700, 3000], True), ([], False), ([100, 1, 700, 3000], False)])
def test_chunks(heads, chunks, lens, scratch):
    c = U.Case(heads, lens, chunks, seed=len(chunks))
    codes, scales = pool8(c)
    want = U.dequantise(codes, scales)
    raw = codes.view(torch.uint8)
    for P, C, _, pages in c.batch.chunks():
        if (P + C) % U.PAGE:
            raw[int(pages[-1]), :, :, (P + C) % U.PAGE:] = 0x7F
    attend(c, codes, scales, scratch)
    c.ok()
    check8(c, want)


@pytest.mark.parametrize("far", [2.0 ** -13, 2.0 ** -30, 2.0 ** -90, 2.0 ** 5, 2.0 ** 40])
@pytest.mark.parametrize("chunks,lens,scratch", [([(600, 300)], [], False), ([(600, 300)], [], True), ([], [700, 45], False)])
def test_scales_that_change_inside_a_context(far, chunks, lens, scratch):
    """V's scales a long way apart from one stretch of a context to the next, and back; what lies far below the largest counts as little as it
    weighs.  (Within a stretch of 128 keys they differ by factors of up to 8, as those of neighbouring blocks do.)"""
    c = U.Case((8, 2, 64), lens, chunks, seed=14)
    codes, scales = pool8(c)
    for _, _, _, pages in U.entries_of(c.batch):
        for j, page in enumerate(pages):
            scales[int(page), 1] = 2.0 ** (j % 4 - 8) * (far if j // 8 % 2 else 1.0)
    attend(c, codes, scales, scratch)
    c.ok()
    check8(c, U.dequantise(codes, scales))


@pytest.mark.parametrize("exponent", [-100, -60, -20, 6, 7, 8, 20, 60])
def test_scales_far_from_one(exponent):
    """V at any scale (its outputs scale along), K at scales whose scores stay in range."""
    c = U.Case((8, 2, 64), [100, 40], [(30, 50)], seed=8)
    codes, scales = pool8(c)
    scales[:, 1] = 2.0 ** exponent
    if -20 <= exponent <= 20:
        scales[:, 0] = 2.0 ** exponent
        c.q = (c.q.float() * 2.0 ** -exponent / 100).to(torch.bfloat16)
    else:
        scales[:, 0] *= 0.25
    attend(c, codes, scales)
    c.ok()
    check8(c, U.dequantise(codes, scales))


def test_nan_scale_reaches_the_rows_that_read_it():
    c = U.Case((8, 2, 64), [100, 40], seed=9)
    codes, scales = pool8(c)
    want = U.dequantise(codes, scales)
    scales[int(c.batch.decode_pages[2]), 1, 0] = math.nan      # request 0, V of head 0
    attend(c, codes, scales)
    c.ok()
    torch.cuda.synchronize()
    assert bool(torch.isnan(c.out[0, :4]).all()) and not bool(torch.isnan(c.out[0, 4:]).any())
    check8(c, want, rows=[1])


def test_append_then_attend_many_iterations():
    """Three iterations as a server runs them: chunk and decode rows appended, then attended."""
    heads, lens, P = (16, 4, 64), np.array([30, 15, 200]), 20
    codes = scales = host = host_scales = None
    for step in range(3):
        c = U.Case(heads, lens + 3, [(P, 50)], seed=10, spare=200)
        c.batch.decode_kv_len[:] = lens + step
        c.batch.prefix_len = P + 50 * step if step == 0 else P
        c.renew()
        gen = torch.Generator(device=c.dev)
        gen.manual_seed(step)
        for t in (c.q, c.k_new, c.v_new):
            t.copy_(torch.randn(t.shape, device=c.dev, generator=gen) * (1 + 3 * step))
        if codes is None:
            codes, scales = pool8(c)
            host, host_scales = codes.view(torch.uint8).cpu().clone(), scales.cpu().clone()
        B.sw_kv8_append(c.ctx, codes, scales, c.db, c.k_new, c.v_new)
        attend(c, codes, scales)
        c.ok()
        U.append8(host, host_scales, U.entries_of(c.batch), c.k_new.cpu(), c.v_new.cpu())
        assert torch.equal(codes.view(torch.uint8).cpu(), host) and torch.equal(scales.cpu(), host_scales)
        check8(c, U.dequantise(codes, scales))


def test_captured_and_replayed_on_another_stream():
    c = U.Case((32, 8, 128), [300, 5000, 40], [(700, 100)], seed=6)
    codes, scales = pool8(c)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        B.sw_kv8_append(c.ctx, codes, scales, c.db, c.k_new, c.v_new, stream=s)
        B.sw_kv8_attn_run(c.ctx, codes, scales, c.db, c.q, c.out, c.lse, stream=s)
    for seed in (1, 2):
        for t in (c.q, c.k_new, c.v_new):
            t.copy_(torch.randn(t.shape, generator=torch.Generator().manual_seed(seed)))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        c.ok()
        check8(c, U.dequantise(codes, scales))


def test_bad_pages_are_reported_and_nothing_else_is_written():
    c = U.Case((8, 2, 64), [40, 20], [(0, 20)], seed=12)
    codes, scales = pool8(c)
    before, before_scales = codes.clone(), scales.clone()
    c.batch.decode_pages[2] = c.pages          # request 0's last page
    c.batch.prefill_pages[0] = -1
    c.renew()
    B.sw_kv8_append(c.ctx, codes, scales, c.db, c.k_new, c.v_new)
    assert B.sw_check_status(c.ctx, raise_on_error=False)[0] == B.SW_ERR_OUT_OF_RANGE
    touched = {int(c.batch.prefill_pages[1]), int(c.batch.decode_pages[4])}
    keep = [i for i in range(c.pages) if i not in touched]
    assert same_bits(codes[keep], before[keep]) and torch.equal(scales[keep], before_scales[keep])
    attend(c, codes, scales)
    assert B.sw_check_status(c.ctx, raise_on_error=False)[0] == B.SW_ERR_OUT_OF_RANGE
    torch.cuda.synchronize()


def test_refusals():
    c = U.Case((8, 2, 64), [40], [(0, 20)])
    codes, scales = pool8(c)
    for args in [(None, scales, c.q, c.out), (codes, None, c.q, c.out), (codes, scales, None, c.out), (codes, scales, c.q, None),
                 (codes.view(torch.uint8).view(-1)[1:], scales, c.q, c.out), (codes, scales.view(-1)[1:], c.q, c.out)]:
        with pytest.raises(B.SwError) as e:
            B.sw_kv8_attn_run(c.ctx, args[0], args[1], c.db, args[2], args[3])
        assert e.value.status == B.SW_ERR_INVALID_ARG
    for args in [(None, scales, c.k_new, c.v_new), (codes, None, c.k_new, c.v_new), (codes, scales, None, c.v_new), (codes, scales, c.k_new, None),
                 (codes.view(torch.uint8).view(-1)[1:], scales, c.k_new, c.v_new), (codes, scales.view(-1)[1:], c.k_new, c.v_new)]:
        with pytest.raises(B.SwError) as e:
            B.sw_kv8_append(c.ctx, args[0], args[1], c.db, args[2], args[3])
        assert e.value.status == B.SW_ERR_INVALID_ARG
