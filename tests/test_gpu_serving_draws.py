"""The serving loop's executor with rotary positions in its layers and the draw of the next tokens at its end."""
import numpy as np
import pytest
import torch

from paper_2609_07883_b200 import binding as B
from paper_2609_07883_b200 import serving
from paper_2609_07883_b200 import workloads as W

pytestmark = pytest.mark.gpu
SHAPE, PAGES = W.AttnShape(8, 2, 64), 512


def setup_layers(layers):
    ctx = B.Context(SHAPE, PAGES, 256, 16, PAGES)
    pools = [torch.zeros(PAGES * SHAPE.page_elems, dtype=torch.bfloat16, device="cuda") for _ in range(layers)]
    return ctx, pools


def test_iteration_with_positions_and_draws():
    ctx, pools = setup_layers(2)
    turns, magnitude = B.sw_rope_frequencies(64, 10000.0, "linear", 2.0)
    execute = serving.gpu_executor(ctx, pools, SHAPE, 256, 16, seed=5, rope=B.Rope(turns, False, magnitude), vocab=3001, top_k=20)
    assert execute.extra_ns > 0 and execute.tokens is None
    rng = np.random.default_rng(2)
    batch = W.make_multi_batch(SHAPE, PAGES, [5, 40, 17], [(0, 33), (16, 20)], rng)
    for pool in pools:
        pool.zero_()
    assert execute(batch) > 0
    assert execute.tokens.shape == (5,) and bool((execute.tokens >= 0).all()) and bool((execute.tokens < 3001).all())
    # the same rows, rotated, in the pool of every layer: the executor's keys come from its seed
    gen = torch.Generator(device="cuda")
    gen.manual_seed(5)
    q = torch.randn(272, 8, 64, device="cuda", generator=gen).to(torch.bfloat16)
    k = torch.randn(272, 2, 64, device="cuda", generator=gen).to(torch.bfloat16)
    v = torch.randn(272, 2, 64, device="cuda", generator=gen).to(torch.bfloat16)
    rows, db = batch.num_rows, B.DeviceBatch(batch, torch.device("cuda", 0))
    want, turned = torch.zeros_like(pools[0]), torch.empty_like(q)
    B.sw_rope_append(ctx, want, db, B.Rope(turns, False, magnitude), q[:rows], k[:rows], v[:rows], turned[:rows])
    torch.cuda.synchronize()
    assert bool((want != 0).any())
    for pool in pools:
        assert torch.equal(pool, want)
    first = execute.tokens.clone()
    execute(batch)
    assert not torch.equal(first, execute.tokens)       # (20 candidates a row, five rows, other numbers: alike once in 20^5 at most)
    assert B.sw_check_status(ctx, raise_on_error=False) == (0, 0)


def test_trace_with_draws():
    ctx, pools = setup_layers(1)
    execute = serving.gpu_executor(ctx, pools, SHAPE, 256, 16, vocab=1000, temperature=0.0)
    table = B.CostTable([1, 16], [1 << 20], [0, 1 << 16], [0, 256], np.full((2, 1, 2, 2), 100_000), make_monotone=True)
    trace = {"arrival_ns": np.arange(6) * 1000, "prompt_len": np.array([30, 1, 100, 17, 250, 64]), "output_len": np.array([3, 5, 1, 8, 2, 4])}
    res = serving.run_trace(trace, 50.0, table, execute, SHAPE, PAGES, c_max=256, max_decode=16, ctx_cap=1 << 20, margin_abs_ns=execute.extra_ns)
    assert res["requests"] == 6 and execute.tokens is not None
    assert B.sw_check_status(ctx, raise_on_error=False) == (0, 0)


def test_without_them_nothing_is_added():
    ctx, pools = setup_layers(1)
    execute = serving.gpu_executor(ctx, pools, SHAPE, 256, 16)
    assert execute.extra_ns == 0 and execute(W.make_batch(SHAPE, PAGES, [5], 0, 10, np.random.default_rng(1))) > 0 and execute.tokens is None
