"""What the serving loop's executor adds to the controller's margin for rotary positions and draws: measured on the launches that it makes."""
import pytest
import torch

from paper_2609_07883_b200 import binding as B
from paper_2609_07883_b200 import serving
from paper_2609_07883_b200 import workloads as W

pytestmark = pytest.mark.gpu
SHAPE = W.AttnShape(8, 2, 64)
CALLS = ("sw_rope_append", "sw_rope_run", "sw_mixed_attn_run", "sw_mixed_iteration_run", "sw_sample_run")


def setup_layers(pages, layers=2):
    ctx = B.Context(SHAPE, pages, 256, 16, pages)
    return ctx, [torch.zeros(pages * SHAPE.page_elems, dtype=torch.bfloat16, device="cuda") for _ in range(layers)]


def rope():
    turns, magnitude = B.sw_rope_frequencies(64)
    return B.Rope(turns, False, magnitude)


@pytest.fixture
def counts(monkeypatch):
    """Calls of the binding by name, and the numbers of rows that the attention was given."""
    seen = {name: [] for name in CALLS}
    for name in CALLS:
        def counted(ctx, *args, _name=name, _call=getattr(B, name), **kw):
            seen[_name].append(next((a.rows for a in args if isinstance(a, B.DeviceBatch)), None))
            return _call(ctx, *args, **kw)
        monkeypatch.setattr(B, name, counted)
    return seen


def test_rotary_positions_are_measured_as_they_run(counts):
    """The append with the rotation and the attention, against the one launch that the cost table knows; at the largest batch, and at the smallest."""
    ctx, pools = setup_layers(512)
    execute = serving.gpu_executor(ctx, pools, SHAPE, 256, 16, rope=rope())
    assert execute.extra_ns >= 0 and execute.tokens is None
    assert not counts["sw_rope_run"] and not counts["sw_sample_run"]
    assert counts["sw_rope_append"] and counts["sw_rope_append"] == counts["sw_mixed_attn_run"]
    assert sorted(counts["sw_mixed_iteration_run"]) == sorted(counts["sw_rope_append"]) and set(counts["sw_rope_append"]) == {1, 272}
    assert len(counts["sw_rope_append"]) % len(pools) == 0
    assert B.sw_check_status(ctx, raise_on_error=False) == (0, 0)


def test_draws_alone_need_no_batch(counts):
    """A pool too small for the largest batch, which the executor never gets then."""
    ctx, pools = setup_layers(8, 1)
    execute = serving.gpu_executor(ctx, pools, SHAPE, 256, 16, vocab=1000)
    assert execute.extra_ns > 0 and execute.tokens is None and bool((pools[0] == 0).all())
    assert counts["sw_sample_run"] and not any(counts[name] for name in CALLS[:4])


@pytest.mark.parametrize("pages", [1, 8, 20])
def test_rotary_positions_in_a_small_pool(counts, pages):
    ctx, pools = setup_layers(pages, 1)
    execute = serving.gpu_executor(ctx, pools, SHAPE, 256, 16, rope=rope(), vocab=1000)
    assert execute.extra_ns > 0 and max(counts["sw_rope_append"]) == (pages if pages <= 16 else 16 + 16 * (pages - 16))
    assert B.sw_check_status(ctx, raise_on_error=False) == (0, 0)


def test_without_either_nothing_is_launched(counts):
    ctx, pools = setup_layers(64, 1)
    assert serving.gpu_executor(ctx, pools, SHAPE, 256, 16).extra_ns == 0 and not any(counts.values())
