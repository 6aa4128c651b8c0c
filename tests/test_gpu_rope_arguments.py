"""Rotary positions: arguments that only the library itself looks at."""
import ctypes as C

import pytest
import torch

from paper_2609_07883_b200 import binding as B
from tests import op_util as U

pytestmark = pytest.mark.gpu


def setup_case():
    c = U.Case((8, 2, 64), [1, 17, 40], [(5, 20)], seed=3)
    turns, magnitude = B.sw_rope_frequencies(64)
    return c, B.Rope(turns, magnitude=magnitude, device=c.dev)


def stream():
    return torch.cuda.current_stream().cuda_stream


@pytest.mark.parametrize("v_stride", [1, -8, 3, (1 << 31) + 8, 1 << 40, -(1 << 63), (1 << 63) - 1])
def test_run_ignores_the_stride_of_values(v_stride):
    """It takes no values."""
    c, rope = setup_case()
    want, got = (tuple(torch.zeros_like(x) for x in (c.q, c.k_new)) for _ in range(2))
    B.sw_rope_run(c.ctx, c.db, rope, c.q, c.k_new, *want)
    fields = {name: getattr(rope.struct(c.batch.num_rows, (512, 128, 0)), name) for name, _ in B.sw_rope._fields_}
    s = B.sw_rope(**{**fields, "v_stride": v_stride})
    tensors = [x.data_ptr() for x in (c.q, c.k_new, *got)]
    assert B._lib.sw_rope_run(c.ctx.handle, C.byref(c.db.struct), C.byref(s), *tensors, stream()) == B.SW_OK, B.sw_last_error()
    c.ok()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_append_takes_the_stride_of_values():
    c, rope = setup_case()
    for v_stride in (1, -8, 3, 120, (1 << 31) + 8):
        s = B.sw_rope(**{**{name: getattr(rope.struct(c.batch.num_rows, (512, 128, 128)), name) for name, _ in B.sw_rope._fields_}, "v_stride": v_stride})
        tensors = [x.data_ptr() for x in (c.q, c.k_new, c.v_new, c.out)]
        assert B._lib.sw_rope_append(c.ctx.handle, c.pool.data_ptr(), C.byref(c.db.struct), C.byref(s), *tensors, stream()) == B.SW_ERR_INVALID_ARG
    c.ok()


def test_append_refuses_queries_over_the_pool():
    """Other rows' keys go there in the same launch."""
    c, rope = setup_case()
    n, size = c.out.numel(), c.pool.numel()
    one = torch.zeros(n + size + n, dtype=torch.bfloat16, device=c.dev)
    pool = one[n:n + size].view(c.pool.shape)
    pool.copy_(c.pool)
    at = lambda first: one[first:first + n].view(c.out.shape)  # noqa: E731
    for first in (n, n + 64, 8, n + size // 2 // 8 * 8, size, n + size - 8):
        with pytest.raises(B.SwError, match="overlaps the pool") as e:
            B.sw_rope_append(c.ctx, pool, c.db, rope, c.q, c.k_new, c.v_new, at(first))
        assert e.value.status == B.SW_ERR_INVALID_ARG
    torch.cuda.synchronize()
    assert torch.equal(pool.nan_to_num(), c.pool.nan_to_num())
    B.sw_rope_append(c.ctx, c.pool, c.db, rope, c.q, c.k_new, c.v_new, c.out)
    for first in (0, n + size):                       # its neighbours on both sides
        B.sw_rope_append(c.ctx, pool, c.db, rope, c.q, c.k_new, c.v_new, at(first))
        c.ok()
        assert torch.equal(at(first), c.out) and torch.equal(pool.nan_to_num(), c.pool.nan_to_num())
