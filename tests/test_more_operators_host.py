"""What rotary positions, cross attention and sampling refuse, and the frequencies of the rotation, without a GPU."""
import ctypes as C
import math
from types import SimpleNamespace

import numpy as np
import pytest
import torch

from paper_2609_07883_b200 import binding as B
from paper_2609_07883_b200 import workloads as W

# seven roundings of fp64 (power, quotient, blend), and a power whose exponent's rounding counts ln(base^(2i/d)) times: 2^-53 (7 + 14)
REL = 2.0 ** -48


def plain(rotary, base):
    return np.array([base ** (-2 * i / rotary) / (2 * math.pi) for i in range(rotary // 2)])


@pytest.mark.parametrize("rotary", [16, 32, 48, 64, 80, 128])
@pytest.mark.parametrize("base", [1.5, 10000.0, 500000.0, 1e6])
def test_plain_linear_and_base(rotary, base):
    turns, m = B.sw_rope_frequencies(rotary, base)
    assert m == 1.0 and np.allclose(turns, plain(rotary, base), rtol=REL, atol=0)
    turns, m = B.sw_rope_frequencies(rotary, base, "linear", 3.5)
    assert m == 1.0 and np.allclose(turns, plain(rotary, base) / 3.5, rtol=REL, atol=0)
    turns, m = B.sw_rope_frequencies(rotary, base, "base", 4.0)
    assert m == 1.0 and turns[0] == plain(rotary, base)[0]
    assert np.allclose(turns[-1], plain(rotary, base)[-1] / 4.0, rtol=2.0 ** -44, atol=0)       # (a power of a power)


@pytest.mark.parametrize("low,high", [(1.0, 4.0), (1.0, 32.0), (0.5, 0.6)])
def test_bands(low, high):
    original, factor = 8192, 8.0
    w = plain(128, 500000.0)
    turns, m = B.sw_rope_frequencies(128, 500000.0, "bands", factor, original, low, high)
    assert m == 1.0
    for got, one in zip(turns, w):
        rounds = original * one                                     # turns over the original length
        if rounds > high:
            want = one
        elif rounds < low:
            want = one / factor
        else:
            share = (rounds - low) / (high - low)
            want = share * one + (1 - share) * one / factor
        assert abs(got - want) <= 2.0 ** -44 * want                 # (a difference next to a border)


def test_ramp():
    w = plain(64, 10000.0)
    turns, m = B.sw_rope_frequencies(64, 10000.0, "ramp", 16.0, 4096, 1.0, 32.0)
    assert abs(m - (0.1 * math.log(16.0) + 1)) < 1e-6
    pair = lambda t: 32 * math.log(4096 / (t * 2 * math.pi)) / math.log(10000.0)  # noqa: E731
    first, last = math.floor(pair(32.0)), math.ceil(pair(1.0))
    assert 0 < first < last < 32
    for i, (got, one) in enumerate(zip(turns, w)):
        share = min(max((i - first) / (last - first), 0.0), 1.0)
        assert abs(got - one * ((1 - share) + share / 16.0)) <= REL * one
    assert (turns[:first + 1] == B.sw_rope_frequencies(64, 10000.0)[0][:first + 1]).all()
    assert B.sw_rope_frequencies(64, 10000.0, "ramp", 1.0, 4096, 1.0, 32.0)[1] == 1.0


@pytest.mark.parametrize("args", [(0,), (-16,), (24,), (144,), (64, 1.0), (64, 0.0), (64, math.nan), (64, math.inf), (64, 1e4, "linear", 0.5),
                                  (64, 1e4, "linear", math.nan), (64, 1e4, "bands", 2.0, 0.0, 1.0, 4.0), (64, 1e4, "bands", 2.0, 8192, 4.0, 4.0),
                                  (64, 1e4, "ramp", 2.0, 8192, 0.0, 4.0), (64, 1e4, "ramp", 2.0, math.inf, 1.0, 4.0)])
def test_frequencies_refused(args):
    with pytest.raises(B.SwError) as e:
        B.sw_rope_frequencies(*args)
    assert e.value.status in (B.SW_ERR_INVALID_ARG, B.SW_ERR_UNSUPPORTED)


def test_frequencies_null_and_unknown():
    m = C.c_float()
    assert B._lib.sw_rope_frequencies(64, 1e4, 0, 1.0, 0.0, 0.0, 0.0, None, C.byref(m)) == B.SW_ERR_INVALID_ARG
    table = (C.c_double * 32)()
    for scaling in (-1, 5):
        assert B._lib.sw_rope_frequencies(64, 1e4, scaling, 1.0, 0.0, 0.0, 0.0, table, C.byref(m)) == B.SW_ERR_INVALID_ARG


@pytest.mark.parametrize("call", [
    lambda: B._lib.sw_rope_append(None, None, None, None, None, None, None, None, None),
    lambda: B._lib.sw_rope_run(None, None, None, None, None, None, None, None),
    lambda: B._lib.sw_cross_attn_run(None, None, None, None, None, None, None),
    lambda: B._lib.sw_sample_run(None, None, None, None, None),
])
def test_null_context(call):
    assert call() == B.SW_ERR_INVALID_ARG
    assert "null context" in B.sw_last_error()


def test_rows_of_an_expanded_tensor_are_refused():
    """One row expanded to many has a stride of 0, which the C interface takes for dense rows: it would read behind the row."""
    shape = W.AttnShape(8, 2, 64)
    ctx, batch = SimpleNamespace(shape=shape, handle=None), SimpleNamespace(rows=5, struct=None)
    turns, magnitude = B.sw_rope_frequencies(64)
    rope = B.Rope(torch.from_numpy(turns), magnitude=magnitude, device="cpu")
    q, k = torch.zeros(5, 8, 64, dtype=torch.bfloat16), torch.zeros(5, 2, 64, dtype=torch.bfloat16)
    for bad_q, bad_k in ((q[:1].expand(5, 8, 64), k), (q, k[:1].expand(5, 2, 64)), (q.as_strided((5, 8, 64), (256, 64, 1)), k)):
        with pytest.raises(ValueError, match="rows overlap"):
            B.sw_rope_run(ctx, batch, rope, bad_q, bad_k, torch.empty_like(q), torch.empty_like(k), stream=0)
        with pytest.raises(ValueError, match="rows overlap"):
            B.sw_rope_append(ctx, None, batch, rope, bad_q, bad_k, k, torch.empty_like(q), stream=0)


def test_a_rope_is_set_once():
    """Its calls read a structure made once: an attribute that is exchanged later would not be seen."""
    rope = B.Rope(torch.zeros(32, dtype=torch.float64), device="cpu", positions=torch.zeros(3, dtype=torch.int32))
    for name in ("turns", "interleaved", "magnitude", "positions"):
        with pytest.raises(AttributeError):
            setattr(rope, name, getattr(rope, name))
