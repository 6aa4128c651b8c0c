"""What the operators beside the plain iteration refuse, or size, without a GPU."""
import pytest

from paper_2609_07883_b200 import binding as B
from paper_2609_07883_b200 import workloads as W


def layout(*heads, pages=1024, **kw):
    return B.make_layout(W.AttnShape(*heads, **kw), pages)


def test_scratch_sizes():
    llama = layout(32, 8, 128)
    assert B.sw_kv8_scratch_bytes(llama, 0) == 0
    assert B.sw_kv8_scratch_bytes(llama, 3) == 3 * 2 * 8 * 16 * 128 * 2 + 256          # three bf16 pages and their list
    assert B.sw_kv8_scratch_bytes(llama, 65) == 65 * 65536 + 512
    assert B.sw_kv8_scratch_bytes(llama, -1) == 0 and B.sw_kv8_scratch_bytes(llama, 1 << 28) == 0
    assert B.sw_kv8_scratch_bytes(layout(32, 8, 96), 3) == 0
    assert B.sw_attn_weights_scratch_bytes(llama, 5) == 5 * 16 * 32 * 4
    assert B.sw_attn_weights_scratch_bytes(llama, 1 << 24) == (1 << 24) * 16 * 32 * 4   # beyond 32 bits
    assert B.sw_attn_weights_scratch_bytes(llama, -1) == 0 and B.sw_attn_weights_scratch_bytes(llama, 1 << 31) == 0
    assert B.sw_attn_weights_scratch_bytes(layout(32, 8, 128, page_size=32), 5) == 0


@pytest.mark.parametrize("call", [
    lambda: B._lib.sw_mixed_attn_window_run(None, None, None, 5, 0, None, None, None, None),
    lambda: B._lib.sw_mixed_iteration_window_run(None, None, None, 5, 0, 256, 256, None, None, None, None),
    lambda: B._lib.sw_kv8_append(None, None, None, None, None, None, None),
    lambda: B._lib.sw_kv8_attn_run(None, None, None, None, None, None, None, None, 0, None),
    lambda: B._lib.sw_decode_attn_weights_run(None, None, None, None, None, None, None, None, 0, None),
    lambda: B._lib.sw_kv_evict(None, None, None, None, None, None, None, 1, 0, 0, None, None, None),
])
def test_null_context(call):
    assert call() == B.SW_ERR_INVALID_ARG
    assert "null context" in B.sw_last_error()


def test_window_is_checked_before_anything_else():
    for window, sinks in [(0, 0), (-3, 0), (1, -1)]:
        assert B._lib.sw_mixed_attn_window_run(None, None, None, window, sinks, None, None, None, None) == B.SW_ERR_INVALID_ARG
        assert "window" in B.sw_last_error()
