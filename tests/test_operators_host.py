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


@pytest.mark.parametrize("new_len,kept,name", [
    (0x10000, 0x90000, "decode_kv_len"), (0x1000C, 0x90000, "decode_kv_len"), (0xFFF4, 0x90000, "decode_kv_len"),   # the same; its last word; from in front
    (0x20010, 0x90000, "decode_page_indptr"), (0x30000, 0x90000, "decode_pages"), (0x40000, 0x90000, "row_of"), (0x50010, 0x90000, "new_page_indptr"),
    (0x60000, 0x90000, "new_pages"), (0x70004, 0x90000, "new_row_of"), (0x80000, 0x10000, "decode_kv_len"), (0x80000, 0x80000 - 4 * 4 * 8 + 4, "new_len"),
    (0x80000, 0x70000 - 4 * 4 * 8 + 4, "new_row_of")])
def test_evict_refuses_outputs_over_inputs(new_len, kept, name):
    """Four requests, a budget of 8: lengths are not updated in place, nor anything else that the call still reads."""
    batch = B.sw_batch(0, 0, None, 0, 4, 0x10000, 0x20000, 0x30000, 0, None, None, None)
    weights = B.sw_key_weights(0x1000000, 8, 64, 0x40000)
    assert B._lib.sw_kv_evict(None, 0x2000000, batch, weights, 0x50000, 0x60000, 0x70000, 8, 0, 0, kept, new_len, None) == B.SW_ERR_INVALID_ARG
    assert "overlaps " + name in B.sw_last_error()


def test_evict_takes_neighbouring_arrays():
    batch = B.sw_batch(0, 0, None, 0, 4, 0x10000, 0x20000, 0x30000, 0, None, None, None)
    weights = B.sw_key_weights(0x1000000, 8, 64, 0x40000)
    for new_len, kept in [(0x10010, 0x90000), (0xFFF0, 0x90000), (0x80000, 0x70010), (0x80000, 0x80000 - 4 * 4 * 8)]:
        assert B._lib.sw_kv_evict(None, 0x2000000, batch, weights, 0x50000, 0x60000, 0x70000, 8, 0, 0, kept, new_len, None) == B.SW_ERR_INVALID_ARG
        assert "null context" in B.sw_last_error()


def test_rows_of_weights_that_are_too_long():
    import torch

    rows = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError):
        B.KeyWeights(torch.empty(1, 1, 2 ** 31, device="meta"), rows)      # (would wrap to a negative capacity)
