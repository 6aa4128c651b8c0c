"""Tensors that the binding of cross attention, rotary positions and sampling refuses, without a GPU: the library would take their addresses as they are."""
from types import SimpleNamespace

import pytest
import torch

from paper_2609_07883_b200 import binding as B
from paper_2609_07883_b200 import workloads as W

SHAPE, ROWS = W.AttnShape(8, 2, 64), 5
STREAM = SimpleNamespace(cuda_stream=0)
BF16, F32 = torch.bfloat16, torch.float32


def context():
    return SimpleNamespace(shape=SHAPE, handle=None, device=torch.device("cuda", 0))


def batch():
    return SimpleNamespace(rows=ROWS, struct=B.sw_batch())


def rows(heads=8, count=ROWS, dtype=BF16, d=64):
    return torch.zeros(count, heads, d, dtype=dtype)


def cross(q, out, lse=None):
    B.sw_cross_attn_run(context(), torch.zeros(64, dtype=BF16), batch(), q, out, lse, stream=STREAM)


@pytest.mark.parametrize("bad", [rows(dtype=F32), rows(dtype=torch.float16), rows(count=4), rows(d=32), rows(heads=4), rows(heads=16)[:, ::2],
                                 rows(count=10)[::2], rows()[:1].expand(5, 8, 64), rows().transpose(0, 1)])
def test_cross_attention_refuses_rows(bad):
    with pytest.raises(ValueError, match="^q must"):
        cross(bad, rows())
    with pytest.raises(ValueError, match="^out must"):
        cross(rows(), bad)


@pytest.mark.parametrize("lse", [torch.zeros(4, 8), torch.zeros(5, 8, dtype=BF16), torch.zeros(5, 8, dtype=torch.float64), torch.zeros(5, 16)[:, ::2],
                                 torch.zeros(1, 8).expand(5, 8)])
def test_cross_attention_refuses_log_sum_exps(lse):
    with pytest.raises(ValueError, match="^lse must"):
        cross(rows(), rows(), lse)


def test_cross_attention_leaves_missing_tensors_to_the_library():
    with pytest.raises(B.SwError) as e:
        B.sw_cross_attn_run(context(), None, batch(), None, None, stream=STREAM)
    assert e.value.status == B.SW_ERR_INVALID_ARG
