"""Tensors that the binding of cross attention, rotary positions and sampling refuses, without a GPU: the library would take their addresses as they are."""
from types import SimpleNamespace

import pytest
import torch

from paper_2609_07883_b200 import binding as B
from paper_2609_07883_b200 import workloads as W

SHAPE, ROWS = W.AttnShape(8, 2, 64), 5
STREAM = SimpleNamespace(cuda_stream=0)
BF16, F32 = torch.bfloat16, torch.float32


def context(device=torch.device("cpu")):
    return SimpleNamespace(shape=SHAPE, handle=None, device=device)


def batch(device="cpu"):
    return SimpleNamespace(rows=ROWS, struct=B.sw_batch(), device=torch.device(device))


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


def column(dtype=F32):
    return torch.zeros(ROWS, dtype=dtype)


def rope(device="cpu", positions=None):
    return B.Rope(torch.zeros(32, dtype=torch.float64), positions=positions, device=device)


I32 = torch.int32
# name of the argument in the message: how the call is made, and its tensors
CALLS = {
    "cross": (lambda ctx, pool, batch, q, out, lse: B.sw_cross_attn_run(ctx, pool, batch, q, out, lse, stream=STREAM),
              lambda: dict(kv_pool=torch.zeros(64, dtype=BF16), batch=batch(), q=rows(), out=rows(), lse=torch.zeros(5, 8))),
    "append": (lambda ctx, pool, batch, rope, q, k, v, q_out: B.sw_rope_append(ctx, pool, batch, rope, q, k, v, q_out, stream=STREAM),
               lambda: dict(kv_pool=torch.zeros(64, dtype=BF16), batch=batch(), rope=rope(), q=rows(), k=rows(2), v=rows(2), q_out=rows())),
    "run": (lambda ctx, batch, rope, q, k, q_out, k_out: B.sw_rope_run(ctx, batch, rope, q, k, q_out, k_out, stream=STREAM),
            lambda: dict(batch=batch(), rope=rope(), q=rows(), k=rows(2), q_out=rows(), k_out=rows(2))),
    "sample": (lambda ctx, *tensors: B.sw_sample_run(ctx, *tensors, stream=STREAM),
               lambda: dict(logits=torch.zeros(5, 100), uniform=column(), tokens=column(I32), log_probs=column(), temperature=column(), top_k=column(I32),
                            top_p=column(), min_p=column())),
}


@pytest.mark.parametrize("call,name", [(call, name) for call, (_, tensors) in CALLS.items() for name in tensors()])
def test_tensors_of_another_device_are_refused(call, name):
    """Its address would go to the kernel.  (The context's device is the CPU here, and the other one has no memory at all.)"""
    function, tensors = CALLS[call]
    given = tensors()
    with pytest.raises(B.SwError):                       # (everything is where it should be: the library's own refusal, of the missing context)
        function(context(), *given.values())
    given[name] = batch("meta") if name == "batch" else rope("meta") if name == "rope" else given[name].to("meta")
    with pytest.raises(ValueError, match=f"^{name} must be on cpu, not meta"):
        function(context(), *given.values())


@pytest.mark.parametrize("call", CALLS)
def test_tensors_of_the_host_are_refused(call):
    function, tensors = CALLS[call]
    with pytest.raises(ValueError, match="must be on cuda:0, not cpu"):
        function(context(torch.device("cuda", 0)), *tensors().values())


def test_positions_lie_where_the_frequencies_do():
    positions = torch.zeros(ROWS, dtype=I32)
    assert rope(positions=positions).positions is positions
    with pytest.raises(ValueError, match="^positions must be on meta, not cpu"):
        rope("meta", positions)
