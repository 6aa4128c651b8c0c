"""Sampling where a row's CTAs have next to nothing to load before they tell one another of their largest logits, and where clusters start while
others run: the same draws in every launch, and those of the plain form."""
import pytest
import torch

from paper_2609_07883_b200 import binding as B
from paper_2609_07883_b200 import workloads as W
from tests import more_op_util as M

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab,rows", [(2049, 1), (2049, 73), (4097, 36), (8193, 1), (8193, 18), (16385, 700), (40000, 300)])
@pytest.mark.parametrize("settings", [dict(), dict(temperature=0.0), dict(top_k=30, top_p=0.9)])
def test_many_launches_in_a_row(dtype, vocab, rows, settings):
    ctx = B.Context(W.AttnShape(8, 2, 64), 64, 1, 1, 0)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(vocab + rows)
    x = (3 * torch.randn(rows, vocab, device="cuda", generator=gen)).to(dtype)
    u = torch.rand(rows, device="cuda", generator=gen)
    kinds = {"top_k": torch.int32}
    columns = {k: torch.full((rows,), v, dtype=kinds.get(k, torch.float32), device="cuda") for k, v in settings.items()}
    launches = 50
    tokens = torch.full((launches, rows), -7, dtype=torch.int32, device="cuda")
    log_probs = torch.zeros(launches, rows, device="cuda")
    for i in range(launches):
        B.sw_sample_run(ctx, x, u, tokens[i], log_probs[i], **columns)
    torch.cuda.synchronize()
    assert bool((tokens == tokens[0]).all()) and bool((log_probs == log_probs[0]).all())
    for r in {0, rows // 2, rows - 1}:
        assert int(tokens[0, r]) == M.draw(x[r].double().cpu().numpy(), float(u[r]), **{k: c[0].item() for k, c in columns.items()})[0]
