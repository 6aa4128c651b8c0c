"""Sampling from rows that do not fit in the shared memory of their CTAs: the last blocks of every warp's run are read again from memory."""
import math

import pytest
import torch

from paper_2609_07883_b200 import binding as B
from paper_2609_07883_b200 import workloads as W
from tests import more_op_util as M

pytestmark = pytest.mark.gpu
INF, NAN = math.inf, math.nan
BLOCK, SMS, LISTED = 128, 148, 1024 * 8     # logits of a block; bytes of shared memory that are certainly not for logits
SETTINGS = [dict(), dict(temperature=0.0), dict(temperature=0.7), dict(top_k=50), dict(top_k=3000), dict(top_p=0.9), dict(top_p=0.999), dict(min_p=0.05),
            dict(temperature=3.0, top_p=0.5), dict(temperature=0.8, top_k=40, top_p=0.95, min_p=0.02), dict(top_k=70000, top_p=0.7), dict(min_p=1.0, top_p=0.3)]
# two CTAs an SM (19 to 37 rows) and three; 16-bit logits only leave shared memory with three
SHAPES = [(64, 151936, torch.float32), (32, 262144, torch.float32), (20, 393216, torch.float32), (40, 300001, torch.float32),
          (128, 300000, torch.bfloat16), (128, 300000, torch.float16)]


def outside(rows, vocab, size, behind):
    """Logits of a row that starts `behind` of them past a 16-byte boundary which no CTA keeps: by the launch's own arithmetic, with the most room there
    can be.  Runs of eight warps in each of eight CTAs."""
    positions = vocab + 16 // size - 1
    stretch = -(-positions // (8 * BLOCK)) * BLOCK
    ctas = 3 if rows * 8 > 2 * SMS else 2
    assert rows * 8 > SMS and positions > 4 * 16384
    blocks, room = stretch // BLOCK, (228 * 1024 // ctas - 1024 - LISTED) // (8 * BLOCK * size)
    at = torch.arange(vocab) + behind
    block = at % stretch // BLOCK
    first = torch.tensor([blocks * w // 8 for w in range(9)])
    warp = torch.searchsorted(first, block, right=True) - 1
    left = block - first[warp] >= room
    assert 0 < int(left.sum()) < vocab
    return left


def special_rows(x, left):
    """Rows whose outcome hangs on what lies outside, in place."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(7)
    vocab, far = x.shape[1], torch.nonzero(left)[:, 0].cuda()
    some = far[torch.randperm(len(far), generator=gen, device="cuda")]
    x[1, some[:40]] += 12
    x[2, ::1009] = INF
    x[3, some[0]] = INF
    x[4] = NAN
    x[4, some[:700]] = x[0, :700]
    x[5] = x[5].clamp(max=3.0)
    x[5, ::3] = 3.0
    x[6, ::2] = NAN
    x[6, 1::4] = -INF
    x[7] = torch.finfo(x.dtype).min
    x[7, some[:3]] = torch.tensor([1.0, 2.0, 2.0], device="cuda", dtype=x.dtype)
    x[8] = torch.round(x[8])
    x[9, some] = INF
    x[10] = -INF
    x[11, some] += 6
    x[12] = x[12] * 0.01
    return list(range(13)) + [x.shape[0] - 1]


@pytest.mark.parametrize("behind", [0, 1])
@pytest.mark.parametrize("rows,vocab,dtype", SHAPES)
def test_rows_beyond_shared_memory(rows, vocab, dtype, behind):
    ctx = B.Context(W.AttnShape(8, 2, 64), 64, 1, 1, 0)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(vocab + behind)
    size = torch.finfo(dtype).bits // 8
    pad = 16 // size
    stride = -(-(vocab + behind) // pad) * pad                    # (every row starts `behind` past a boundary)
    x = torch.full((rows, stride), INF, device="cuda", dtype=dtype)[:, behind:behind + vocab]
    x.copy_(2 * torch.randn(rows, vocab, device="cuda", generator=gen))
    assert x.data_ptr() % 16 == behind * size and x.stride(0) % pad == 0
    looked_at = special_rows(x, outside(rows, vocab, size, behind))
    u = torch.rand(rows, device="cuda", generator=gen)
    x64 = {r: x[r].double().cpu().numpy() for r in looked_at}
    for settings in SETTINGS if behind == 0 else SETTINGS[::2]:
        columns = {k: torch.full((rows,), v, dtype=torch.int32 if k == "top_k" else torch.float32, device="cuda") for k, v in settings.items()}
        given = {k: c[0].item() for k, c in columns.items()}      # (as fp32 holds them)
        tokens, log_probs = torch.full((rows,), -7, dtype=torch.int32, device="cuda"), torch.full((rows,), 7.0, device="cuda")
        B.sw_sample_run(ctx, x, u, tokens, log_probs, **columns)
        for r in looked_at:
            token, lp, _ = M.draw(x64[r], float(u[r]), **given)
            assert int(tokens[r]) == token, f"row {r}: {int(tokens[r])} and not {token} ({settings})"
            got = float(log_probs[r])
            # fp32's rounding, and half a unit of a weight and of their sum, as in the other tests of sampling
            assert got == lp or abs(got - lp) <= 2.0 ** -24 * abs(lp) + 2e-13 + 1.0 / (math.exp(lp) * M.UNIT), f"row {r}: {got} and not {lp}"
