"""Successive iterations over an 8-bit pool as a server runs them: a prompt's chunks one after another beside decodes, each appended and then attended."""
import numpy as np
import pytest
import torch

from paper_2609_07883_b200 import binding as B
from tests import op_util as U

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,first,chunk,scratch", [((16, 4, 64), 20, 50, False), ((8, 2, 64), 0, 16, True), ((32, 8, 128), 700, 500, False),
                                                       ((32, 8, 128), 700, 500, True), ((8, 1, 128), 13, 129, False)])
def test_chunks_of_one_prompt(heads, first, chunk, scratch):
    """What an iteration appends is part of the prefix that the next one attends, and later rows may raise the scale of its last page."""
    steps, lens = 3, np.array([30, 15, 200], dtype=np.int32)
    c = U.Case(heads, lens + steps, [(first, steps * chunk)], seed=chunk)
    c.batch.chunk_len = chunk
    rows = chunk + len(lens)
    q, k_new, v_new, out, lse = c.q, c.k_new, c.v_new, c.out, c.lse
    codes, scales = U.quantise(c.pool)
    host, host_scales = codes.view(torch.uint8).cpu().clone(), scales.cpu().clone()
    gen = torch.Generator(device=c.dev)
    gen.manual_seed(chunk)
    room = torch.empty(B.sw_kv8_scratch_bytes(c.ctx.layout, len(c.batch.prefill_pages)), dtype=torch.uint8, device=c.dev) if scratch else None
    for step in range(steps):
        c.batch.prefix_len = first + chunk * step
        c.batch.decode_kv_len[:] = lens + step
        c.renew()
        c.q, c.k_new, c.v_new, c.out, c.lse = q[:rows], k_new[:rows], v_new[:rows], out[:rows], lse[:rows]
        for t in (c.q, c.k_new, c.v_new):
            t.copy_(torch.randn(t.shape, device=c.dev, generator=gen) * (1 + 3 * step))
        c.q /= 1 + 3 * step
        B.sw_kv8_append(c.ctx, codes, scales, c.db, c.k_new, c.v_new)
        B.sw_kv8_attn_run(c.ctx, codes, scales, c.db, c.q, c.out, c.lse, room)
        c.ok()
        U.append8(host, host_scales, U.entries_of(c.batch), c.k_new.cpu(), c.v_new.cpu())
        assert torch.equal(codes.view(torch.uint8).cpu(), host) and torch.equal(scales.cpu(), host_scales)
        c.check(U.dequantise(codes, scales), floor=2.0 ** -32)
