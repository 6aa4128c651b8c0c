"""The operators one after another as a layer of an encoder-decoder model calls them: sources into a pool of their own, then for the prompts and for
some tokens after them rotary positions with the append, attention, cross attention, logits, and the draw of the next tokens.  What each call returns is
compared with its plain form on the inputs it had."""
import numpy as np
import pytest
import torch

from paper_2609_07883_b200 import binding as B
from paper_2609_07883_b200 import workloads as W
from tests import more_op_util as M
from tests import op_util as U

pytestmark = pytest.mark.gpu

SHAPE, VOCAB, PAGES = W.AttnShape(8, 2, 64), 4001, 64
PROMPTS, SOURCES, STEPS = [37, 20, 1], [50, 0, 129], 20


def pages_of(n):
    return -(-n // U.PAGE)


def chunk_batch(lists, prefixes, lens):
    indptr = np.concatenate([[0], np.cumsum([len(x) for x in lists])]).astype(np.int32)
    none = np.zeros(0, np.int32)
    return W.MixedBatch(SHAPE, PAGES, prefixes[0], sum(lens), np.concatenate(lists).astype(np.int32), none, np.zeros(1, np.int32), none,
                        chunk_prefix_lens=np.array(prefixes, np.int32), chunk_lens=np.array(lens, np.int32), chunk_page_indptr=indptr)


def decode_batch(lists, lens):
    lists = [x[:pages_of(n)] for x, n in zip(lists, lens)]
    indptr = np.concatenate([[0], np.cumsum([len(x) for x in lists])]).astype(np.int32)
    none = np.zeros(0, np.int32)
    return W.MixedBatch(SHAPE, PAGES, 0, 0, none, np.array(lens, np.int32), indptr, np.concatenate(lists).astype(np.int32))


@pytest.mark.parametrize("interleaved,settings", [(False, dict(temperature=0.8, top_k=40, top_p=0.9)), (True, dict(min_p=0.05))])
def test_layer(interleaved, settings):
    dev = torch.device("cuda", 0)
    gen = torch.Generator(device=dev)
    gen.manual_seed(17)
    normal = lambda *s: torch.randn(*s, device=dev, generator=gen).to(torch.bfloat16)  # noqa: E731
    ctx = B.Context(SHAPE, PAGES, 256, 8, 0)
    pool, source_pool = (torch.zeros(PAGES, 2, 2, U.PAGE, 64, device=dev, dtype=torch.bfloat16) for _ in range(2))
    ids = np.random.default_rng(3).permutation(PAGES)
    room = [pages_of(n + STEPS) for n in PROMPTS]
    lists = np.split(ids[:sum(room)], np.cumsum(room)[:-1])
    source_lists = np.split(ids[:sum(pages_of(n) for n in SOURCES)], np.cumsum([pages_of(n) for n in SOURCES])[:-1])
    live = [i for i, n in enumerate(SOURCES) if n > 0]
    batch = chunk_batch([source_lists[i] for i in live], [0] * len(live), [SOURCES[i] for i in live])
    B.sw_kv_append(ctx, source_pool, B.DeviceBatch(batch, dev), normal(batch.num_rows, 2, 64), normal(batch.num_rows, 2, 64))

    turns, magnitude = B.sw_rope_frequencies(64, 10000.0, "ramp", 4.0, 1024, 1.0, 32.0)
    rope = B.Rope(turns, interleaved, magnitude, device=dev)
    embed, project, head = normal(VOCAB, 256), normal(256, 12 * 64) / 16, normal(512, VOCAB) / 8
    tokens = torch.randint(VOCAB, (sum(PROMPTS),), device=dev, generator=gen)
    drawn = []
    for step in range(STEPS):
        if step == 0:
            batch = chunk_batch([x[:pages_of(n)] for x, n in zip(lists, PROMPTS)], [0, 0, 0], PROMPTS)
            sources = chunk_batch(source_lists, SOURCES, PROMPTS)
        else:
            batch = decode_batch(lists, [n + step for n in PROMPTS])
            sources = decode_batch(source_lists, SOURCES)
        db, source_db = B.DeviceBatch(batch, dev), B.DeviceBatch(sources, dev)
        qkv = (embed[tokens] @ project).view(-1, 12, 64)
        q, k, v = qkv[:, :8], qkv[:, 8:10], qkv[:, 10:]
        q_turned, out, crossed = (torch.full((len(tokens), 8, 64), float("nan"), device=dev, dtype=torch.bfloat16) for _ in range(3))
        lse, cross_lse = (torch.empty(len(tokens), 8, device=dev) for _ in range(2))
        B.sw_rope_append(ctx, pool, db, rope, q, k, v, q_turned)
        B.sw_mixed_attn_run(ctx, pool, db, q_turned, out, lse)
        B.sw_cross_attn_run(ctx, source_pool, source_db, q_turned, crossed, cross_lse)
        last = np.cumsum(PROMPTS) - 1 if step == 0 else np.arange(len(PROMPTS))
        logits = ((out + crossed)[torch.from_numpy(last).to(dev)].flatten(1) @ head).float()
        u = torch.rand(len(PROMPTS), device=dev, generator=gen)
        next_tokens, log_probs = torch.empty(len(PROMPTS), dtype=torch.int32, device=dev), torch.empty(len(PROMPTS), device=dev)
        columns = {k_: torch.full((len(PROMPTS),), v_, device=dev, dtype=torch.int32 if k_ == "top_k" else torch.float32) for k_, v_ in settings.items()}
        B.sw_sample_run(ctx, logits, u, next_tokens, log_probs, **columns)
        assert B.sw_check_status(ctx, raise_on_error=False) == (0, 0)

        want, tol = M.rotate(q, M.batch_positions(batch), turns, interleaved, magnitude)
        assert bool(((q_turned.double() - want).abs() <= tol).all())
        want, _, tol, _, _ = U.attention(batch, pool.double(), q_turned)
        assert bool(((out.double() - want).abs() <= tol).all())
        want, want_lse, tol, _ = M.cross_attention(sources, source_pool, q_turned)
        assert bool(((crossed.double() - want).abs() <= tol).all()) and torch.equal(torch.isinf(cross_lse), torch.isinf(want_lse))
        for r in range(len(PROMPTS)):
            token, lp, _ = M.draw(logits[r].double().cpu().numpy(), float(u[r]), **{k_: float(c[r]) if k_ != "top_k" else int(c[r]) for k_, c in columns.items()})
            assert int(next_tokens[r]) == token
        tokens = next_tokens.long()
        drawn.append(tokens.tolist())
    assert len({tuple(x) for x in drawn}) > 1
