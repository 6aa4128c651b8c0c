"""Sampling (sw_sample_run) against the plain form: tokens are equal, log-probabilities to fp32.

A log-probability is rounded to fp32 (2^-24 of it), and weights and their sum are off by 8e-14 of themselves and half a unit each: 2^-45 of the largest
weight, which of a token with n units is 1 / (2 n).
"""
import math

import numpy as np
import pytest
import torch

from paper_2609_07883_b200 import binding as B
from paper_2609_07883_b200 import workloads as W
from tests import more_op_util as M

pytestmark = pytest.mark.gpu
INF, NAN, LOWEST = math.inf, math.nan, float(np.finfo(np.float32).min)


@pytest.fixture(scope="module")
def ctx():
    return B.Context(W.AttnShape(8, 2, 64), 64, 1, 1, 0)


def column(v, rows, dtype):
    if v is None or isinstance(v, torch.Tensor):
        return v
    return torch.tensor([v] * rows if np.isscalar(v) else list(v), dtype=dtype, device="cuda")


def sample(ctx, x, u, temperature=None, top_k=None, top_p=None, min_p=None):
    rows = x.shape[0]
    f = torch.float32
    args = [column(temperature, rows, f), column(top_k, rows, torch.int32), column(top_p, rows, f), column(min_p, rows, f)]
    tokens = torch.full((rows,), -7, dtype=torch.int32, device="cuda")
    log_probs = torch.full((rows,), 7.0, device="cuda")
    B.sw_sample_run(ctx, x, column(u, rows, f), tokens, log_probs, *args)
    torch.cuda.synchronize()
    return tokens.cpu().numpy(), log_probs.cpu().numpy(), args


def check(ctx, x, u, temperature=None, top_k=None, top_p=None, min_p=None):
    u = column(u, x.shape[0], torch.float32)
    tokens, log_probs, args = sample(ctx, x, u, temperature, top_k, top_p, min_p)
    x64 = x.double().cpu().numpy()
    settings = [a.cpu().numpy() if a is not None else None for a in args]
    for r in range(x.shape[0]):
        t, k, p, least = (float(s[r]) if s is not None else d for s, d in zip(settings, (1.0, 0, 1.0, 0.0)))
        token, lp, _ = M.draw(x64[r], float(u[r]), t, int(k), p, least)
        assert tokens[r] == token, f"row {r}: {tokens[r]} and not {token} (of {x.shape[1]}; u {float(u[r])}, T {t}, k {k}, p {p}, min_p {least})"
        if lp == -INF:
            assert log_probs[r] == -INF
        else:
            assert abs(log_probs[r] - lp) <= 2.0 ** -24 * abs(lp) + 2e-13 + 1.0 / (math.exp(lp) * M.UNIT), f"row {r}: {log_probs[r]} and not {lp}"
    return tokens


def logits(rows, vocab, seed, dtype=torch.float32, kind="usual"):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    x = torch.randn(rows, vocab, device="cuda", generator=gen) * 2
    if kind == "usual":
        at = torch.randint(vocab, (rows, 40), device="cuda", generator=gen)
        x.scatter_add_(1, at, 6 + 10 * torch.rand(rows, 40, device="cuda", generator=gen))
    return x.to(dtype)


def uniforms(rows, seed):
    return torch.from_numpy(np.random.default_rng(seed).random(rows).astype(np.float32)).cuda()


VOCABS = [1, 2, 3, 7, 31, 127, 128, 129, 1000, 2047, 2048, 4100, 16384, 16385, 32003, 50257, 128256, 151936, 262144, 393216]
SETTINGS = [dict(), dict(temperature=0.7), dict(temperature=0.0), dict(top_k=1), dict(top_k=50), dict(top_p=0.9), dict(min_p=0.05),
            dict(temperature=0.8, top_k=40, top_p=0.95), dict(temperature=1.3, top_k=200, top_p=0.8, min_p=0.02), dict(top_p=0.999), dict(top_k=3000)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("vocab", VOCABS)
def test_sizes(ctx, vocab, dtype):
    rows = 3
    for i, settings in enumerate(SETTINGS):
        for kind in ("usual", "flat"):
            check(ctx, logits(rows, vocab, vocab + i, dtype, kind), uniforms(rows, i), **settings)


@pytest.mark.parametrize("vocab,rows", [(128256, 70), (32003, 300), (1000, 700), (2049, 40)])
def test_batches_with_settings_of_their_own(ctx, vocab, rows):
    rng = np.random.default_rng(rows)
    pick = lambda *v: rng.choice(v, rows)  # noqa: E731
    check(ctx, logits(rows, vocab, rows), uniforms(rows, rows), pick(0.0, 0.3, 0.7, 1.0, 1.5, 5.0), pick(0, 0, 1, 2, 20, 100, 1500, vocab, vocab - 1, vocab + 5, -3),
          pick(1.0, 1.5, 0.0, 0.1, 0.5, 0.9, 0.99, 0.99999), pick(0.0, 0.0, 0.01, 0.1, 0.5, 1.0, 2.0))


def test_rows_at_any_place(ctx):
    """Rows that begin anywhere, with a stride of their own; what lies between them is not looked at."""
    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        for first in (0, 1, 2, 3, 5, 7):
            whole = torch.full((5, 1013), INF, device="cuda", dtype=dtype)
            part = whole[:, first:first + 1000]
            part.copy_(logits(5, 1000, first, dtype))
            check(ctx, part, uniforms(5, first), top_k=30, top_p=0.9)
            check(ctx, part, uniforms(5, first + 1))


def test_equal_logits(ctx):
    """Ties go to the lowest index: of equal logits the limits keep the first ones."""
    for vocab in (5, 128, 1000, 40000):
        for dtype in (torch.float32, torch.bfloat16):
            x = torch.full((64, vocab), 1.5, device="cuda", dtype=dtype)
            u = torch.linspace(0, 1, 65)[:64].cuda()
            check(ctx, x, u)
            check(ctx, x, u, top_k=3)
            check(ctx, x, u, top_p=0.5)
            check(ctx, x, u, top_k=4, top_p=0.5)
            check(ctx, x, u, top_k=vocab - 1, top_p=0.26, min_p=1.0)
            x[:, vocab // 2:] = 0.5
            check(ctx, x, u, top_k=vocab // 2 + 1)
            check(ctx, x, u, top_k=vocab // 2 + 1, top_p=0.9999)
            check(ctx, x, u, top_p=0.9)
            check(ctx, x, u, temperature=0.0)
            x[:, ::3] = 2.5
            check(ctx, x, u, top_k=vocab // 3 + vocab // 10 + 2, top_p=0.97)


def test_half_of_two(ctx):
    x = torch.tensor([[0.0, 3.0, 3.0, -1.0]], device="cuda").repeat(4, 1)
    tokens = check(ctx, x, [0.0, 0.4, 0.6, 0.999], top_p=0.4)
    assert tokens.tolist() == [1, 1, 1, 1]
    assert check(ctx, x, [0.0, 0.4, 0.6, 0.999], top_k=2).tolist() == [1, 1, 2, 2]


@pytest.mark.parametrize("fill", [-INF, LOWEST, NAN])
@pytest.mark.parametrize("vocab", [40, 3001, 128256])
def test_masks(ctx, vocab, fill):
    x = logits(8, vocab, 5)
    keep = [vocab, 1, 2, 3, 20, 0, 30, vocab - 1]
    rng = np.random.default_rng(vocab)
    for r, n in enumerate(keep):
        gone = torch.from_numpy(rng.permutation(vocab)[n:].copy()).cuda()
        x[r, gone] = fill
    for settings in SETTINGS + [dict(temperature=1e30), dict(temperature=INF), dict(temperature=1e-30)]:
        check(ctx, x, uniforms(8, 3), **settings)


def test_infinite_and_extreme_logits(ctx):
    x = logits(9, 5000, 6)
    x[0, 17] = INF
    x[1, [5, 100, 4999]] = INF
    x[2] = -INF
    x[2, 4444] = INF
    x[3] = LOWEST
    x[3, 1000:] = -INF
    x[4] = -LOWEST
    x[5] *= 1e30
    x[6] *= 1e-30
    x[7] += 1e4
    x[8] = torch.where(x[8] > 0, 0.0, -0.0)
    for settings in SETTINGS + [dict(temperature=1e30, top_p=0.5), dict(temperature=1e-38, top_p=0.5), dict(temperature=INF, top_p=0.3)]:
        check(ctx, x, uniforms(9, 4), **settings)


@pytest.mark.parametrize("vocab", [700, 5000, 33000, 128256])
def test_many_at_the_threshold(ctx, vocab):
    """More logits at, or just above, a threshold than one CTA can collect; infinite ones among them; spread evenly or all in one place."""
    x = logits(6, vocab, 21, kind="flat").clamp(max=3.0)
    x[1, : vocab // 2] = INF
    x[2, ::7] = INF
    x[3] = torch.round(x[3])
    x[4] = torch.where(torch.arange(vocab, device="cuda") % 50 == 0, 3.0, x[4])
    x[5, -vocab // 3:] = 3.0
    u = torch.tensor([0.02, 0.3, 0.5, 0.7, 0.9, 0.999], device="cuda")
    for dtype in (torch.float32, torch.bfloat16):
        for settings in (dict(top_p=0.2), dict(top_p=0.6), dict(top_p=0.97), dict(top_k=vocab // 9 + 1), dict(top_k=vocab // 3, top_p=0.7, min_p=0.5),
                         dict(top_p=0.95, temperature=3.0), dict(top_p=0.9, temperature=0.05)):
            check(ctx, x.to(dtype), u, **settings)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("vocab", [5000, 50257, 128256, 300000])
def test_a_tail_of_small_weights(ctx, vocab, dtype):
    """A threshold far down among logits that are each nothing beside the largest; or just behind a step, where nothing follows for long; and wide spreads."""
    g = torch.Generator(device="cuda")
    g.manual_seed(vocab)
    x = torch.randn(8, vocab, device="cuda", generator=g) * 0.05 - torch.tensor([14.0, 16.5, 20.0, 28.0, 9.0, 3.0, 0.0, 0.0], device="cuda")[:, None]
    x[:6, vocab // 3] = 0.0
    x[4, 5:505] = 0.0
    x[5, ::2] -= 12.0
    x[6] *= 60.0
    x[7] *= 400.0
    u = torch.tensor([0.9999999, 0.99, 0.5, 0.999, 0.9, 0.97, 0.6, 0.8], device="cuda")
    x = x.to(dtype)
    for settings in (dict(top_p=0.9), dict(top_p=0.99), dict(top_p=0.9995), dict(top_p=0.9999999), dict(top_p=0.95, temperature=1.5),
                     dict(top_p=0.99, temperature=20.0), dict(top_k=vocab // 2, top_p=0.95, temperature=1.2)):
        check(ctx, x, u, **settings)


def test_extreme_settings(ctx):
    x = logits(10, 3001, 8)
    for t in (0.0, -1.0, NAN, 1e-45, 1e-30, 1e-8, 1e-4, 1e4, 1e30, 3e38, INF):
        check(ctx, x, uniforms(10, 1), temperature=t)
        check(ctx, x, uniforms(10, 2), temperature=t, top_p=0.7, top_k=100)
    for p in (-1.0, 0.0, 1e-30, 1e-9, 0.3, 1 - 2.0 ** -24, 1.0, 7.0, INF):
        check(ctx, x, uniforms(10, 3), top_p=p)
        check(ctx, x, uniforms(10, 3), top_p=p, top_k=17)
    for least in (-1.0, 1e-30, 1e-9, 0.5, 1 - 2.0 ** -24, 1.0, 5.0, INF):
        check(ctx, x, uniforms(10, 4), min_p=least)
        check(ctx, x, uniforms(10, 4), min_p=least, top_p=0.6)
    for k in (-2 ** 31, -1, 0, 1, 2, 3000, 3001, 2 ** 31 - 1):
        check(ctx, x, uniforms(10, 5), top_k=k)
    off = dict(top_p=NAN, min_p=NAN)
    assert (sample(ctx, x, uniforms(10, 6), **off)[0] == sample(ctx, x, uniforms(10, 6))[0]).all()


def test_uniform_at_its_ends(ctx):
    x = logits(8, 40000, 9)
    u = [0.0, 2.0 ** -149, 2.0 ** -24, 1 - 2.0 ** -24, 1.0, 5.0, -3.0, NAN]
    for settings in SETTINGS:
        check(ctx, x, u, **settings)
        check(ctx, x.half(), u, **settings)


@pytest.mark.parametrize("order", ["falling", "rising", "blocks"])
def test_logits_in_order(ctx, order):
    """The large logits side by side: in one CTA's stretch, at its ends, most of the warps far below."""
    for vocab in (20000, 128256):
        x = logits(4, vocab, 10, kind="flat").sort(dim=1, descending=order == "falling").values
        if order == "blocks":
            x = torch.cat([x[:, vocab // 2:], x[:, :vocab // 2] - 40], 1)
        for settings in SETTINGS:
            check(ctx, x, uniforms(4, 7), **settings)


@pytest.mark.parametrize("settings", [dict(), dict(top_k=20), dict(top_p=0.8), dict(temperature=0.6, top_k=30, top_p=0.9, min_p=0.05)])
def test_share_of_every_token(ctx, settings):
    """Draws at equal steps of u: every kept token as often as its weight says, to within one draw, and no other."""
    one = logits(1, 700, 11)
    n = 4096
    u = (torch.arange(n, device="cuda") + 0.5) / n
    tokens, _, _ = sample(ctx, one.repeat(n, 1), u, **settings)
    assert (np.diff(tokens) >= 0).all()
    x = one[0].double().cpu().numpy()
    _, _, kept = M.draw(x, 0.5, **settings)
    w = np.exp((x[kept] - x.max()) / settings.get("temperature", 1.0))
    counts = np.bincount(tokens, minlength=700)
    assert counts.sum() == counts[kept].sum() == n
    assert np.abs(counts[kept] - n * w / w.sum()).max() <= 1.01


def test_alone_and_in_a_batch(ctx):
    """A row's result does not depend on the other rows, nor on how many CTAs it gets."""
    x, u = logits(200, 32003, 12), uniforms(200, 8)
    many, lp, _ = sample(ctx, x, u, top_p=0.95)
    for r in (0, 77, 199):
        tokens, one, _ = sample(ctx, x[r:r + 1].clone(), u[r:r + 1].clone(), top_p=0.95)
        assert tokens[0] == many[r] and one[0] == lp[r]


def test_captured_on_streams_of_their_own(ctx):
    """Two captured launches replayed beside each other, one context."""
    xs, us = [logits(40, 128256, 13), logits(40, 32003, 14)], [uniforms(40, 9), uniforms(40, 10)]
    settings = dict(top_k=column(30, 40, torch.int32), top_p=column(0.9, 40, torch.float32))
    tokens = [torch.zeros(40, dtype=torch.int32, device="cuda") for _ in xs]
    log_probs = [torch.zeros(40, device="cuda") for _ in xs]
    streams, graphs = [torch.cuda.Stream() for _ in xs], []
    for i, st in enumerate(streams):
        st.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(st):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=st):
                B.sw_sample_run(ctx, xs[i], us[i], tokens[i], log_probs[i], **settings)
            graphs.append(g)
    for _ in range(20):
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
    torch.cuda.synchronize()
    for i in range(2):
        want, lp, _ = sample(ctx, xs[i], us[i], **settings)
        assert (tokens[i].cpu().numpy() == want).all() and (log_probs[i].cpu().numpy() == lp).all()


def test_without_log_probs_and_no_rows(ctx):
    x, u = logits(3, 1000, 15), uniforms(3, 11)
    tokens = torch.zeros(3, dtype=torch.int32, device="cuda")
    B.sw_sample_run(ctx, x, u, tokens)
    assert (tokens.cpu().numpy() == sample(ctx, x, u)[0]).all()
    B.sw_sample_run(ctx, x[:0], u, tokens)
    torch.cuda.synchronize()


def test_refusals(ctx):
    x, u = logits(3, 1000, 15), uniforms(3, 11)
    tokens = torch.zeros(3, dtype=torch.int32, device="cuda")
    for args in ((x.double(), u, tokens), (x.T, u, tokens), (x, u[:2], tokens), (x, u.double(), tokens), (x, u, tokens.long()), (x[0], u, tokens),
                 (x, u, tokens, u, u, u)):
        with pytest.raises(ValueError):
            B.sw_sample_run(ctx, *args)
    with pytest.raises(B.SwError) as e:
        B.sw_sample_run(ctx, torch.zeros(1, 393217, device="cuda"), u, tokens)
    assert e.value.status == B.SW_ERR_UNSUPPORTED
    with pytest.raises(B.SwError) as e:
        B.sw_sample_run(ctx, x[:1].expand(3, 1000), u, tokens)       # rows upon one another
    assert e.value.status == B.SW_ERR_INVALID_ARG
    for missing in ((None, tokens), (u, None)):
        with pytest.raises(B.SwError) as e:
            B.sw_sample_run(ctx, x, *missing)
        assert e.value.status == B.SW_ERR_INVALID_ARG
