"""Plain 64-bit forms of the operators beside the plain iteration (window with sinks, 8-bit pool, weights of keys, eviction), and the batches
their tests run.  Everything here is elementary torch in float64, on whatever device its inputs are.

Tolerances are sums of the roundings that a result goes through, taken at their largest:
  bf16 output                    2^-8 |o|                    (half a step of bf16, relative)
  softmax weights as bf16        2^-8 sum p |v|              (the products take them in 16 bits; their sum l is kept in 32)
  2^x on the FMA pipe            7.5e-5 of a weight, numerator and denominator: 1.5e-4 sum p |v|
  a score's products and sum     D additions of fp32: D 2^-24 sum |q k| scale, an exponent's error, so relative in p; twice (p and l)
  weights as f16 (8-bit pools)   times 2^7 (chunks) or 2^15 (decodes) in a format whose smallest step is 2^-24: half of that, 2^-32 of the row's
                                 largest weight at most, for each key: 2^-32 sum |v| (`floor`)
  sums of p and of p v           N additions of fp32, pairwise or in tiles of 16 or 128: N 2^-24 at most with N <= 8192 here: 5e-4
"""
from __future__ import annotations

import math

import numpy as np
import torch

from paper_2609_07883_b200 import binding as B
from paper_2609_07883_b200 import workloads as W

PAGE = 16


# ---- e4m3 ------------------------------------------------------------------------------------------------------------------
E4M3 = torch.tensor([(m / 8 if e == 0 else 1 + m / 8) * 2.0 ** ((e or 1) - 7) for e in range(16) for m in range(8)][:127], dtype=torch.float64)


def e4m3_codes(x):
    """Nearest e4m3 code (halves to even) of float64 values of magnitude 448 or less; NaN: 0x7f."""
    table = E4M3.to(x.device)
    a = torch.nan_to_num(x.abs(), nan=0.0).contiguous()
    up = torch.searchsorted(table, a).clamp(max=126)
    down = (up - 1).clamp(min=0)
    du, dd = table[up] - a, a - table[down]
    code = torch.where((dd < du) | ((dd == du) & (down % 2 == 0)), down, up)
    code = code + 128 * torch.signbit(x)
    return torch.where(torch.isnan(x), 0x7F, code).to(torch.uint8)


def e4m3_values(codes):
    table = torch.cat([E4M3, torch.tensor([math.nan], dtype=torch.float64)]).to(codes.device)
    v = table[(codes & 127).long()]
    return torch.where(codes >= 128, -v, v)


def scale_of(largest: float) -> float:
    if not math.isfinite(largest):
        return math.nan
    e = -100
    while largest > 448 * 2.0 ** e:
        e += 1
    return 2.0 ** e


def append8(codes, scales, entries, k_new, v_new):
    """Rows [first row, count) of an entry (position, page list) one after another into ``codes`` (uint8) and ``scales``, in place."""
    for row0, count, pos0, pages in entries:
        done = 0
        while done < count:
            pos = pos0 + done
            first, m = pos % PAGE, min(PAGE - pos % PAGE, count - done)
            page = int(pages[pos // PAGE])
            for side, src in ((0, k_new), (1, v_new)):
                for h in range(src.shape[1]):
                    x = src[row0 + done:row0 + done + m, h].double()
                    s = scale_of(float("nan") if not bool(torch.isfinite(x).all()) else float(x.abs().max()))
                    before = float(scales[page, side, h])
                    if first:
                        s = math.nan if math.isnan(s) or math.isnan(before) else max(s, before)
                        if s != before:
                            codes[page, side, h, :first] = e4m3_codes(e4m3_values(codes[page, side, h, :first]) * (before / s))
                    codes[page, side, h, first:first + m] = e4m3_codes(x / s)
                    scales[page, side, h] = s
            done += m


# ---- attention ---------------------------------------------------------------------------------------------------------------
def entries_of(batch):
    """(first row, rows, position of the first row, page list) of every chunk, then of every decode request."""
    out = [(row, C, P, pages) for P, C, row, pages in batch.chunks()]
    for i in range(batch.num_decode):
        n = int(batch.decode_kv_len[i])
        out.append((batch.chunk_len + i, 1 if n > 0 else 0, n - 1, batch.decode_pages[batch.decode_page_indptr[i]:batch.decode_page_indptr[i + 1]]))
    return out


def attention(batch, pool, q, window=None, sinks=0, scale=None, floor=0.0):
    """Outputs, log-sum-exps and their tolerances in float64; ``pool`` float64 [pages][2][heads][16][D].  Keys nobody attends may be NaN."""
    sh = batch.shape
    g, D = sh.group, sh.head_dim
    scale = scale or 1 / math.sqrt(D)
    q = q.double().view(-1, sh.num_kv_heads, g, D)
    out, tol = torch.zeros_like(q), torch.zeros_like(q)
    lse, lse_tol = torch.zeros(q.shape[:3], dtype=torch.float64, device=q.device), torch.zeros(q.shape[:3], dtype=torch.float64, device=q.device)
    weights = {}
    for e, (row, count, pos0, pages) in enumerate(entries_of(batch)):
        if count == 0:
            continue
        n = pos0 + count
        pos, key = torch.arange(pos0, n, device=q.device)[:, None], torch.arange(n, device=q.device)[None]
        seen = key <= pos
        if window is not None:
            seen &= (key > pos - window) | (key < sinks)
        used = seen.any(0)
        ids = torch.from_numpy(np.asarray(pages[:-(-n // PAGE)], dtype=np.int64)).to(q.device)
        ids = torch.where(torch.nn.functional.pad(used, (0, len(ids) * PAGE - n)).view(-1, PAGE).any(1), ids, 0)   # (others are not looked at)
        for h in range(sh.num_kv_heads):
            k, v = (pool[ids, side, h].reshape(-1, D)[:n] for side in (0, 1))
            k, v = (torch.where(used[:, None], t, 0.0) for t in (k, v))
            x = q[row:row + count, h]
            s = torch.where(seen[:, None], x @ k.T * scale, -math.inf)
            total = torch.logsumexp(s, -1)
            p = torch.exp(s - total[..., None])
            o, mass = p @ v, p @ v.abs()
            s_err = (D + 8) * 2.0 ** -24 * torch.where(seen[:, None], x.abs() @ k.abs().T * scale, 0.0).amax(-1)
            out[row:row + count, h], lse[row:row + count, h] = o, total
            rel = 2.0 ** -8 + 1.5e-4 + 5e-4 + 2 * s_err
            least = floor * seen.double() @ v.abs()
            tol[row:row + count, h] = 2.0 ** -8 * o.abs() + rel[..., None] * mass + least[:, None] + 1e-30
            lse_tol[row:row + count, h] = s_err + 7.5e-5 + 5e-4 + 2.0 ** -22 * total.abs()
            if e >= len(batch.chunks()):
                weights[e - len(batch.chunks()), h] = (p[0].sum(0), seen[0], (2 * s_err[0].max() + 1e-5).item())
    shape = (q.shape[0], sh.num_q_heads, D)
    return out.view(shape), lse.view(shape[:2]), tol.view(shape), lse_tol.view(shape[:2]), weights


# ---- a batch on the device -----------------------------------------------------------------------------------------------------
class Case:
    """One iteration's batch, tensors and context.  Pools hold N(0,1) values; q, k_new, v_new likewise."""

    def __init__(self, heads, lens, chunks=(), seed=1, spare=40):
        hq, hkv, d = heads
        rng = np.random.default_rng(seed)
        self.shape = W.AttnShape(hq, hkv, d)
        need = sum(-(-int(n) // PAGE) for n in lens) + sum(-(-(p + c) // PAGE) for p, c in chunks)
        self.pages = need + spare
        if len(chunks) <= 1:
            P, C = chunks[0] if chunks else (0, 0)
            self.batch = W.make_batch(self.shape, self.pages, lens, P, C, rng)
        else:
            self.batch = W.make_multi_batch(self.shape, self.pages, lens, chunks, rng)
        self.dev = torch.device("cuda", 0)
        gen = torch.Generator(device=self.dev)
        gen.manual_seed(seed)
        rows = self.batch.num_rows
        normal = lambda *s: torch.randn(*s, device=self.dev, generator=gen).to(torch.bfloat16)  # noqa: E731
        self.q, self.k_new, self.v_new = normal(rows, hq, d), normal(rows, hkv, d), normal(rows, hkv, d)
        self.pool = normal(self.pages, 2, hkv, PAGE, d)
        self.out = torch.full_like(self.q, math.nan)
        self.lse = torch.full((rows, hq), math.nan, device=self.dev)
        self.ctx = B.Context(self.shape, self.pages, max(self.batch.chunk_len, 1), max(self.batch.num_decode, 1), 16)
        self.renew()

    def renew(self):
        """The device copy of the batch, after its host arrays were changed."""
        self.db = B.DeviceBatch(self.batch, self.dev)

    def free_pages(self):
        used = set(self.batch.decode_pages.tolist()) | set(self.batch.prefill_pages.tolist())
        return [i for i in range(self.pages) if i not in used]

    def ok(self):
        assert B.sw_check_status(self.ctx, raise_on_error=False) == (0, 0)

    def check(self, pool64, window=None, sinks=0, rows=None, floor=0.0):
        """out and lse against the plain form over ``pool64``."""
        torch.cuda.synchronize()
        out, lse, tol, lse_tol, weights = attention(self.batch, pool64, self.q, window, sinks, floor=floor)
        live = torch.ones(out.shape[0], dtype=torch.bool, device=self.dev)
        for row, count, _, _ in entries_of(self.batch):
            if count == 0:
                live[row] = False
        if rows is not None:
            keep = torch.zeros_like(live)
            keep[rows] = True
            live &= keep
        err = (self.out.double() - out).abs()[live]
        assert bool((err <= tol[live]).all()), f"output off by {float((err / tol[live]).max()):.3g} of its tolerance"
        err = (self.lse.double() - lse).abs()[live]
        assert bool((err <= lse_tol[live]).all()), f"lse off by {float((err / lse_tol[live]).max()):.3g} of its tolerance"
        return weights


def quantise(pool):
    """A pool in 8 bits, each block at its own scale: (codes as float8, scales)."""
    x = pool.double()
    top = x.abs().amax((-1, -2))
    e = torch.ceil(torch.log2(torch.clamp(top, min=1e-30) / 448))
    e = torch.where(top > 448 * 2.0 ** e, e + 1, torch.where(top <= 448 * 2.0 ** (e - 1), e - 1, e)).clamp(min=-100)
    s = torch.tensor([2.0 ** i for i in range(-100, 128)], dtype=torch.float64, device=pool.device)[(e + 100).long()]
    return e4m3_codes(x / s[..., None, None]).view(torch.float8_e4m3fn), s.float()


def dequantise(codes, scales):
    return e4m3_values(codes.view(torch.uint8)) * scales.double()[..., None, None]
