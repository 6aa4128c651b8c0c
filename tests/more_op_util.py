"""Plain 64-bit forms of the operators in front of, beside and behind the iteration's attention (rotary positions, cross attention, sampling).

Tolerances are sums of the roundings that a result goes through, taken at their largest.  Cross attention: as listed in op_util.  Rotations:
  bf16 output                   2^-8 |o|                       (half a step of bf16, relative)
  fraction of a turn in fp32    2^-26 turns                    (half a step at 1/2: 2 pi 2^-26 < 2^-23 radians)
  sine, cosine, times magnitude 2^-23                          (two units in the last place each, then half of one)
  two products and their sum    3 2^-24                        together less than 2^-21 (|a| + |b|) magnitude
  position times turns          2^-53 position turns 2 pi      (half a step of fp64, relative; likewise the table's own rounding)
"""
from __future__ import annotations

import math
from fractions import Fraction

import numpy as np
import torch

from tests import op_util as U

PAGE = 16


# ---- cross attention ---------------------------------------------------------------------------------------------------------
def cross_attention(batch, pool, q, scale=None):
    """Outputs, log-sum-exps and tolerances in float64; ``pool`` float64 [pages][2][heads][16][D]."""
    sh = batch.shape
    g, D = sh.group, sh.head_dim
    scale = scale or 1 / math.sqrt(D)
    q = q.double().view(-1, sh.num_kv_heads, g, D)
    out, tol = torch.zeros_like(q), torch.full_like(q, 0.0)
    lse = torch.full(q.shape[:3], -math.inf, dtype=torch.float64, device=q.device)
    lse_tol = torch.zeros_like(lse)
    entries = [(row, C, P, pages) for P, C, row, pages in batch.chunks()]
    for i in range(batch.num_decode):
        entries.append((batch.chunk_len + i, 1, int(batch.decode_kv_len[i]), batch.decode_pages[batch.decode_page_indptr[i]:batch.decode_page_indptr[i + 1]]))
    for row, count, n, pages in entries:
        if n <= 0:
            continue
        ids = torch.from_numpy(np.asarray(pages[:-(-n // PAGE)], dtype=np.int64)).to(q.device)
        for h in range(sh.num_kv_heads):
            k, v = (pool[ids, side, h].reshape(-1, D)[:n].double() for side in (0, 1))
            x = q[row:row + count, h]
            s = x @ k.T * scale
            total = torch.logsumexp(s, -1)
            p = torch.exp(s - total[..., None])
            o, mass = p @ v, p @ v.abs()
            s_err = (D + 8) * 2.0 ** -24 * (x.abs() @ k.abs().T * scale).amax(-1)
            out[row:row + count, h], lse[row:row + count, h] = o, total
            rel = 2.0 ** -8 + 1.5e-4 + max(5e-4, n * 2.0 ** -24) + 2 * s_err
            tol[row:row + count, h] = 2.0 ** -8 * o.abs() + rel[..., None] * mass + 1e-30
            lse_tol[row:row + count, h] = s_err + 7.5e-5 + max(5e-4, n * 2.0 ** -24) + 2.0 ** -22 * total.abs()
    shape = (q.shape[0], sh.num_q_heads, D)
    return out.view(shape), lse.view(shape[:2]), tol.view(shape), lse_tol.view(shape[:2])


class CrossCase(U.Case):
    """A batch whose page lists end with the keys: ``chunks`` are (keys, rows).  What lies behind the keys in their last pages is NaN."""

    def __init__(self, heads, lens, chunks=(), seed=1):
        super().__init__(heads, lens, [(max(p, 1), c) for p, c in chunks], seed)
        b = self.batch
        lists = [pages[:-(-p // PAGE)] for (p, _), (_, _, _, pages) in zip(chunks, b.chunks())]
        b.prefill_pages = np.concatenate(lists).astype(np.int32) if lists else b.prefill_pages
        b.prefix_len = chunks[0][0] if chunks else 0
        if len(chunks) > 1:
            b.chunk_prefix_lens = np.array([p for p, _ in chunks], dtype=np.int32)
            b.chunk_page_indptr = np.concatenate([[0], np.cumsum([len(x) for x in lists])]).astype(np.int32)
        for n, pages in [(p, x) for (p, _), x in zip(chunks, lists)] + [
                (int(b.decode_kv_len[i]), b.decode_pages[b.decode_page_indptr[i]:b.decode_page_indptr[i + 1]]) for i in range(b.num_decode)]:
            if n % PAGE:
                self.pool[int(pages[n // PAGE]), :, :, n % PAGE:] = math.nan
        self.renew()

    def check_cross(self, rows=slice(None)):
        torch.cuda.synchronize()
        out, lse, tol, lse_tol = cross_attention(self.batch, self.pool, self.q)
        err = (self.out.double() - out).abs()[rows]
        assert bool((err <= tol[rows]).all()), f"output off by {float((err / tol[rows].clamp(min=1e-30)).max()):.3g} of its tolerance"
        none = torch.isinf(lse)
        assert torch.equal(torch.isinf(self.lse)[rows], none[rows]) and bool((self.lse[none] < 0).all())
        err = torch.where(none, 0.0, (self.lse.double() - lse).abs())[rows]
        assert bool((err <= lse_tol[rows]).all()), "lse"


# ---- rotary positions ----------------------------------------------------------------------------------------------------------
def batch_positions(batch):
    pos = [np.arange(P, P + C) for P, C, _, _ in batch.chunks()] + [batch.decode_kv_len.astype(np.int64) - 1]
    return np.concatenate(pos).astype(np.int64)


def rotate(x, pos, turns, interleaved, magnitude):
    """Rotated rows and their tolerances in float64; x [rows][heads][D] bf16, pos int64 [rows], turns float64 [pairs] (numpy)."""
    half = len(turns)
    t = pos.astype(np.longdouble)[:, None] * turns.astype(np.longdouble)[None]
    angle = torch.from_numpy((2 * np.pi * (t - np.rint(t)).astype(np.float64))).to(x.device)[:, None]
    slack = torch.from_numpy(np.abs(pos)[:, None] * turns[None] * 2.0 ** -52 * 2 * np.pi).to(x.device)[:, None]
    y = x.double().clone()
    tol = torch.zeros_like(y)
    a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    xa, xb = x[..., a].double(), x[..., b].double()
    y[..., a] = magnitude * (xa * torch.cos(angle) - xb * torch.sin(angle))
    y[..., b] = magnitude * (xb * torch.cos(angle) + xa * torch.sin(angle))
    for part in (a, b):
        tol[..., part] = 2.0 ** -8 * y[..., part].abs() + (2.0 ** -21 + slack) * (xa.abs() + xb.abs()) * abs(magnitude)
    return y, tol


# ---- sampling --------------------------------------------------------------------------------------------------------------------
UNIT = 2.0 ** 44


def draw(x, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """Token, log-probability and the kept indices of one row; x float64 (numpy).  Weights are whole units, as the header says, so sums are exact."""
    x = np.where(np.isnan(x), -np.inf, x)
    top = x.max()
    if top == -np.inf:
        return -1, -math.inf, np.zeros(0, dtype=np.int64)
    best = int(np.argmax(x))
    if not temperature > 0:
        return best, 0.0, np.array([best])
    with np.errstate(invalid="ignore", over="ignore", under="ignore"):
        w = np.where(x == top, 1.0, np.where(x == -np.inf, 0.0, np.exp((x - top) / temperature) if top < np.inf else 0.0))
    w = np.rint(w * UNIT).astype(np.int64)
    order = np.argsort(-x, kind="stable")
    live = x[order] > -np.inf
    order = order[live]
    if 0 < top_k < len(x):
        order = order[:top_k]
    if top_p < 1:
        sums = np.cumsum(w[order])
        order = order[: 1 + int(np.sum(sums[:-1] < math.ceil(Fraction(max(top_p, 0.0)) * int(sums[-1]))))]
    if min_p > 0:
        order = order[w[order] >= min(min_p, 1.0) * UNIT]
    kept = np.sort(order)
    sums = np.cumsum(w[kept])
    drawn = min(math.floor(Fraction(min(max(u, 0.0), 1.0)) * int(sums[-1])) if u == u else 0, int(sums[-1]) - 1)
    at = int(np.searchsorted(sums, drawn, side="right"))
    return int(kept[at]), math.log(int(w[kept[at]]) / int(sums[-1])), kept
