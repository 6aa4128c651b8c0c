"""Cases of the operators around a long or a small KV cache: a cache held in 8 bits with the attention that reads it,
attention inside a sliding window with sinks, and eviction from a cache by accumulated attention weight.

A case is one call of one operator, for one layer, as a serving program makes it.  Fields:

    op        "append8": the iteration's new K/V rows into an 8-bit pool (sw_kv8_append)
              "attn8":   attention of the iteration over an 8-bit pool (sw_kv8_attn_run)
              "window":  attention of the iteration inside a window, with sinks (sw_mixed_attn_window_run)
              "weights": attention of a decode-only iteration that also adds up what weight every key got
                         (sw_decode_attn_weights_run)
              "evict":   keep `budget` keys of every (request, KV head) pair, by that weight (sw_kv_evict)
    heads     query heads / KV heads / head size
    decodes   active requests; their contexts are the quantiles of ctx_dist between ctx_lo and ctx_hi, in a random order
    chunks    prefill chunks as "prefix+tokens" joined by commas, longest first ("" = decode-only)
    window, sinks     the last `window` keys and the first `sinks` keys are attended
    budget, recent    keys kept of a pair; the newest `recent` and the first `sinks` of them always are
    lse       whether the log-sum-exp of every row is asked for as well

8-bit pool: e4m3 values [page][K|V][KV head][16 slots][head size] and one fp32 scale, a power of two, for each (page, K|V,
KV head): an element stands for its value times the scale.  A block's scale is the smallest power of two (2^-100 at least) that
brings the largest magnitude of its rows to 448 or less; it never shrinks while rows are added behind others.
"""
from __future__ import annotations

import math
import statistics

import torch

own = False

PAGE = 16
E4M3_MAX = 448.0
MIN_EXP = -100
LOGNORMAL_MEDIAN, LOGNORMAL_SIGMA = 2048.0, 1.0
MAX_BYTES, MAX_FLOPS, MAX_PLAIN = 1.7e9, 2.2e12, 2.2e9


def _case(name, op, heads, decodes, ctx_dist, ctx_lo, ctx_hi, chunks="", window=0, sinks=0, budget=0, recent=0, lse=False):
    return {"name": name, "op": op, "heads": heads, "decodes": decodes, "ctx_dist": ctx_dist, "ctx_lo": ctx_lo, "ctx_hi": ctx_hi,
            "chunks": chunks, "window": window, "sinks": sinks, "budget": budget, "recent": recent, "lse": lse}


def listed():
    llama = "32/8/128"
    return [
        # the append of the usual chat iteration: 64 users' new tokens and a chunk of somebody's prompt
        _case("append8_chat_64_c512", "append8", llama, 64, "uniform", 256, 2048, "512+512"),
        # a whole prompt written at once on an idle server
        _case("append8_prompt_8192", "append8", llama, 0, "uniform", 1, 1, "0+8192"),
        # one user alone with a medium document: latency
        _case("attn8_one_8k", "attn8", llama, 1, "uniform", 8192, 8192),
        # a full batch of mixed lengths without pending prompts: bound by the cache
        _case("attn8_mixed_128", "attn8", llama, 128, "lognormal", 128, 16384),
        # the usual chat iteration
        _case("attn8_chat_64_c512", "attn8", llama, 64, "uniform", 256, 2048, "512+512", lse=True),
        # the smallest call: a small model with four short requests and one chunk, a window that ends inside pages
        _case("window_tiny", "window", "8/2/64", 4, "uniform", 64, 256, "256+128", window=100, sinks=4, lse=True),
        # long documents being answered inside a window
        _case("window_long_16", "window", llama, 16, "uniform", 32768, 131072, window=4096, sinks=4),
        # a chunk far inside a long prompt
        _case("window_chunk_4096", "window", llama, 0, "uniform", 1, 1, "28672+4096", window=4096, sinks=4),
        # a chat batch whose keys are weighed for a later eviction
        _case("weights_chat_64", "weights", llama, 64, "uniform", 256, 2048),
        # a few long documents likewise
        _case("weights_long_4", "weights", llama, 4, "uniform", 49152, 49152),
        # one document cut to a quarter
        _case("evict_one_32k", "evict", llama, 1, "uniform", 32768, 32768, sinks=4, budget=8192, recent=512),
        # a batch of documents brought down to one size
        _case("evict_16", "evict", llama, 16, "uniform", 8192, 32768, sinks=4, budget=4096, recent=256),
    ]


def draw(rng):
    """One more call of the same ranges: the same head shapes, 1 to 256 requests of 16 to 131072 tokens, up to 3 chunks of 1 to
    8192 tokens at prefixes 0 to 98304, windows of 16 to 16384 tokens, budgets of 16 tokens to half the context."""
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))

    while True:
        op = rng.choice(["append8", "attn8", "window", "weights", "evict"])
        heads = rng.choice(["32/8/128"] * 4 + ["16/4/64", "8/2/64", "16/8/128", "8/1/128", "8/8/64"])
        kind = rng.choice(["decode", "prefill", "mixed"]) if op in ("append8", "attn8", "window") else "decode"
        n, dist, lo, hi = 0, "uniform", 1, 1
        if kind != "prefill":
            n = log_int(1, 256)
            if rng.random() < 0.3:
                dist, lo, hi = "lognormal", 128, 16384
            else:
                lo = log_int(16, 65536)
                hi = min(131072, log_int(lo, 8 * lo))
        chunks = []
        if kind != "decode":
            k = rng.choice([1, 1, 1, 2, 3])
            for _ in range(k):
                chunks.append((0 if rng.random() < 0.3 else log_int(16, 98304), log_int(16, 8192 // k)))
            chunks.sort(key=lambda c: -(2 * c[0] + c[1]) * c[1])
        case = _case("", op, heads, n, dist, lo, hi, ",".join("%d+%d" % c for c in chunks), lse=rng.random() < 0.3)
        if op == "window":
            case.update(window=log_int(16, 16384), sinks=rng.choice([0, 1, 4, 16, log_int(1, 300)]))
        if op == "evict":
            budget = log_int(16, max(32, lo // 2))
            sinks = rng.randint(0, min(8, budget // 4))
            case.update(budget=budget, sinks=sinks, recent=rng.randint(0, budget // 4), lse=False)
        if op == "append8":
            case["lse"] = False
        del case["name"]
        one, (hq, hkv, d) = work(case), _heads(case)
        full = _contexts(case)
        padded = 4 * len(full) * max(full, default=0) * hkv * d           # bytes of one padded fp32 copy of the decodes' K
        tokens = sum(full) + sum(p + c for p, c in _chunks(case))
        scores = max([c * (p + c) * hq // hkv * 4 for p, c in _chunks(case)], default=0)
        dense = sum(4 * c * (p + c) * hq * d for p, c in _chunks(case))
        if one["bytes"] > MAX_BYTES or max(one["flops"], dense) > MAX_FLOPS or max(padded / 4, scores / 2, tokens * hkv * d) > MAX_PLAIN:
            continue
        return case


# ---- sizes -----------------------------------------------------------------------------------------------------------------
def _heads(case):
    return tuple(int(x) for x in case["heads"].split("/"))


def _chunks(case):
    return [tuple(int(x) for x in c.split("+")) for c in case["chunks"].split(",") if c]


def _contexts(case):
    n, lo, hi = case["decodes"], case["ctx_lo"], case["ctx_hi"]
    at = [(i + 0.5) / n for i in range(n)]
    if case["ctx_dist"] == "lognormal":
        z = [statistics.NormalDist().inv_cdf(u) for u in at]
        return [int(min(max(math.floor(LOGNORMAL_MEDIAN * math.exp(LOGNORMAL_SIGMA * v)), lo), hi)) for v in z]
    return [int(math.floor(lo + u * (hi - lo + 1))) for u in at]


def _visible(pos, window, sinks):
    """Keys that the row at position `pos` attends."""
    return min(pos + 1, window + min(sinks, max(0, pos + 1 - window)))


def work(case):
    """Each K/V row that some row attends is read once, the iteration's q read and out written once, page tables read once;
    an append reads the new rows in 16 bits and writes them in 8; weights are read and written once; an eviction reads the
    weights and the kept rows and writes rows, weights and list.  Two multiply-adds per (query head, attended key, element)."""
    hq, hkv, d = _heads(case)
    chunks, lens, op = _chunks(case), _contexts(case), case["op"]
    rows = sum(c for _, c in chunks) + len(lens)
    io = 4 * rows * hq * d + (4 * rows * hq if case["lse"] or op == "weights" else 0)
    pages = lambda tokens: -(-tokens // PAGE)  # noqa: E731
    if op == "append8":
        blocks = len(lens) + sum(pages(p + c) - p // PAGE for p, c in chunks)
        return {"bytes": rows * 2 * hkv * d * 3 + blocks * (2 * hkv * 4 + 4), "flops": 0}
    if op == "evict":
        kept = sum(min(case["budget"], n) for n in lens)
        return {"bytes": hkv * (4 * sum(lens) + kept * (2 * 2 * d * 2 + 4 + 4)) + 4 * sum(pages(n) for n in lens), "flops": 0}
    if op == "window":
        w, s = case["window"], case["sinks"]
        seen = [_visible(n - 1, w, s) for n in lens]
        keys = sum(seen) + sum(sum(_visible(p + j, w, s) for j in range(c)) for p, c in chunks)
        cached = sum(seen) + sum(min(p + c, w + c - 1 + min(s, max(0, p + 1 - w))) for p, c in chunks)
    else:
        keys = sum(lens) + sum(c * p + c * (c + 1) // 2 for p, c in chunks)
        cached = sum(lens) + sum(p + c for p, c in chunks)
    size = cached * 2 * hkv * d * (1 if op == "attn8" else 2) + 4 * pages(cached) * (2 * hkv + 1 if op == "attn8" else 1)
    if op == "weights":
        size += 8 * hkv * sum(lens)
    return {"bytes": size + io, "flops": 4 * hq * d * keys}


# ---- inputs ----------------------------------------------------------------------------------------------------------------
def _normal(shape, gen, channel=None):
    x = torch.randn(shape, device="cuda", generator=gen)
    return (x if channel is None else x * channel).to(torch.bfloat16)


def _fill(pool, gen, channel):
    """The cached rows: N(0,1) values, the keys with a few large channels, as those of trained models have."""
    step = max(1, (1 << 26) // pool[0].numel())
    for at in range(0, pool.shape[0], step):
        part = torch.randn(pool[at:at + step].shape, device="cuda", generator=gen)
        part[:, 0] *= channel
        if pool.dtype == torch.bfloat16:
            pool[at:at + step] = part
        else:
            yield at, part


def prepare(case, seed):
    """Page tables with randomly scattered pages, the pool with its cached rows, the iteration's queries and new rows."""
    hq, hkv, d = _heads(case)
    chunks, op = _chunks(case), case["op"]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    cpu = torch.Generator()
    cpu.manual_seed(seed)
    lens = [_contexts(case)[i] for i in torch.randperm(case["decodes"], generator=cpu).tolist()]
    per = [-(-n // PAGE) for n in lens]
    per_chunk = [-(-(p + c) // PAGE) for p, c in chunks]
    per_new = [-(-min(n, case["budget"]) // PAGE) for n in lens] if op == "evict" else []
    need = sum(per) + sum(per_chunk) + sum(per_new)
    num_pages = need + 64                                                  # some free pages, as any pool has
    ids = torch.randperm(num_pages, generator=cpu)[:need].to(torch.int32)
    ints = lambda v: torch.tensor(v, dtype=torch.int32)  # noqa: E731
    starts = lambda v: torch.cat([ints([0]), torch.cumsum(ints(v), 0).to(torch.int32)])  # noqa: E731
    host = {"kv_len": ints(lens), "indptr": starts(per), "pages": ids[:sum(per)], "chunk_indptr": starts(per_chunk),
            "chunk_pages": ids[sum(per):sum(per) + sum(per_chunk)], "new_indptr": starts(per_new),
            "new_pages": ids[sum(per) + sum(per_chunk):]}
    st = {"case": case, "chunks": chunks, "longest": max(lens, default=0), "num_pages": num_pages}
    st.update({k: v.cuda() for k, v in host.items()})
    channel = torch.ones(d, device="cuda")
    channel[torch.randperm(d, generator=cpu)[:4].cuda()] = 5.0
    rows = sum(c for _, c in chunks) + len(lens)
    if op in ("append8", "attn8"):
        st["pool"] = torch.zeros(num_pages, 2, hkv, PAGE, d, device="cuda", dtype=torch.float8_e4m3fn)
        st["scales"] = torch.ones(num_pages, 2, hkv, device="cuda")
        for at, part in _fill(st["pool"], gen, channel):
            scale = _scale_for(part.abs().amax((-1, -2)))
            st["pool"][at:at + len(part)] = (part / scale[..., None, None]).to(torch.float8_e4m3fn)
            st["scales"][at:at + len(part)] = scale
    else:
        st["pool"] = torch.empty(num_pages, 2, hkv, PAGE, d, device="cuda", dtype=torch.bfloat16)
        for _ in _fill(st["pool"], gen, channel):
            pass
    if op == "append8":
        st["k_new"], st["v_new"] = _normal((rows, hkv, d), gen, channel), _normal((rows, hkv, d), gen)
    elif op != "evict":
        st["q"] = _normal((rows, hq, d), gen)
        st["out"] = torch.zeros_like(st["q"])
        st["lse"] = torch.zeros(rows, hq, device="cuda") if case["lse"] or op == "weights" else None
    if op in ("weights", "evict"):
        n, capacity = len(lens), -(-max(lens) // PAGE) * PAGE
        total = n if op == "weights" else 2 * n
        st["weight_row"] = torch.randperm(total, generator=cpu)[:n].to(torch.int32).cuda()
        left = sorted(set(range(total)) - set(st["weight_row"].tolist()))
        st["new_weight_row"] = ints(left).cuda()
        # weights of many steps: a heavy tail, and keys that never got any
        w = torch.exp(2 * torch.randn(total, hkv, capacity, device="cuda", generator=gen))
        st["weights"] = torch.where(torch.rand(w.shape, device="cuda", generator=gen) < 0.1, 0.0, w)
    if op == "evict":
        st["kept"] = torch.full((len(lens), hkv, case["budget"]), -1, device="cuda", dtype=torch.int32)
        st["new_len"] = torch.zeros(len(lens), device="cuda", dtype=torch.int32)
    if own:
        _plan(st, host)
    return st


def _plan(st, host):
    """What a program of this framework keeps: the context with its workspace, the batch's struct, scratch of the call."""
    from paper_2609_07883_b200 import binding as B
    from paper_2609_07883_b200 import workloads as W

    case, chunks = st["case"], st["chunks"]
    shape, tokens = W.AttnShape(*_heads(case)), sum(c for _, c in chunks)
    np32 = {k: v.numpy() for k, v in host.items()}
    P, C = chunks[0] if chunks else (0, 0)
    batch = W.MixedBatch(shape=shape, num_pages=st["num_pages"], prefix_len=P, chunk_len=tokens, prefill_pages=np32["chunk_pages"],
                         decode_kv_len=np32["kv_len"], decode_page_indptr=np32["indptr"], decode_pages=np32["pages"])
    if len(chunks) > 1:
        batch.chunk_prefix_lens = torch.tensor([p for p, _ in chunks], dtype=torch.int32).numpy()
        batch.chunk_lens = torch.tensor([c for _, c in chunks], dtype=torch.int32).numpy()
        batch.chunk_page_indptr = np32["chunk_indptr"]
    dev = torch.device("cuda", torch.cuda.current_device())
    st["ctx"] = B.Context(shape, st["num_pages"], max(tokens, 1), max(case["decodes"], 1), len(np32["pages"]) + len(np32["chunk_pages"]),
                          device=dev.index)
    st["batch"] = B.DeviceBatch(batch, dev)
    bytes_ = {"attn8": lambda: B.sw_kv8_scratch_bytes(st["ctx"].layout, len(np32["chunk_pages"])),
              "weights": lambda: B.sw_attn_weights_scratch_bytes(st["ctx"].layout, len(np32["pages"]))}.get(case["op"], lambda: 0)()
    st["scratch"] = torch.empty(bytes_, dtype=torch.uint8, device=dev)
    if case["op"] in ("weights", "evict"):
        st["key_weights"] = B.KeyWeights(st["weights"], st["weight_row"])
    if case["op"] == "evict":
        st["new_key_weights"] = B.KeyWeights(st["weights"], st["new_weight_row"])


# ---- one pass --------------------------------------------------------------------------------------------------------------
def run(st):
    case = st["case"]
    op = case["op"]
    if own:
        from paper_2609_07883_b200 import binding as B

        if op == "append8":
            B.sw_kv8_append(st["ctx"], st["pool"], st["scales"], st["batch"], st["k_new"], st["v_new"])
        elif op == "attn8":
            B.sw_kv8_attn_run(st["ctx"], st["pool"], st["scales"], st["batch"], st["q"], st["out"], st["lse"], st["scratch"])
        elif op == "window":
            B.sw_mixed_attn_window_run(st["ctx"], st["pool"], st["batch"], case["window"], case["sinks"], st["q"], st["out"], st["lse"])
        elif op == "weights":
            B.sw_decode_attn_weights_run(st["ctx"], st["pool"], st["batch"], st["q"], st["out"], st["lse"], st["key_weights"], st["scratch"])
        else:
            B.sw_kv_evict(st["ctx"], st["pool"], st["batch"], st["key_weights"], st["new_indptr"], st["new_pages"], st["new_key_weights"],
                          case["budget"], case["sinks"], case["recent"], st["kept"], st["new_len"])
    elif op == "append8":
        _append8(st)
    elif op == "evict":
        _evict(st)
    else:
        _attend(st)
    if op == "append8":
        return {"pool": st["pool"], "scales": st["scales"]}
    if op == "evict":
        return {"kept": st["kept"], "new_len": st["new_len"], "pool": st["pool"], "weights": st["weights"]}
    got = {"out": st["out"]}
    if st["lse"] is not None:
        got["lse"] = st["lse"]
    if op == "weights":
        got["weights"] = st["weights"]
    return got


# ---- the plain forms -------------------------------------------------------------------------------------------------------
def _scale_for(largest):
    """The smallest power of two, 2^-100 at least, that brings `largest` to 448 or less; NaN where it is not finite."""
    fraction, exponent = torch.frexp(largest.float())
    e = (exponent - 9 + (fraction > 0.875).int()).clamp(min=MIN_EXP)
    e = torch.where(largest == 0, MIN_EXP, e)
    power = ((e + 127) << 23).to(torch.int32).view(torch.float32)          # exactly 2^e, which a call of pow is not always
    return torch.where(torch.isfinite(largest), power, math.nan)


def _append8(st):
    pool, scales, chunks = st["pool"], st["scales"], st["chunks"]
    # a written block: its page, the slots [first, last) that get rows, the row of slot `first`
    page, first, last, row = [], [], [], []
    at = 0
    for j, (p, c) in enumerate(chunks):
        k = torch.arange(p // PAGE, (p + c - 1) // PAGE + 1, device="cuda")
        begin, end = (k * PAGE).clamp(min=p), (k * PAGE + PAGE).clamp(max=p + c)
        page.append(st["chunk_pages"][st["chunk_indptr"][j].long() + k])
        first.append(begin % PAGE)
        last.append(end - k * PAGE)
        row.append(at + begin - p)
        at += c
    pos = st["kv_len"].long() - 1
    page.append(st["pages"][st["indptr"][:-1].long() + pos // PAGE])
    first.append(pos % PAGE)
    last.append(pos % PAGE + 1)
    row.append(at + torch.arange(len(pos), device="cuda"))
    page, first, last, row = (torch.cat(v).long() for v in (page, first, last, row))
    slot = torch.arange(PAGE, device="cuda")
    new, old = (slot >= first[:, None]) & (slot < last[:, None]), slot < first[:, None]
    source = (row[:, None] + slot - first[:, None]).clamp(0, at + len(pos) - 1)
    x = torch.stack([st["k_new"][source], st["v_new"][source]], 1).float().transpose(2, 3)    # [block][K|V][head][slot][element]
    new, old = new[:, None, None, :, None], old[:, None, None, :, None]
    before = scales[page]
    scale = _scale_for(torch.where(new, x.abs(), 0.0).amax((-1, -2)))
    scale = torch.where(old.any(3)[..., 0], torch.maximum(scale, before), scale)              # (NaN stays NaN)
    held = pool[page].float()
    grown = (held * (before / scale)[..., None, None]).to(torch.float8_e4m3fn).float()
    value = torch.where(new, (x / scale[..., None, None]).to(torch.float8_e4m3fn).float(), torch.where(old, grown, held))
    pool[page] = value.to(torch.float8_e4m3fn)
    scales[page] = scale


def _rows_of(st, pages):
    """K and V rows of a page list [..., pages] in 32 bits: two tensors [..., head, token, element]."""
    pages = pages.long()
    x = st["pool"][pages].float()                                          # [..., page, K|V, head, slot, element]
    if "scales" in st:
        x = x * st["scales"][pages][..., None, None]
    return (x.select(-4, side).movedim(-3, -4).flatten(-3, -2) for side in (0, 1))


def _softmax(s, seen):
    """Weights and log-sum-exp of scores `s` where `seen`."""
    s = torch.where(seen, s, -math.inf)
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - top)
    total = p.sum(-1, keepdim=True)
    return p / total, (top + torch.log(total)).squeeze(-1)


def _sees(case, pos, key):
    """Whether the row at position `pos` attends position `key`."""
    seen = key <= pos
    if case["op"] == "window":
        seen = seen & ((key > pos - case["window"]) | (key < case["sinks"]))
    return seen


def _attend(st):
    case = st["case"]
    hq, hkv, d = _heads(case)
    g, scale, at = hq // hkv, 1.0 / math.sqrt(d), 0

    def store(rows, o, lse):                                               # [row][KV head][query head of its group](element)
        st["out"][rows] = o.flatten(1, 2).to(torch.bfloat16)
        if st["lse"] is not None:
            st["lse"][rows] = lse.flatten(1, 2)

    for j, (p, c) in enumerate(st["chunks"]):
        k, v = _rows_of(st, st["chunk_pages"][st["chunk_indptr"][j]:st["chunk_indptr"][j + 1]])
        q = st["q"][at:at + c].float().view(c, hkv, g, d)
        seen = _sees(case, p + torch.arange(c, device="cuda")[:, None], torch.arange(k.shape[1], device="cuda"))[:, None]
        o, lse = torch.empty_like(q), torch.empty(c, hkv, g, device="cuda")
        for h in range(hkv):                                               # (the scores of all heads at once would fill the card)
            w, lse[:, h] = _softmax(q[:, h] @ k[h].T * scale, seen)
            o[:, h] = w @ v[h]
        store(slice(at, at + c), o, lse)
        at += c
    n = case["decodes"]
    if n == 0:
        return
    length = st["kv_len"].long()
    index = torch.arange(-(-st["longest"] // PAGE), device="cuda")
    listed_ = index < (-(-length // PAGE))[:, None]
    k, v = _rows_of(st, st["pages"][torch.where(listed_, st["indptr"][:-1, None].long() + index, 0)])
    q = st["q"][at:].float().view(n, hkv, g, d)
    key = torch.arange(k.shape[2], device="cuda")
    seen = _sees(case, length[:, None] - 1, key)
    w, lse = _softmax(q @ k.transpose(-1, -2) * scale, seen[:, None, None])
    store(slice(at, at + n), w @ v, lse)
    if case["op"] == "weights":
        got, row = w.sum(2), st["weight_row"].long()
        before = torch.where((key < length[:, None] - 1)[:, None], st["weights"][row, :, :len(key)], 0.0)
        st["weights"][row, :, :len(key)] = torch.where(seen[:, None], before + got, st["weights"][row, :, :len(key)])


def _evict(st):
    case = st["case"]
    budget, sinks, recent = case["budget"], case["sinks"], case["recent"]
    length, rows, new_rows = st["kv_len"].long(), st["weight_row"].long(), st["new_weight_row"].long()
    n, cap = len(length), st["weights"].shape[-1]
    w = st["weights"][rows]                                                # [request][head][position]
    pos = torch.arange(cap, device="cuda")
    inside = pos < length[:, None]
    always = inside & ((pos < sinks) | (pos >= length[:, None] - recent) | (length[:, None] <= budget))
    rank = torch.where(always[:, None], math.inf, torch.where(inside[:, None], w, -math.inf))
    first = torch.argsort(rank, dim=-1, descending=True, stable=True)[..., :budget]      # ties: the lowest position
    keep = torch.zeros_like(rank, dtype=torch.bool).scatter_(-1, first, True) & inside[:, None]
    new_len = length.clamp(max=budget)
    order = torch.where(keep, pos, cap).sort(-1).values[..., :budget]      # kept positions, in order
    live = (torch.arange(order.shape[-1], device="cuda") < new_len[:, None])[:, None]
    order = order.clamp(max=cap - 1)
    m = order.shape[-1]
    st["kept"][..., :m] = torch.where(live, order, st["kept"][..., :m]).to(torch.int32)
    st["new_len"].copy_(new_len)
    st["weights"][new_rows, :, :m] = torch.where(live, w.gather(-1, order), st["weights"][new_rows, :, :m])
    # the rows of K and V: one (request, head, kept row) after another
    i, h, j = torch.nonzero(live.expand(order.shape), as_tuple=True)
    source = order[i, h, j]
    page = st["pages"][st["indptr"][i].long() + source // PAGE].long()
    to = st["new_pages"][st["new_indptr"][i].long() + j // PAGE].long()
    st["pool"][to, :, h, j % PAGE] = st["pool"][page, :, h, source % PAGE]


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------------
def exact(case, seed):
    """The operators' results from their definitions, one (request, KV head) pair or one block after another, in 64 bits."""
    st, op = prepare(case, seed), case["op"]
    hq, hkv, d = _heads(case)
    g = hq // hkv
    pool, indptr, pages = st["pool"], st["indptr"].tolist(), st["pages"].long()
    lens, cptr, cpages = st["kv_len"].tolist(), st["chunk_indptr"].tolist(), st["chunk_pages"].long()
    if op == "append8":
        return _exact_append8(st, lens, indptr, pages, cptr, cpages)
    if op == "evict":
        return _exact_evict(st, lens, indptr, pages)
    out = torch.zeros(st["q"].shape, device="cuda", dtype=torch.float64)
    lse = torch.zeros(st["q"].shape[:2], device="cuda", dtype=torch.float64)
    weights = st["weights"].double() if op == "weights" else None
    prompts, at = [], 0
    for j, (p, c) in enumerate(st["chunks"]):
        prompts.append((at, c, p, cpages[cptr[j]:cptr[j + 1]]))
        at += c
    prompts += [(at + i, 1, n - 1, pages[indptr[i]:indptr[i + 1]]) for i, n in enumerate(lens)]
    for i, (row, c, p, ids) in enumerate(prompts):
        position, key = torch.arange(p, p + c, device="cuda"), torch.arange(p + c, device="cuda")
        apart = position[:, None] - key[None, :]
        dead = apart < 0
        if op == "window":
            dead |= (apart >= case["window"]) & (key >= case["sinks"])[None, :]
        for h in range(hkv):
            k, v = pool[ids, 0, h].double(), pool[ids, 1, h].double()
            if op == "attn8":
                k, v = k * st["scales"][ids, 0, h].double()[:, None, None], v * st["scales"][ids, 1, h].double()[:, None, None]
            k, v = k.reshape(-1, d)[:p + c], v.reshape(-1, d)[:p + c]
            for r in range(h * g, h * g + g):
                s = (st["q"][row:row + c, r].double() @ k.T) / d ** 0.5
                s.masked_fill_(dead, -math.inf)
                lse[row:row + c, r] = torch.logsumexp(s, 1)
                s -= lse[row:row + c, r, None]
                s.exp_()
                out[row:row + c, r] = s @ v
                if weights is not None:
                    if r == h * g:
                        weights[st["weight_row"][i], h, p] = 0.0
                    weights[st["weight_row"][i], h, :p + 1] += s[0]
    got = {"out": out}
    if st["lse"] is not None:
        got["lse"] = lse
    if weights is not None:
        got["weights"] = weights
    return got


def _exact_append8(st, lens, indptr, pages, cptr, cpages):
    values, scales = st["pool"].double(), st["scales"].double()
    powers = torch.tensor([2.0 ** e for e in range(MIN_EXP, 129)], device="cuda", dtype=torch.float64)
    e4m3 = torch.tensor([(m / 8 if e == 0 else 1 + m / 8) * 2.0 ** ((e or 1) - 7) for e in range(16) for m in range(8)][:127],
                        device="cuda", dtype=torch.float64)               # every magnitude, in order of its code

    def rounded(x):
        """To the nearest magnitude, halves to the even code."""
        a = x.abs()
        up = torch.searchsorted(e4m3, a.contiguous()).clamp(max=126)
        down = (up - 1).clamp(min=0)
        to_up, to_down = e4m3[up] - a, a - e4m3[down]
        take = torch.where((to_down < to_up) | ((to_down == to_up) & (down % 2 == 0)), down, up)
        return torch.copysign(e4m3[take], x)

    def write(page, first, k, v):
        """Rows k, v [block][slot][head][element] behind the first `first` slots of the pages."""
        for side, x in ((0, k.double()), (1, v.double())):
            x = x.transpose(1, 2)                                          # [block][head][slot][element]
            largest = x.abs().amax((-1, -2))
            scale = powers[(largest[..., None] > E4M3_MAX * powers).sum(-1)]
            if first:
                scale = torch.maximum(scale, scales[page, side])
                values[page, side, :, :first] = rounded(values[page, side, :, :first] * (scales[page, side] / scale)[..., None, None])
            values[page, side, :, first:first + x.shape[2]] = rounded(x / scale[..., None, None])
            scales[page, side] = scale

    at = 0
    for j, (p, c) in enumerate(st["chunks"]):
        ids, done = cpages[cptr[j]:cptr[j + 1]], 0
        while done < c:
            slot = (p + done) % PAGE
            blocks = 1 if slot or c - done < PAGE else (c - done) // PAGE
            m = blocks * PAGE if blocks > 1 else min(PAGE - slot, c - done)
            rows = slice(at + done, at + done + m)
            shape = (blocks, m // blocks) + tuple(st["k_new"].shape[1:])
            write(ids[(p + done) // PAGE:(p + done) // PAGE + blocks], slot, st["k_new"][rows].reshape(shape), st["v_new"][rows].reshape(shape))
            done += m
        at += c
    for i, n in enumerate(lens):
        write(pages[indptr[i] + (n - 1) // PAGE][None], (n - 1) % PAGE, st["k_new"][at + i][None, None], st["v_new"][at + i][None, None])
    return {"pool": values, "scales": scales}


def _exact_evict(st, lens, indptr, pages):
    case, pool, kept, weights = st["case"], st["pool"].clone(), st["kept"].clone(), st["weights"].double()
    to, to_ptr = st["new_pages"].long(), st["new_indptr"].tolist()
    for i, n in enumerate(lens):
        m = min(n, case["budget"])
        for h in range(kept.shape[1]):
            w = st["weights"][st["weight_row"][i], h, :n].double()
            if n > case["budget"]:
                w = w.clone()
                w[:case["sinks"]] = math.inf
                w[n - case["recent"]:] = math.inf
                order = sorted(range(n), key=lambda t, v=w.tolist(): (-v[t], t))[:m]
            else:
                order = range(n)
            keep = torch.tensor(sorted(order), device="cuda")
            kept[i, h, :m] = keep.to(torch.int32)
            weights[st["new_weight_row"][i], h, :m] = st["weights"][st["weight_row"][i], h, keep].double()
            source = st["pool"][pages[indptr[i]:indptr[i + 1]], :, h]      # [page][K|V][slot][element]
            rows = source[keep // PAGE, :, keep % PAGE]
            j = torch.arange(m, device="cuda")
            pool[to[to_ptr[i] + j // PAGE], :, h, j % PAGE] = rows
    return {"kept": kept, "new_len": torch.tensor([min(n, case["budget"]) for n in lens], device="cuda", dtype=torch.int32),
            "pool": pool, "weights": weights}
