"""Cases of the operators in front of, beside and behind the attention of a serving iteration: rotary positions (with the append of the rotated
keys), cross attention to the cached states of an encoder, and the draw of the next tokens from logits.

A case is one call of one operator, for one layer, as a serving program makes it.  Fields:

    op        "rope":   queries and new keys rotated by their positions; the keys, with their values, go into the paged pool
                        (sw_rope_append) or, where `append` is false, to a tensor of their own (sw_rope_run)
              "cross":  every row attends all cached keys of its sequence's encoder (sw_cross_attn_run)
              "sample": one token a row, from logits and a given uniform number (sw_sample_run)
    heads     query heads / KV heads / head size
    decodes   active requests; their cached lengths (cross: keys) are the quantiles of ctx_dist between ctx_lo and ctx_hi, in a random order
    chunks    prefill chunks as "prefix+tokens" joined by commas ("" = decode-only); cross: "keys+tokens"
    rope: rotary  elements of a head that are rotated
          layout  "half": element i with element i + rotary / 2; "interleaved": element 2 i with element 2 i + 1
          scaling "plain", "bands", "ramp" (below), with `factor` and `original`, the length that the frequencies were trained for
          packed  q, k and v are slices of one projection's rows
          shift   where not 0, positions are given: those of the batch plus this (a cache that keys were evicted from)
    cross: lse    whether the log-sum-exp of every row is asked for as well
    sample: rows, vocab, dtype ("f32", "bf16", "f16") of the logits; temperature, top_k, top_p, min_p: one number for all rows, or "mixed": a
            batch of users with settings of their own

Rotary positions: pair i of a head turns by position * w_i radians.  "plain": w_i = base^(-2 i / rotary).  "bands": wavelengths 2 pi / w_i above
original / low are stretched by `factor`, those below original / high are kept, and between them the frequency goes over linearly in
original / wavelength.  "ramp": pairs go over from kept to stretched linearly in i, between the pairs that turn `high` and `low` times over
`original` positions (these two rounded outward), and the result is multiplied by 0.1 ln(factor) + 1.

Sampling: weights are exp((x - max) / temperature); a temperature of 0 takes the largest logit.  Of the logits in falling order (equal ones by
index), top_k keeps the first k; of their total weight, top_p keeps those in front of which less than the share p lies; min_p keeps those whose
weight is at least min_p of the largest.  The token is the first, by index, up to which the kept weights sum to more than the uniform number
times their total.  Its log-probability is that of this draw.
"""
from __future__ import annotations

import math
import statistics

import torch

own = False

PAGE = 16
BASE = 500000.0
LOW, HIGH = {"bands": 1.0, "ramp": 1.0}, {"bands": 4.0, "ramp": 32.0}
LOGNORMAL_MEDIAN, LOGNORMAL_SIGMA = 2048.0, 1.0
MAX_BYTES, MAX_FLOPS = {"rope": 2.0e8, "cross": 3.9e8}, 5.4e11
MAX_CACHED, MAX_SCORES, MAX_LOGITS = 1.9e8, 1.3e8, 256 * 128256          # elements, which bound the plain forms


def _rope(name, heads, decodes, ctx_lo, ctx_hi, chunks, rotary, layout="half", scaling="plain", factor=1.0, original=8192, append=True, packed=False, shift=0):
    return {"name": name, "op": "rope", "heads": heads, "decodes": decodes, "ctx_dist": "uniform", "ctx_lo": ctx_lo, "ctx_hi": ctx_hi, "chunks": chunks,
            "rotary": rotary, "layout": layout, "scaling": scaling, "factor": factor, "original": original, "append": append, "packed": packed,
            "shift": shift}


def _cross(name, heads, decodes, ctx_lo, ctx_hi, chunks="", ctx_dist="uniform", lse=False):
    return {"name": name, "op": "cross", "heads": heads, "decodes": decodes, "ctx_dist": ctx_dist, "ctx_lo": ctx_lo, "ctx_hi": ctx_hi, "chunks": chunks,
            "lse": lse}


def _sample(name, rows, vocab, dtype, temperature, top_k=0, top_p=1.0, min_p=0.0):
    return {"name": name, "op": "sample", "rows": rows, "vocab": vocab, "dtype": dtype, "temperature": temperature, "top_k": top_k, "top_p": top_p,
            "min_p": min_p}


def listed():
    llama = "32/8/128"
    return [
        # one user alone, whose long document has been evicted down to 4096 keys: latency, and a far position
        _rope("rope_one_far", llama, 1, 4096, 4096, "", 128, scaling="bands", factor=8.0, packed=True, shift=122880),
        # the usual chat iteration, from the rows of one projection
        _rope("rope_chat_64_c512", llama, 64, 256, 2048, "512+512", 128, scaling="bands", factor=8.0, packed=True),
        # a whole prompt at once on an idle server, half of each head rotated, neighbouring elements paired
        _rope("rope_prompt_8192", llama, 0, 1, 1, "0+8192", 64, layout="interleaved"),
        # in front of an iteration that appends by itself: an odd chunk far inside a long prompt beside a batch
        _rope("rope_run_d64", "16/4/64", 128, 500, 3000, "30011+1777", 64, scaling="ramp", factor=4.0, append=False),
        # the smallest call: a small model with four short sources and one chunk
        _cross("cross_tiny", "8/2/64", 4, 64, 256, "256+128", lse=True),
        # transcriptions under way: one token each against 30 seconds of speech
        _cross("cross_speech_64", "16/16/64", 64, 1500, 1500),
        # three prompts that begin beside a batch, sources of unlike lengths
        _cross("cross_prompts_32", llama, 32, 300, 4000, "4111+448,1500+224,333+77"),
        # a long answer scored against a long document in one go
        _cross("cross_document", llama, 0, 1, 1, "16384+2048"),
        # one user alone, usual settings: latency
        _sample("sample_one", 1, 128256, "f32", 0.7, top_k=50, top_p=0.9),
        # a chat batch, everybody's own settings
        _sample("sample_mixed_64", 64, 128256, "bf16", "mixed", top_k="mixed", top_p="mixed", min_p="mixed"),
        # a large batch cut by probability alone: bound by the logits
        _sample("sample_top_p_256", 256, 128256, "f32", 1.0, top_p=0.95),
        # a smaller vocabulary of an odd size, nothing cut off
        _sample("sample_plain_128", 128, 32003, "f32", 0.8),
    ]


def draw(rng):
    """One more call of the same ranges: 1 to 256 requests of 16 to 16384 cached tokens (positions to 150000), up to 3 chunks of 1 to 8192 tokens
    in all; sources of 16 to 32768 keys; 1 to 256 rows of 1000 to 262144 logits, with every setting."""
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))

    while True:
        op = rng.choice(["rope", "cross", "sample"])
        if op == "sample":
            case = _sample("", log_int(1, 256), rng.choice([log_int(1000, 262144), 32000, 50257, 128256, 151936]), rng.choice(["f32", "f32", "bf16", "f16"]),
                           rng.choice([0.0, 0.3, 0.7, 1.0, 1.5, "mixed", "mixed"]), rng.choice([0, 0, 1, 20, 50, log_int(1, 5000), "mixed"]),
                           rng.choice([1.0, 1.0, 0.5, 0.9, 0.95, 0.99, "mixed"]), rng.choice([0.0, 0.0, 0.05, 0.3, "mixed"]))
            del case["name"]
            if case["rows"] * case["vocab"] <= MAX_LOGITS:
                return case
            continue
        heads = rng.choice(["32/8/128"] * 4 + ["16/4/64", "8/2/64", "16/8/128", "8/1/128", "16/16/64"])
        kind = rng.choice(["decode", "prefill", "mixed"])
        n, dist, lo, hi = 0, "uniform", 1, 1
        if kind != "prefill":
            n = log_int(1, 256)
            if op == "cross" and rng.random() < 0.3:
                dist, lo, hi = "lognormal", 128, 16384
            else:
                lo = log_int(16, 8192)
                hi = min(16384, log_int(lo, 8 * lo))
        chunks = []
        if kind != "decode":
            k = rng.choice([1, 1, 1, 2, 3])
            for _ in range(k):
                if op == "rope":
                    chunks.append((0 if rng.random() < 0.3 else log_int(16, 16384), log_int(1, 8192 // k)))
                else:
                    chunks.append((log_int(16, 32768), log_int(1, 2048 // k)))
            chunks.sort(key=lambda c: -c[0] * c[1] if op == "cross" else -(2 * c[0] + c[1]) * c[1])
        text = ",".join("%d+%d" % c for c in chunks)
        if op == "rope":
            d = int(heads.split("/")[2])
            case = _rope("", heads, n, lo, hi, text, rng.choice([d, d, d // 2, d // 4, 3 * d // 4]), rng.choice(["half", "half", "interleaved"]),
                         *rng.choice([("plain", 1.0, 8192), ("bands", 8.0, 8192), ("ramp", 4.0, 32768), ("ramp", 16.0, 4096)]),
                         append=rng.random() < 0.6, packed=rng.random() < 0.5, shift=rng.choice([0, 0, log_int(1, 131072)]))
        else:
            case = _cross("", heads, n, lo, hi, text, dist, lse=rng.random() < 0.3)
        del case["name"]
        (hq, hkv, d), full = _heads(case), _contexts(case)
        one = work(case)
        cached = (sum(full) + sum(p + (c if op == "rope" else 0) for p, c in _chunks(case))) * 2 * hkv * d
        padded = 2 * len(full) * max(full, default=0) * hkv * d if op == "cross" else 0
        scores = max([c * p * hq // hkv for p, c in _chunks(case)], default=0) if op == "cross" else 0
        if one["bytes"] <= MAX_BYTES[op] and one["flops"] <= MAX_FLOPS and max(cached, padded) <= MAX_CACHED and scores <= MAX_SCORES:
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


def work(case):
    """rope: every row's q, k (with an append also v) read once and written once, six operations a pair.  cross: each cached K/V row that some row
    attends read once, q read and out written once, page tables once; two multiply-adds per (query head, attended key, element).  sample: each
    logit read once; a subtraction, a product, an exponential and a sum of it."""
    if case["op"] == "sample":
        size = case["rows"] * case["vocab"]
        return {"bytes": size * (4 if case["dtype"] == "f32" else 2) + case["rows"] * 28, "flops": 4 * size}
    hq, hkv, d = _heads(case)
    chunks, lens = _chunks(case), _contexts(case)
    rows = sum(c for _, c in chunks) + len(lens)
    pages = lambda tokens: -(-tokens // PAGE)  # noqa: E731
    if case["op"] == "rope":
        ids = len(lens) + sum(pages(p + c) - p // PAGE for p, c in chunks) if case["append"] else 0
        return {"bytes": rows * (hq + (2 if case["append"] else 1) * hkv) * d * 4 + 4 * ids, "flops": 6 * rows * (hq + hkv) * case["rotary"] // 2}
    keys, cached = sum(lens) + sum(p * c for p, c in chunks), sum(lens) + sum(p for p, c in chunks)
    return {"bytes": cached * 2 * hkv * d * 2 + 4 * pages(cached) + 4 * rows * hq * d + (4 * rows * hq if case["lse"] else 0), "flops": 4 * hq * d * keys}


# ---- inputs ----------------------------------------------------------------------------------------------------------------
def _frequencies(case):
    """Radians per position of every pair, and the factor of the result."""
    half, base = case["rotary"] // 2, BASE
    w = [base ** (-i / half) for i in range(half)]
    low, high, f, length = LOW.get(case["scaling"]), HIGH.get(case["scaling"]), case["factor"], case["original"]
    if case["scaling"] == "bands":
        turns = [length * x / (2 * math.pi) for x in w]
        part = [min(max((t - low) / (high - low), 0.0), 1.0) for t in turns]
        return [x * (s + (1 - s) / f) for x, s in zip(w, part)], 1.0
    if case["scaling"] == "ramp":
        pair = lambda t: half * math.log(length / (t * 2 * math.pi)) / math.log(base)  # noqa: E731
        first, last = max(math.floor(pair(high)), 0), min(math.ceil(pair(low)), 2 * half - 1)
        part = [1 - min(max((i - first) / max(last - first, 1e-3), 0.0), 1.0) for i in range(half)]
        return [x * (s + (1 - s) / f) for x, s in zip(w, part)], 0.1 * math.log(f) + 1
    return w, 1.0


def _normal(shape, gen, channel=None):
    x = torch.randn(shape, device="cuda", generator=gen)
    return (x if channel is None else x * channel).to(torch.bfloat16)


def prepare(case, seed):
    """Page tables with randomly scattered pages, the pool with its cached rows, the iteration's rows; or logits with settings and random numbers."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    cpu = torch.Generator()
    cpu.manual_seed(seed)
    if case["op"] == "sample":
        return _prepare_sample(case, gen, cpu)
    hq, hkv, d = _heads(case)
    chunks, op = _chunks(case), case["op"]
    lens = [_contexts(case)[i] for i in torch.randperm(case["decodes"], generator=cpu).tolist()]
    per = [-(-n // PAGE) for n in lens]
    per_chunk = [-(-(p + (c if op == "rope" else 0)) // PAGE) for p, c in chunks]
    need = sum(per) + sum(per_chunk)
    num_pages = need + 64                                                  # some free pages, as any pool has
    ids = torch.randperm(num_pages, generator=cpu)[:need].to(torch.int32)
    ints = lambda v: torch.tensor(v, dtype=torch.int32)  # noqa: E731
    starts = lambda v: torch.cat([ints([0]), torch.cumsum(ints(v), 0).to(torch.int32)])  # noqa: E731
    host = {"kv_len": ints(lens), "indptr": starts(per), "pages": ids[:sum(per)], "chunk_indptr": starts(per_chunk), "chunk_pages": ids[sum(per):]}
    st = {"case": case, "chunks": chunks, "longest": max(lens, default=0), "num_pages": num_pages}
    st.update({k: v.cuda() for k, v in host.items()})
    channel = torch.ones(d, device="cuda")                                 # a few large channels, as keys of trained models have
    channel[torch.randperm(d, generator=cpu)[:4].cuda()] = 5.0
    rows = sum(c for _, c in chunks) + len(lens)
    if op == "cross" or case["append"]:
        st["pool"] = torch.empty(num_pages, 2, hkv, PAGE, d, device="cuda", dtype=torch.bfloat16)
        step = max(1, (1 << 26) // st["pool"][0].numel())
        for at in range(0, num_pages, step):
            part = torch.randn(st["pool"][at:at + step].shape, device="cuda", generator=gen)
            part[:, 0] *= channel
            st["pool"][at:at + step] = part
    if op == "cross":
        st["q"] = _normal((rows, hq, d), gen)
        st["out"] = torch.zeros_like(st["q"])
        st["lse"] = torch.zeros(rows, hq, device="cuda") if case["lse"] else None
    else:
        one = _normal((rows, hq + 2 * hkv, d), gen, channel)
        parts = (one[:, :hq], one[:, hq:hq + hkv], one[:, hq + hkv:])
        st["q"], st["k"], st["v"] = parts if case["packed"] else (x.contiguous() for x in parts)
        st["q_out"] = torch.zeros(rows, hq, d, device="cuda", dtype=torch.bfloat16)
        st["k_out"] = None if case["append"] else torch.zeros(rows, hkv, d, device="cuda", dtype=torch.bfloat16)
        st["positions"] = None
        if case["shift"]:
            st["positions"] = (torch.cat([torch.arange(p, p + c) for p, c in chunks] + [ints(lens) - 1]) + case["shift"]).to(torch.int32).cuda()
        w, st["magnitude"] = _frequencies(case)
        st["frequencies"] = torch.tensor(w, dtype=torch.float64, device="cuda")
    if own:
        _plan(st, host)
    return st


def _prepare_sample(case, gen, cpu):
    """Logits as language models make them: a wide bulk, some tens of plausible tokens far above it, sure rows and open ones."""
    rows, vocab = case["rows"], case["vocab"]
    x = torch.randn(rows, vocab, device="cuda", generator=gen) * (1.2 + 1.3 * torch.rand(rows, 1, device="cuda", generator=gen))
    plausible = torch.randint(vocab, (rows, 48), device="cuda", generator=gen)
    lift = (6 + 10 * torch.rand(rows, 48, device="cuda", generator=gen)) * (torch.rand(rows, 1, device="cuda", generator=gen) < 0.85)
    x.scatter_add_(1, plausible, lift)
    x = x.to({"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[case["dtype"]])
    st = {"case": case, "logits": x}
    st["uniform"] = torch.rand(rows, device="cuda", generator=gen).clamp(min=1e-6)
    choices = {"temperature": [0.0, 0.6, 0.7, 0.8, 1.0, 1.2], "top_k": [0, 0, 20, 40, 50, 100], "top_p": [1.0, 0.8, 0.9, 0.95], "min_p": [0.0, 0.0, 0.05, 0.1]}
    for name, values in choices.items():
        if case[name] == "mixed":
            picked = [values[i] for i in torch.randint(len(values), (rows,), generator=cpu).tolist()]
        else:
            picked = [case[name]] * rows
        st[name] = torch.tensor(picked, dtype=torch.int32 if name == "top_k" else torch.float32, device="cuda")
    st["tokens"] = torch.zeros(rows, dtype=torch.int32, device="cuda")
    st["log_probs"] = torch.zeros(rows, device="cuda")
    if own:
        from paper_2609_07883_b200 import binding as B
        from paper_2609_07883_b200 import workloads as W

        st["ctx"] = B.Context(W.AttnShape(8, 2, 64), 64, 1, 1, 0, device=torch.cuda.current_device())
    return st


def _plan(st, host):
    """What a program of this framework keeps: the context with its workspace, the batch's struct, the table of frequencies."""
    from paper_2609_07883_b200 import binding as B
    from paper_2609_07883_b200 import workloads as W

    case, chunks = st["case"], st["chunks"]
    shape, tokens = W.AttnShape(*_heads(case)), sum(c for _, c in chunks)
    np32 = {k: v.numpy() for k, v in host.items()}
    batch = W.MixedBatch(shape=shape, num_pages=st["num_pages"], prefix_len=chunks[0][0] if chunks else 0, chunk_len=tokens,
                         prefill_pages=np32["chunk_pages"], decode_kv_len=np32["kv_len"], decode_page_indptr=np32["indptr"], decode_pages=np32["pages"])
    if len(chunks) > 1:
        batch.chunk_prefix_lens = torch.tensor([p for p, _ in chunks], dtype=torch.int32).numpy()
        batch.chunk_lens = torch.tensor([c for _, c in chunks], dtype=torch.int32).numpy()
        batch.chunk_page_indptr = np32["chunk_indptr"]
    dev = torch.device("cuda", torch.cuda.current_device())
    st["ctx"] = B.Context(shape, st["num_pages"], max(tokens, 1), max(case["decodes"], 1), 0, device=dev.index)
    st["batch"] = B.DeviceBatch(batch, dev)
    if case["op"] == "rope":
        turns, magnitude = B.sw_rope_frequencies(case["rotary"], BASE, case["scaling"], case["factor"], case["original"], LOW.get(case["scaling"], 0.0),
                                                 HIGH.get(case["scaling"], 0.0))
        st["rope"] = B.Rope(turns, case["layout"] == "interleaved", magnitude, st["positions"], device=dev)


# ---- one pass --------------------------------------------------------------------------------------------------------------
def run(st):
    case = st["case"]
    if case["op"] == "sample":
        if own:
            from paper_2609_07883_b200 import binding as B

            B.sw_sample_run(st["ctx"], st["logits"], st["uniform"], st["tokens"], st["log_probs"], st["temperature"], st["top_k"], st["top_p"], st["min_p"])
        else:
            _sample_rows(st)
        return {"tokens": st["tokens"], "log_probs": st["log_probs"]}
    if case["op"] == "cross":
        if own:
            from paper_2609_07883_b200 import binding as B

            B.sw_cross_attn_run(st["ctx"], st["pool"], st["batch"], st["q"], st["out"], st["lse"])
        else:
            _attend(st)
        return {"out": st["out"]} if st["lse"] is None else {"out": st["out"], "lse": st["lse"]}
    if own:
        from paper_2609_07883_b200 import binding as B

        if case["append"]:
            B.sw_rope_append(st["ctx"], st["pool"], st["batch"], st["rope"], st["q"], st["k"], st["v"], st["q_out"])
        else:
            B.sw_rope_run(st["ctx"], st["batch"], st["rope"], st["q"], st["k"], st["q_out"], st["k_out"])
    else:
        _rotate_rows(st)
    return {"q": st["q_out"], "pool": st["pool"]} if case["append"] else {"q": st["q_out"], "k": st["k_out"]}


# ---- the plain forms -------------------------------------------------------------------------------------------------------
def _places(st):
    """Position in its sequence, page and slot of every row."""
    pos = torch.cat([torch.arange(p, p + c, device="cuda") for p, c in st["chunks"]] + [st["kv_len"].long() - 1])
    first = [st["chunk_indptr"][j].expand(c) for j, (_, c) in enumerate(st["chunks"])]
    page = [st["chunk_pages"][torch.cat(first).long() + pos[:sum(c for _, c in st["chunks"])] // PAGE]] if first else []
    decodes = pos[len(pos) - len(st["kv_len"]):]
    page.append(st["pages"][st["indptr"][:-1].long() + decodes // PAGE])
    return pos, torch.cat(page).long(), pos % PAGE


def _rotate_rows(st):
    case = st["case"]
    pos, page, slot = _places(st)
    angle = (pos if st["positions"] is None else st["positions"]).double()[:, None] * st["frequencies"]    # (far positions need 64 bits)
    cos, sin = ((f(angle) * st["magnitude"]).float()[:, None] for f in (torch.cos, torch.sin))
    rotary = case["rotary"]
    if case["layout"] == "half":
        a, b = slice(0, rotary // 2), slice(rotary // 2, rotary)
    else:
        a, b = slice(0, rotary, 2), slice(1, rotary, 2)

    def rotated(x):
        x = x.float()
        y = x.clone()
        y[..., a] = x[..., a] * cos - x[..., b] * sin
        y[..., b] = x[..., b] * cos + x[..., a] * sin
        return y.to(torch.bfloat16)

    st["q_out"].copy_(rotated(st["q"]))
    if case["append"]:
        st["pool"][page, 0, :, slot] = rotated(st["k"])
        st["pool"][page, 1, :, slot] = st["v"]
    else:
        st["k_out"].copy_(rotated(st["k"]))


def _softmax(s):
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - top)
    total = p.sum(-1, keepdim=True)
    return p / total, (top + torch.log(total)).squeeze(-1)


def _attend(st):
    case = st["case"]
    hq, hkv, d = _heads(case)
    g, scale, at = hq // hkv, 1.0 / math.sqrt(d), 0

    def rows_of(pages):
        """K and V rows of a page list [..., pages] in 32 bits: two tensors [..., head, token, element]."""
        x = st["pool"][pages.long()].float()
        return (x.select(-4, side).movedim(-3, -4).flatten(-3, -2) for side in (0, 1))

    def store(rows, o, lse):                                               # [row][KV head][query head of its group](element)
        st["out"][rows] = o.flatten(1, 2).to(torch.bfloat16)
        if st["lse"] is not None:
            st["lse"][rows] = lse.flatten(1, 2)

    for j, (keys, c) in enumerate(st["chunks"]):
        k, v = rows_of(st["chunk_pages"][st["chunk_indptr"][j]:st["chunk_indptr"][j + 1]])
        q = st["q"][at:at + c].float().view(c, hkv, g, d)
        o, lse = torch.empty_like(q), torch.empty(c, hkv, g, device="cuda")
        for h in range(hkv):                                               # (the scores of all heads at once would fill the card)
            w, lse[:, h] = _softmax(q[:, h] @ k[h, :keys].T * scale)
            o[:, h] = w @ v[h, :keys]
        store(slice(at, at + c), o, lse)
        at += c
    n = case["decodes"]
    if n == 0:
        return
    length = st["kv_len"].long()
    index = torch.arange(-(-st["longest"] // PAGE), device="cuda")
    listed_ = index < (-(-length // PAGE))[:, None]
    k, v = rows_of(st["pages"][torch.where(listed_, st["indptr"][:-1, None].long() + index, 0)])
    q = st["q"][at:].float().view(n, hkv, g, d)
    seen = torch.arange(k.shape[2], device="cuda") < length[:, None]
    w, lse = _softmax(torch.where(seen[:, None, None], q @ k.transpose(-1, -2) * scale, -math.inf))
    store(slice(at, at + n), w @ v, lse)


def _sample_rows(st):
    x = st["logits"].double()                                              # (sums of all weights, and values next to a border)
    rows, vocab = x.shape
    t = st["temperature"].double()[:, None]
    w = torch.exp((x - x.amax(-1, keepdim=True)) / torch.where(t > 0, t, 1.0))
    order = torch.sort(x, dim=-1, descending=True, stable=True).indices    # ties: the lowest index
    falling = w.gather(-1, order)
    rank = torch.arange(vocab, device="cuda")
    top_k = torch.where(st["top_k"] > 0, st["top_k"], vocab)[:, None]
    falling = torch.where(rank < top_k, falling, 0.0)
    share = st["top_p"].double()[:, None]
    before = falling.cumsum(-1) - falling
    keep = (rank < top_k) & ((share >= 1) | (rank == 0) | (before < share * falling.sum(-1, keepdim=True)))
    keep &= falling >= st["min_p"].double()[:, None]
    kept = torch.zeros_like(w).scatter_(-1, order, torch.where(keep, falling, 0.0))
    sums = kept.cumsum(-1)
    token = (sums > st["uniform"].double()[:, None] * sums[:, -1:]).int().argmax(-1)
    greedy = t[:, 0] <= 0
    token = torch.where(greedy, order[:, 0], token)
    p = kept.gather(-1, token[:, None])[:, 0] / sums[:, -1]
    st["tokens"].copy_(token)
    st["log_probs"].copy_(torch.where(greedy, 0.0, torch.log(p)))


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------------
def exact(case, seed):
    """The operators' results from their definitions in 64 bits: rotations as products of complex numbers, one (sequence, head) pair of an attention
    after another, one row of logits after another."""
    st = prepare(case, seed)
    return {"rope": _exact_rope, "cross": _exact_cross, "sample": _exact_sample}[case["op"]](st)


def _exact_rope(st):
    case = st["case"]
    rotary, half = case["rotary"], case["rotary"] // 2
    where = []                                                             # (first row, rows, position of the first, page list)
    at, cptr, ptr = 0, st["chunk_indptr"].tolist(), st["indptr"].tolist()
    for j, (p, c) in enumerate(st["chunks"]):
        where.append((at, c, p, st["chunk_pages"][cptr[j]:cptr[j + 1]].long()))
        at += c
    where += [(at + i, 1, n - 1, st["pages"][ptr[i]:ptr[i + 1]].long()) for i, n in enumerate(st["kv_len"].tolist())]
    q, k = st["q"].double().contiguous(), st["k"].double().contiguous()
    pool = st["pool"].double() if case["append"] else None
    w, magnitude = _frequencies(case)
    w = torch.tensor(w, dtype=torch.float64, device="cuda")
    for row, c, p, pages in where:
        pos = torch.arange(p + case["shift"], p + case["shift"] + c, device="cuda", dtype=torch.float64)
        turn = torch.polar(torch.full((c, half), magnitude, dtype=torch.float64, device="cuda"), pos[:, None] * w)
        for x in (q, k):
            z = x[row:row + c, :, :rotary].clone()
            if case["layout"] == "half":
                z = torch.complex(z[..., :half].contiguous(), z[..., half:].contiguous()) * turn[:, None]
                x[row:row + c, :, :rotary] = torch.cat([z.real, z.imag], -1)
            else:
                z = torch.view_as_complex(z.view(c, -1, half, 2)) * turn[:, None]
                x[row:row + c, :, :rotary] = torch.view_as_real(z).flatten(-2)
        if case["append"]:
            place = torch.arange(p, p + c, device="cuda")
            pool[pages[place // PAGE], 0, :, place % PAGE] = k[row:row + c]
            pool[pages[place // PAGE], 1, :, place % PAGE] = st["v"][row:row + c].double()
    return {"q": q, "pool": pool} if case["append"] else {"q": q, "k": k}


def _exact_cross(st):
    hq, hkv, d = _heads(st["case"])
    g = hq // hkv
    out = torch.zeros(st["q"].shape, device="cuda", dtype=torch.float64)
    lse = torch.zeros(st["q"].shape[:2], device="cuda", dtype=torch.float64)
    sequences, at, cptr, ptr = [], 0, st["chunk_indptr"].tolist(), st["indptr"].tolist()
    for j, (keys, c) in enumerate(st["chunks"]):
        sequences.append((at, c, keys, st["chunk_pages"][cptr[j]:cptr[j + 1]].long()))
        at += c
    sequences += [(at + i, 1, n, st["pages"][ptr[i]:ptr[i + 1]].long()) for i, n in enumerate(st["kv_len"].tolist())]
    for row, c, keys, ids in sequences:
        for h in range(hkv):
            k, v = (st["pool"][ids, side, h].double().reshape(-1, d)[:keys] for side in (0, 1))
            for r in range(h * g, h * g + g):
                s = (st["q"][row:row + c, r].double() @ k.T) / d ** 0.5
                lse[row:row + c, r] = torch.logsumexp(s, 1)
                out[row:row + c, r] = torch.exp(s - lse[row:row + c, r, None]) @ v
    return {"out": out} if st["lse"] is None else {"out": out, "lse": lse}


def _exact_sample(st):
    settings = zip(*(st[name].tolist() for name in ("temperature", "top_k", "top_p", "min_p", "uniform")))
    tokens, log_probs = [], []
    for x, (t, k, p, least, u) in zip(st["logits"], settings):
        x = x.double()
        best = int(torch.nonzero(x == x.max())[0, 0])
        if t <= 0:
            tokens.append(best)
            log_probs.append(0.0)
            continue
        weight = torch.exp((x - x[best]) / t)
        index = torch.argsort(-x, stable=True)
        if 0 < k < len(x):
            index = index[:k]
        if p < 1:
            share = torch.cumsum(weight[index], 0)
            enough = int((share < p * share[-1]).sum()) + 1                # as many as it takes to reach the share
            index = index[:enough]
        index = index[weight[index] >= least].sort().values
        sums = torch.cumsum(weight[index], 0)
        token = index[int((sums <= u * sums[-1]).sum())]
        tokens.append(int(token))
        log_probs.append(float(torch.log(weight[token] / sums[-1])))
    return {"tokens": torch.tensor(tokens, dtype=torch.int32, device="cuda"), "log_probs": torch.tensor(log_probs, dtype=torch.float64, device="cuda")}
