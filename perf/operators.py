"""What is measured of the operators for long prompts and bounded caches: inputs, plain forms and calls.

Four operators over a paged K/V cache ([page, slot, KV head, dim], found through a block table):

* window_step   one new token per sequence attends over the last `window` tokens and the first `sinks` ones
* weights_step  one new token per sequence attends over its whole cache, and the weight that each cached token got
                (summed over the query heads of its KV head) is added to a running total
* evict         of a cache that grew past its budget the first tokens, the most recent ones and those with the
                largest totals are kept: their K/V rows move to fresh pages, in their order
* prompt        a chunk of new tokens per sequence attends causally over the cache that already holds it, with or
                without a window and sinks

Head layouts are those of the repository's configurations (32/8 heads of 128, 8/2 heads of 64), pages hold 16 tokens
unless the case says otherwise.
"""
import math
import random

import torch

own = False

HEADS = {"large": (32, 8, 128), "tiny": (8, 2, 64), "mha": (8, 8, 128), "wide": (48, 4, 128), "odd": (20, 4, 64)}
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


# ------------------------------------------------------------------------------------------------ cases

def listed():
    return [
        # one long conversation, a single user waiting: a call is mostly latency
        {"name": "window_step_one", "op": "window_step", "heads": "large", "dtype": "bf16", "page": 16, "batch": 1,
         "lo": 32768, "hi": 32768, "lens": 1, "window": 1024, "sinks": 4},
        # a batch of short chats, most of them longer than a small window, some shorter
        {"name": "window_step_chat", "op": "window_step", "heads": "large", "dtype": "bf16", "page": 16, "batch": 64,
         "lo": 30, "hi": 900, "lens": 2, "window": 256, "sinks": 4},
        # a full serving batch of long sequences of which the window is all that is still cached
        {"name": "window_step_batch", "op": "window_step", "heads": "large", "dtype": "bf16", "page": 16, "batch": 256,
         "lo": 3000, "hi": 32768, "lens": 3, "window": 4096, "sinks": 4},
        # the smallest model served alone
        {"name": "weights_step_one", "op": "weights_step", "heads": "tiny", "dtype": "fp16", "page": 16, "batch": 1,
         "lo": 2049, "hi": 2049, "lens": 4},
        # a chat batch whose caches are bounded by eviction: up to a budget and what came since
        {"name": "weights_step_chat", "op": "weights_step", "heads": "large", "dtype": "bf16", "page": 16, "batch": 64,
         "lo": 1, "hi": 2176, "lens": 5},
        # long generations just before their caches are cut
        {"name": "weights_step_long", "op": "weights_step", "heads": "large", "dtype": "bf16", "page": 16, "batch": 16,
         "lo": 30000, "hi": 32768, "lens": 6},
        # a few small caches
        {"name": "evict_few", "op": "evict", "heads": "tiny", "dtype": "fp16", "page": 16, "batch": 4,
         "lo": 120, "hi": 300, "lens": 7, "budget": 128, "sinks": 4, "recent": 32},
        # the steady state of a serving batch: every row is cut back once it is some 128 tokens over its budget
        {"name": "evict_steady", "op": "evict", "heads": "large", "dtype": "bf16", "page": 16, "batch": 64,
         "lo": 1100, "hi": 1180, "lens": 8, "budget": 1024, "sinks": 4, "recent": 256},
        # long contexts cut to an eighth
        {"name": "evict_long", "op": "evict", "heads": "large", "dtype": "bf16", "page": 16, "batch": 8,
         "lo": 30001, "hi": 32768, "lens": 9, "budget": 4096, "sinks": 4, "recent": 1024},
        # short prompts of a few users, nothing cached before them
        {"name": "prompt_short", "op": "prompt", "heads": "large", "dtype": "bf16", "page": 16, "batch": 8,
         "lo": 1, "hi": 70, "lens": 10, "cached_lo": 0, "cached_hi": 0, "window": 0, "sinks": 0},
        # chunked prefill: a few hundred new tokens behind contexts of some thousand, windowed
        {"name": "prompt_chunk", "op": "prompt", "heads": "large", "dtype": "bf16", "page": 16, "batch": 4,
         "lo": 400, "hi": 512, "lens": 11, "cached_lo": 1500, "cached_hi": 9000, "window": 2048, "sinks": 4},
        # one long prompt's later chunk, windowed
        {"name": "prompt_long", "op": "prompt", "heads": "large", "dtype": "bf16", "page": 16, "batch": 1,
         "lo": 4096, "hi": 4096, "lens": 12, "cached_lo": 12288, "cached_hi": 12288, "window": 4096, "sinks": 4},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["window_step", "weights_step", "evict", "prompt"])
    c = {"op": op, "heads": rng.choice(["large", "large", "tiny", "mha", "wide", "odd"]), "dtype": rng.choice(["bf16", "fp16"]),
         "page": rng.choice([16, 16, 32, 64, 128, 256]), "lens": rng.randrange(1 << 30)}
    if op == "window_step":
        c["window"], c["sinks"] = _log(rng, 1, 4096), rng.choice([0, 1, 4, 4, 16, 37, 128])
        c["batch"] = min(_log(rng, 1, 256), max(1, 1_000_000 // (c["window"] + c["sinks"])))
        c["hi"] = _log(rng, 1, 32768)
        c["lo"] = rng.randint(1, c["hi"])
    elif op == "weights_step":
        c["hi"] = _log(rng, 1, 32768)
        c["lo"] = rng.randint(1, c["hi"])
        c["batch"] = min(_log(rng, 1, 128), max(1, 400_000 // c["hi"]))
    elif op == "evict":
        c["budget"] = _log(rng, 16, 4096)
        c["sinks"] = min(rng.choice([0, 1, 4, 16]), c["budget"] // 4)
        c["recent"] = rng.randint(0, c["budget"] // 2)
        c["hi"] = min(32768, c["budget"] + _log(rng, 1, 16384))
        c["lo"] = rng.randint(max(1, c["budget"] // 2), c["hi"])
        c["batch"] = min(_log(rng, 1, 64), max(1, 250_000 // c["hi"]))
    else:
        c["window"] = rng.choice([0, _log(rng, 1, 4096)])
        c["sinks"] = rng.choice([0, 1, 4, 16, 37]) if c["window"] else 0
        c["hi"] = _log(rng, 1, 4096)
        c["cached_hi"] = rng.choice([0, _log(rng, 1, 8192)])
        hq, _, d = HEADS[c["heads"]]
        most = 4096 * 4100 * 32 * 128                                          # what the largest listed prompt costs
        cost = lambda: c["hi"] * ((c["window"] + c["sinks"]) or (c["hi"] + c["cached_hi"])) * hq * d
        while cost() > most:
            c["hi"], c["cached_hi"] = c["hi"] * 3 // 4, c["cached_hi"] * 3 // 4
        c["lo"] = rng.randint(1, c["hi"])
        c["cached_lo"] = rng.randint(0, c["cached_hi"])
        c["batch"] = min(_log(rng, 1, 16), max(1, most // cost()))
    return c


def _lengths(case):
    """Cached tokens of every sequence (with the new ones) and its new tokens: of the case alone."""
    rng = random.Random(case["lens"])
    lens = [rng.randint(case["lo"], case["hi"]) for _ in range(case["batch"])]
    if case["op"] == "prompt":
        news = lens
        return [n + rng.randint(case["cached_lo"], case["cached_hi"]) for n in news], news
    if case["op"] == "evict" and max(lens) <= case["budget"]:
        lens[0] = case["budget"] + 1
    return lens, [1] * case["batch"]


def _visible(length, new, window):
    """The first position that the oldest of the `new` last queries sees through its window."""
    return max(0, length - new - window + 1) if window else 0


# ------------------------------------------------------------------------------------------------ inputs

def prepare(case, seed):
    hq, hkv, d = HEADS[case["heads"]]
    dt, page, batch, op = DTYPES[case["dtype"]], case["page"], case["batch"], case["op"]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1000 + seed)
    host = random.Random(seed)
    lens, news = _lengths(case)
    window, sinks = case.get("window", 0), case.get("sinks", 0)
    # Pages: a window's sequences hold the pages of their visible tokens alone (an engine takes the others back), and
    # their other block-table entries are -1; an eviction has fresh pages to move to.
    wide = max(-(-n // page) for n in lens)
    rows, used = [], 0
    for n, new in zip(lens, news):
        first = _visible(n, new, window) // page if op in ("window_step", "prompt") else 0
        live = [i for i in range(-(-n // page)) if i >= first or i * page < sinks]
        rows.append(live)
        used += len(live)
    fresh = -(-case["budget"] // page) * batch if op == "evict" else 0
    num_pages = used + fresh + 1
    ids = list(range(num_pages))
    host.shuffle(ids)
    table, at = [], 0
    for live in rows:
        row = [-1] * wide
        for i in live:
            row[i] = ids[at]
            at += 1
        table.append(row)
    s = {"case": case, "op": op, "hq": hq, "hkv": hkv, "d": d, "page": page, "batch": batch, "window": window,
         "sinks": sinks, "lens_host": lens, "news_host": news}
    s["block_table"] = torch.tensor(table, dtype=torch.int32, device="cuda")
    s["seq_lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    pool = (num_pages, page, hkv, d)
    s["k"] = torch.randn(pool, dtype=dt, device="cuda", generator=gen)
    s["v"] = torch.randn(pool, dtype=dt, device="cuda", generator=gen)
    if op != "evict":
        total = sum(news)
        s["q"] = torch.randn((total, hq, d), dtype=dt, device="cuda", generator=gen)
        s["out"] = torch.zeros((total, hq, d), dtype=dt, device="cuda")
        s["lse"] = torch.zeros((total, hq), dtype=torch.float32, device="cuda")
    if op == "prompt":
        s["new_lens"] = torch.tensor(news, dtype=torch.int32, device="cuda")
        s["row_seq"] = torch.repeat_interleave(torch.arange(batch, device="cuda"), s["new_lens"].long())
        starts = torch.cumsum(s["new_lens"].long(), 0) - s["new_lens"].long()
        s["row_pos"] = torch.arange(total, device="cuda") - starts[s["row_seq"]]
        s["starts"] = starts
    if op in ("weights_step", "evict"):
        most = max(lens)
        # totals of attention weights: most tokens got next to nothing, a few got a lot
        s["weights"] = torch.exp(2.0 * torch.randn((batch, hkv, most), device="cuda", generator=gen) - 3.0)
        s["weights_out"] = torch.zeros_like(s["weights"])
    if op == "evict":
        n_dst = -(-case["budget"] // page)
        s["dst_table"] = torch.tensor([[ids[at + b * n_dst + i] for i in range(n_dst)] for b in range(batch)],
                                      dtype=torch.int32, device="cuda")
        s["kept"] = torch.zeros((batch, hkv, case["budget"]), dtype=torch.int32, device="cuda")
        s["lens_out"] = torch.zeros(batch, dtype=torch.int32, device="cuda")
        s["over"] = torch.tensor([b for b in range(batch) if lens[b] > case["budget"]], device="cuda")
    if own:
        from paper_2609_37062_b200 import binding as da
        strides = (page * hkv * d, hkv * d, d)
        kind = da.DA_DTYPE_FP16 if case["dtype"] == "fp16" else da.DA_DTYPE_BF16
        s["da"] = da
        s["shape"] = da.make_shape(batch, hq, hkv, d, page, wide, num_pages, strides, out_dtype=kind, in_dtype=kind)
        if op == "window_step":
            s["plan"] = da.decode_attn_plan(s["shape"], da.make_policy(window_tokens=window, sink_tokens=sinks), lens)
        elif op == "weights_step":
            s["plan"] = da.decode_attn_plan(s["shape"], da.make_policy(track_weights=1), lens)
        elif op == "prompt":
            s["plan"] = da.decode_attn_prompt_plan(s["shape"], da.make_policy(window_tokens=window, sink_tokens=sinks), news, lens)
        if "plan" in s:
            s["ws"] = torch.empty(max(s["plan"].workspace_bytes, 256), dtype=torch.uint8, device="cuda")
    return s


# ------------------------------------------------------------------------------------------------ one pass

def run(s):
    return _RUN[bool(own)][s["op"]](s)


def _own_step(s):
    da = s["da"]
    da.decode_attn_run(s["plan"], s["q"], s["k"], s["v"], s["block_table"], s["seq_lens"], s["out"], s["lse"], s["ws"])
    da.decode_attn_combine(s["plan"], s["ws"], s["out"], s["lse"])
    return {"out": s["out"], "lse": s["lse"]}


def _own_weights(s):
    r = _own_step(s)
    s["da"].decode_attn_add_weights(s["plan"], s["ws"], s["lse"], s["seq_lens"], s["weights"], s["weights_out"])
    return {**r, "weights": s["weights_out"]}


def _own_evict(s):
    c = s["case"]
    s["da"].decode_attn_evict(s["shape"], c["budget"], c["sinks"], c["recent"], s["seq_lens"], s["block_table"], s["dst_table"],
                              s["k"], s["v"], s["weights"], s["weights_out"], s["kept"], s["lens_out"])
    return {"kept": s["kept"], "lens": s["lens_out"], "weights": s["weights_out"], "k": s["k"], "v": s["v"]}


def _own_prompt(s):
    s["da"].decode_attn_prompt_run(s["plan"], s["q"], s["k"], s["v"], s["block_table"], s["seq_lens"], s["out"], s["lse"], s["ws"])
    return {"out": s["out"], "lse": s["lse"]}


def _rows(s, pool, pos):
    """K or V rows of the logical positions pos [batch, n] in 32 bits: [batch, KV head, n, dim]."""
    pages = s["block_table"].long().gather(1, pos // s["page"])
    return pool[pages, pos % s["page"]].float().permute(0, 2, 1, 3)


def _attend(q, k, v, seen, scale):
    """q [b, g, r, d] over k, v [b, g, n, d] where seen (broadcast to [b, g, r, n]); outputs, log-sum-exps, weights."""
    x = torch.where(seen, (q @ k.transpose(-1, -2)) * scale, float("-inf"))
    m = x.amax(-1, keepdim=True)
    m = torch.where(torch.isinf(m), 0.0, m)
    p = torch.exp(x - m)
    total = p.sum(-1, keepdim=True)
    out = (p @ v) / torch.where(total > 0, total, 1.0)
    return out, (m + torch.log(total)).squeeze(-1), p, total


def _plain_positions(s, first, n):
    """Positions that some query may see: the sinks, then n from `first` [batch] on; and which of them are real."""
    at, lens = first[:, None] + torch.arange(n, device="cuda"), s["seq_lens"].long()[:, None]
    sinks = torch.arange(s["sinks"], device="cuda").expand(s["batch"], -1)
    pos = torch.cat([sinks, at], 1)
    real = torch.cat([sinks < torch.minimum(lens, first[:, None]), at < lens], 1)
    # what is not real is read from the last position and not looked at
    return torch.where(real, pos, lens - 1), pos, real


def _plain_step(s):
    g, lens = s["hq"] // s["hkv"], s["seq_lens"].long()
    window = s["window"] if s["op"] == "window_step" else 0
    first = (lens - window).clamp(min=0) if window else torch.zeros_like(lens)
    widest = max(s["lens_host"])
    pos, _, real = _plain_positions(s, first, min(window, widest) if window else widest)
    q = s["q"].float().view(s["batch"], s["hkv"], g, s["d"])
    out, lse, p, total = _attend(q, _rows(s, s["k"], pos), _rows(s, s["v"], pos), real[:, None, None], 1 / math.sqrt(s["d"]))
    r = {"out": out.reshape(s["out"].shape).to(s["out"].dtype), "lse": lse.reshape(s["lse"].shape)}
    if s["op"] == "weights_step":
        grown = s["weights"] + (p / total).sum(2)
        at = torch.arange(widest, device="cuda")
        r["weights"] = torch.where((at < lens[:, None])[:, None], grown, s["weights_out"])
    return r


def _plain_evict(s):
    c, lens = s["case"], s["seq_lens"].long()[:, None, None]
    budget, most = c["budget"], s["weights"].shape[2]
    at = torch.arange(most, device="cuda")
    safe = (at < c["sinks"]) | (at >= lens - c["recent"])
    rank = torch.where(safe, float("inf"), s["weights"])
    rank = torch.where(at < lens, rank, float("-inf"))
    best = torch.sort(rank, dim=-1, descending=True, stable=True).indices[..., :budget]
    n = lens.clamp(max=budget)
    place = torch.arange(best.shape[-1], device="cuda")
    kept = torch.sort(torch.where(place < n, best, most), dim=-1).values
    total = torch.where(place < n, s["weights"].gather(2, kept.clamp(max=most - 1)), 0.0)
    weights = torch.zeros_like(s["weights"])
    weights[..., :total.shape[-1]] = total
    weights = torch.where(at < lens, weights, s["weights_out"])
    out = torch.full_like(s["kept"], -1)
    out[..., :kept.shape[-1]] = torch.where(place < n, kept, -1).int()
    over = s["over"]
    rows = kept[over]
    pages = s["block_table"].long()[over][:, None].expand(-1, s["hkv"], -1).gather(2, rows // s["page"])
    heads = torch.arange(s["hkv"], device="cuda")[None, :, None]
    to = torch.arange(budget, device="cuda")
    to_pages = s["dst_table"].long()[over][:, None, to // s["page"]]
    s["k"][to_pages, to % s["page"], heads] = s["k"][pages, rows % s["page"], heads]
    s["v"][to_pages, to % s["page"], heads] = s["v"][pages, rows % s["page"], heads]
    return {"kept": out, "lens": lens.view(-1).clamp(max=budget).int(), "weights": weights, "k": s["k"], "v": s["v"]}


def _plain_prompt(s):
    g, lens, news = s["hq"] // s["hkv"], s["seq_lens"].long(), s["new_lens"].long()
    window, most = s["window"], max(s["news_host"])
    first = (lens - news - window + 1).clamp(min=0) if window else torch.zeros_like(lens)
    span = max(n - _visible(n, new, window) for n, new in zip(s["lens_host"], s["news_host"]))
    pos, at, real = _plain_positions(s, first, span)
    rows = torch.arange(most, device="cuda")
    mine = (lens - news)[:, None] + rows                                       # a query's own position
    seen = real[:, None] & (at[:, None] <= mine[:, :, None])
    if window:
        seen = seen & ((mine[:, :, None] - at[:, None] < window) | (at[:, None] < s["sinks"]))
    pick = s["starts"][:, None] + torch.minimum(rows, news[:, None] - 1)
    q = s["q"][pick].float().view(s["batch"], most, s["hkv"], g, s["d"]).permute(0, 2, 3, 1, 4)
    seen = seen[:, None, None].expand(-1, 1, g, -1, -1).reshape(s["batch"], 1, g * most, -1)
    q = q.reshape(s["batch"], s["hkv"], g * most, s["d"])
    out, lse, _, _ = _attend(q, _rows(s, s["k"], pos), _rows(s, s["v"], pos), seen, 1 / math.sqrt(s["d"]))
    out = out.view(s["batch"], s["hq"], most, s["d"])[s["row_seq"], :, s["row_pos"]]
    lse = lse.reshape(s["batch"], s["hq"], most)[s["row_seq"], :, s["row_pos"]]
    return {"out": out.to(s["out"].dtype), "lse": lse}


_RUN = {False: {"window_step": _plain_step, "weights_step": _plain_step, "evict": _plain_evict, "prompt": _plain_prompt},
        True: {"window_step": _own_step, "weights_step": _own_weights, "evict": _own_evict, "prompt": _own_prompt}}


# ------------------------------------------------------------------------------------------------ the least work

def work(case):
    hq, hkv, d = HEADS[case["heads"]]
    lens, news = _lengths(case)
    window, sinks, op = case.get("window", 0), case.get("sinks", 0), case["op"]
    row = hkv * d * 2 * 2                                                      # K and V of a token
    if op == "evict":
        kept = sum(min(n, case["budget"]) for n in lens if n > case["budget"])
        return {"bytes": kept * row * 2 + sum(lens) * hkv * 8 + case["batch"] * (hkv * case["budget"] * 4 + 4),
                "flops": 0}
    read, pairs = 0, 0
    for n, new in zip(lens, news):
        first = _visible(n, new, window)
        read += n - first + min(sinks, first)
        i = torch.arange(n - new, n)
        low = (i - window + 1).clamp(min=0) if window else torch.zeros_like(i)
        pairs += int((i + 1 - low + low.clamp(max=sinks)).sum())
    rows = sum(news) * hq
    total = read * row + rows * (d * 4 + 4)
    if op == "weights_step":
        total += sum(lens) * hkv * 8
    return {"bytes": total, "flops": 4 * d * hq * pairs}


# ------------------------------------------------------------------------------------------------ 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    lens, news, page, d = s["lens_host"], s["news_host"], s["page"], s["d"]
    if s["op"] == "evict":
        return _exact_evict(s)
    g = s["hq"] // s["hkv"]
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device="cuda")
    weights = s["weights_out"].double() if s["op"] == "weights_step" else None
    start = 0
    for b, (n, new) in enumerate(zip(lens, news)):
        at = torch.arange(n, device="cuda")
        first = _visible(n, new, s["window"])
        at = at[(at >= first) | (at < s["sinks"])]
        pages = s["block_table"][b].long()[at // page]
        for lo in range(0, new, 512):
            hi = min(new, lo + 512)
            mine = torch.arange(n - new + lo, n - new + hi, device="cuda")
            hidden = at[None] > mine[:, None]
            if s["window"]:
                hidden |= (mine[:, None] - at[None] >= s["window"]) & (at[None] >= s["sinks"])
            for h in range(s["hkv"]):
                k, v = s["k"][pages, at % page, h].double(), s["v"][pages, at % page, h].double()
                q = s["q"][start + lo:start + hi, h * g:(h + 1) * g].double()
                x = torch.einsum("rjd,nd->rjn", q, k) / math.sqrt(d)
                x.masked_fill_(hidden[:, None], -math.inf)
                e = torch.logsumexp(x, -1)
                p = torch.exp(x - e[..., None])
                lse[start + lo:start + hi, h * g:(h + 1) * g] = e
                out[start + lo:start + hi, h * g:(h + 1) * g] = torch.einsum("rjn,nd->rjd", p, v)
                if weights is not None:
                    weights[b, h, :n] = s["weights"][b, h, :n].double() + p[0].sum(0)
        start += new
    r = {"out": out, "lse": lse}
    return r if weights is None else {**r, "weights": weights}


def _exact_evict(s):
    """Nothing is computed: which tokens stay, said once more token by token; the moved rows have no value of their own here."""
    c = s["case"]
    budget, w = c["budget"], s["weights"].double().cpu()
    kept, weights = torch.full(s["kept"].shape, -1, dtype=torch.int32), s["weights_out"].double().cpu()
    for b, n in enumerate(s["lens_host"]):
        for h in range(s["hkv"]):
            row = w[b, h, :n].tolist()
            if n <= budget:
                stay = list(range(n))
            else:
                sure = set(range(c["sinks"])) | set(range(n - c["recent"], n))
                rest = sorted((t for t in range(n) if t not in sure), key=lambda t: (-row[t], t))
                stay = sorted(sure | set(rest[:budget - len(sure)]))
            kept[b, h, :len(stay)] = torch.tensor(stay, dtype=torch.int32)
            weights[b, h, :n] = 0
            weights[b, h, :len(stay)] = w[b, h, stay]
    return {"kept": kept.cuda(), "lens": torch.tensor([min(n, budget) for n in s["lens_host"]], dtype=torch.int32, device="cuda"),
            "weights": weights.cuda(), "k": None, "v": None}
