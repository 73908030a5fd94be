"""What is measured of the operators around a decode step: inputs, plain forms and calls.

Four operators of a serving step with a paged K/V cache, in the order in which a step uses them:

* tables   block tables, slots, positions and row starts of a step from how many tokens every sequence gains or gives
           back, with the free pages in a list on the GPU
* rows     the projected q, k and v rows of the step's tokens: a norm of every query and key head, the rotation of
           their positions, and K and V written to their slots of the cache
* chunk    K and V rows of a prompt's chunk written to a cache held in 4 bits, and that cache's sequences expanded
           to 16-bit pages, which the attention of prompts reads
* step4    one new token per sequence attends over a cache held in 4 bits

The cache in 4 bits is one array of bytes [page, KV head, page_size / 16 tiles]. A tile holds 16 tokens of one head in
16 * dim + 64 * (dim / 32) bytes: K codes, V codes, K scales, V scales. A value is its code in e2m1 (sign, magnitude 0,
.5, 1, 1.5, 2, 3, 4 or 6) times the fp16 scale of its 32 dims; the scale is the largest magnitude over 6, and a code
is the nearest to the value over the scale, ties to the even code. `_places` says which byte holds what.

Head layouts are those of the repository's configurations (32/8 heads of 128, 8/2 heads of 64).
"""
import math
import random

import torch

own = False

HEADS = {"large": (32, 8, 128), "tiny": (8, 2, 64), "mha": (8, 8, 128), "wide": (48, 4, 128), "odd": (20, 4, 64)}
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
EPS = 1e-6


# ------------------------------------------------------------------------------------------------ cases

def listed():
    return [
        # a decode step of a chat batch: every sequence gains a token, some need a page; a call is all latency
        {"name": "tables_step", "op": "tables", "page": 16, "batch": 64, "lo": 30, "hi": 4000, "grow": 1, "end": 0.0,
         "prompt": 0.0, "pad": 0, "lens": 1},
        # continuous batching: most rows decode, some take a prompt's chunk, some have ended or lose rejected tokens;
        # the row buffers are those of a captured step, longer than what it needs
        {"name": "tables_mixed", "op": "tables", "page": 64, "batch": 256, "lo": 1, "hi": 8000, "grow": 512, "end": 0.1,
         "prompt": 0.2, "pad": 3001, "lens": 2},
        # an offline batch of prompts: a million tokens
        {"name": "tables_prompts", "op": "tables", "page": 16, "batch": 256, "lo": 0, "hi": 0, "grow": 8192, "end": 0.0,
         "prompt": 1.0, "pad": 0, "lens": 3},
        # the rows of a decode step, a few of them padding of a captured batch
        {"name": "rows_step", "op": "rows", "heads": "large", "dtype": "bf16", "page": 16, "rows": 61, "pad": 3, "norm": True,
         "rotary": 128, "pairs": False, "far": 32768},
        # a small model with a partial rotation of neighbouring pairs, no norms
        {"name": "rows_odd", "op": "rows", "heads": "odd", "dtype": "fp16", "page": 32, "rows": 1777, "pad": 0, "norm": False,
         "rotary": 32, "pairs": True, "far": 8000},
        # the tokens of a prefill step
        {"name": "rows_prompt", "op": "rows", "heads": "large", "dtype": "bf16", "page": 16, "rows": 8192, "pad": 0, "norm": True,
         "rotary": 128, "pairs": False, "far": 32768},
        # short prompts behind little
        {"name": "chunk_short", "op": "chunk", "heads": "tiny", "dtype": "fp16", "page": 16, "batch": 4, "lo": 1, "hi": 70,
         "cached_lo": 0, "cached_hi": 400, "lens": 4},
        # chunked prefill behind long contexts
        {"name": "chunk_long", "op": "chunk", "heads": "large", "dtype": "bf16", "page": 16, "batch": 4, "lo": 400, "hi": 512,
         "cached_lo": 8000, "cached_hi": 30000, "lens": 5},
        # one long conversation, a single user waiting
        {"name": "step4_one", "op": "step4", "heads": "large", "dtype": "bf16", "page": 16, "batch": 1, "lo": 32768, "hi": 32768,
         "lens": 6},
        # a batch of short chats
        {"name": "step4_chat", "op": "step4", "heads": "large", "dtype": "bf16", "page": 16, "batch": 64, "lo": 30, "hi": 900,
         "lens": 7},
        # many query heads to a KV head, larger pages
        {"name": "step4_wide", "op": "step4", "heads": "wide", "dtype": "fp16", "page": 64, "batch": 24, "lo": 1, "hi": 8191,
         "lens": 8},
        # a full batch of long sequences: three and a half times what the card holds in 16 bits
        {"name": "step4_long", "op": "step4", "heads": "large", "dtype": "bf16", "page": 16, "batch": 64, "lo": 28000,
         "hi": 32768, "lens": 9},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["tables", "rows", "chunk", "step4", "step4"])
    c = {"op": op, "page": rng.choice([16, 16, 32, 64, 128, 256]), "lens": rng.randrange(1 << 30)}
    if op == "tables":
        c["batch"] = _log(rng, 1, 2048)
        c["hi"] = _log(rng, 1, 16384)
        c["lo"] = rng.randint(0, c["hi"])
        c["grow"] = _log(rng, 1, max(1, min(8192, 2_000_000 // c["batch"])))
        c["end"] = rng.choice([0.0, 0.0, round(rng.uniform(0, 0.5), 3)])
        c["prompt"] = rng.choice([0.0, 1.0, round(rng.uniform(0, 1), 3)])
        c["pad"] = rng.choice([0, _log(rng, 1, 5000)])
        return c
    c["heads"] = rng.choice(["large", "large", "tiny", "mha", "wide", "odd"])
    c["dtype"] = rng.choice(["bf16", "fp16"])
    hq, hkv, d = HEADS[c["heads"]]
    if op == "rows":
        c["rows"] = min(_log(rng, 1, 8192), 8192 * 48 * 128 // ((hq + 2 * hkv) * d))
        c["pad"] = rng.choice([0, 0, _log(rng, 1, 64)])
        c["norm"] = rng.choice([True, True, False])
        c["rotary"] = rng.choice([d, d, d // 2, d // 4, 8])
        c["pairs"] = rng.choice([False, False, True])
        c["far"] = max(c["rows"], _log(rng, 64, 131072))
    elif op == "chunk":
        c["hi"] = _log(rng, 1, 2048)
        c["lo"] = rng.randint(1, c["hi"])
        c["cached_hi"] = rng.choice([0, _log(rng, 1, 30000)])
        c["cached_lo"] = rng.randint(0, c["cached_hi"])
        c["batch"] = min(_log(rng, 1, 16), max(1, 60_000 * 8 * 128 // (hkv * d) // (c["hi"] + c["cached_hi"])))
    else:
        c["hi"] = _log(rng, 1, 32768)
        c["lo"] = rng.randint(1, c["hi"])
        c["batch"] = min(_log(rng, 1, 256), max(1, 1_500_000 * 8 * 128 // (hkv * d) // c["hi"]))
    return c


def _lengths(case):
    """Tokens before the call and what each sequence gains (or gives back), of the case alone."""
    rng = random.Random(case["lens"])
    batch = case["batch"]
    if case["op"] == "tables":
        lens = [rng.randint(case["lo"], case["hi"]) for _ in range(batch)]
        gain = [rng.randint(1, case["grow"]) if rng.random() < case["prompt"] else 1 for _ in range(batch)]
        for b in range(batch):
            if rng.random() < case["end"]:
                gain[b] = -lens[b] if rng.random() < 0.5 else -rng.randint(0, min(8, lens[b]))
        return lens, gain
    if case["op"] == "chunk":
        return ([rng.randint(case["cached_lo"], case["cached_hi"]) for _ in range(batch)],
                [rng.randint(case["lo"], case["hi"]) for _ in range(batch)])
    return [rng.randint(case["lo"], case["hi"]) for _ in range(batch)], [0] * batch


# ------------------------------------------------------------------------------------------------ the format of 4 bits

def _tile_bytes(d):
    return 16 * d + 64 * (d // 32)


def _places(d, device):
    """Within a tile: the byte of every pair of dims of K and of V [16, d / 2], the 2-byte word of every scale [16, d / 32]."""
    r, j, b = (torch.arange(n, device=device) for n in (16, d // 2, d // 32))
    r, pair = r[:, None], 2 * j
    k = r * (d // 2) + (pair % 32 // 8) * (d // 8) + 4 * (pair // 32) + pair % 8 // 2
    v = 8 * d + r * (d // 2) + (j ^ (32 * (r // 8)) if d == 128 else j)
    ks = 8 * d + r * (d // 32) + b
    vs = 8 * d + 16 * (d // 32) + 16 * b + 4 * (r // 4) + ((r % 4) ^ (r // 4))
    return k, v, ks, vs


def _encode(x):
    """Rows [..., d] to codes as bytes of two [..., d / 2] and fp16 scales [..., d / 32]."""
    x = x.float()
    blocks = x.reshape(*x.shape[:-1], -1, 32)
    scale = (blocks.abs().amax(-1) / 6).half()
    y = blocks / torch.where(scale > 0, scale, 1.0).float()[..., None]
    a = y.abs()
    code = (a > 0.25).byte() + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5)
    code = (code + 8 * ((y < 0) & (code > 0)).byte()).reshape(x.shape)
    return code[..., 0::2] + 16 * code[..., 1::2], scale


def _decode(codes, scale):
    """The values [..., d] in 32 bits."""
    code = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).long()
    size = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6], device=codes.device)[code]
    return (size.unflatten(-1, (-1, 32)) * scale.float()[..., None]).flatten(-2)


def _fill(pool, d, gen, dt):
    """Pages of normal K and V in the format, a few at a time."""
    at = _places(d, pool.device)
    tiles = pool.view(-1, _tile_bytes(d))
    for lo in range(0, tiles.shape[0], 1 << 16):
        part = tiles[lo:lo + (1 << 16)]
        words = part.view(torch.float16)
        for codes_at, scales_at in ((at[0], at[2]), (at[1], at[3])):
            codes, scale = _encode(torch.randn((part.shape[0], 16, d), device=pool.device, generator=gen).to(dt))
            part[:, codes_at] = codes
            words[:, scales_at] = scale


# ------------------------------------------------------------------------------------------------ inputs

def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3000 + seed)
    s = {"case": case, "op": case["op"], "page": case["page"]}
    _PREPARE[case["op"]](case, s, gen, random.Random(seed))
    if own:
        _prepare_own(case, s)
    return s


def _ints(x, dtype=torch.int32):
    return torch.tensor(x, dtype=dtype, device="cuda")


def _prepare_tables(case, s, gen, host):
    page, batch = case["page"], case["batch"]
    lens, gain = _lengths(case)
    after = [max(0, n + g) for n, g in zip(lens, gain)]
    s["wide"] = max(1, max(-(-max(n, m) // page) for n, m in zip(lens, after)))
    s["max_rows"] = sum(max(0, g) for g in gain) + case["pad"]
    held = [-(-n // page) for n in lens]
    need = sum(max(0, -(-m // page) - h) for m, h in zip(after, held))
    back = sum(max(0, h - -(-m // page)) for m, h in zip(after, held))
    free = need + 7                                          # (pages given back come on top of these)
    ids = torch.randperm(sum(held) + free + 1, device="cuda", generator=gen).int()
    s["num_pages"] = ids.numel()
    table = torch.full((batch, s["wide"]), -1, dtype=torch.int32, device="cuda")
    at = torch.arange(s["wide"], device="cuda") < _ints(held)[:, None]
    table[at] = ids[:sum(held)]
    s["block_table"], s["seq_lens"], s["gain"] = table, _ints(lens), _ints(gain)
    s["free_pages"] = torch.full((free + back,), -1, dtype=torch.int32, device="cuda")
    s["free_pages"][:free] = ids[sum(held):sum(held) + free]
    s["free_count"] = _ints([free])
    s["seq_lens_out"], s["free_count_out"] = torch.zeros_like(s["seq_lens"]), torch.zeros_like(s["free_count"])
    s["row_starts"] = torch.zeros(batch + 1, dtype=torch.int32, device="cuda")
    s["page_starts"] = torch.zeros(batch + 1, dtype=torch.int32, device="cuda")
    s["slots"] = torch.zeros(s["max_rows"], dtype=torch.int64, device="cuda")
    s["positions"] = torch.zeros(s["max_rows"], dtype=torch.int32, device="cuda")
    s["row_seq"] = torch.zeros(s["max_rows"], dtype=torch.int32, device="cuda")


def _prepare_rows(case, s, gen, host):
    hq, hkv, d = HEADS[case["heads"]]
    dt, page, n = DTYPES[case["dtype"]], case["page"], case["rows"] + case["pad"]
    s |= {"hq": hq, "hkv": hkv, "d": d}
    # one row of the projection holds the heads of q, k and v behind each other
    qkv = torch.randn((n, (hq + 2 * hkv) * d), device="cuda", generator=gen).to(dt)
    s["qkv"] = qkv
    s["q"], s["k"], s["v"] = (x.unflatten(1, (-1, d)) for x in qkv.split([hq * d, hkv * d, hkv * d], 1))
    norm = lambda: (1 + 0.1 * torch.randn(d, device="cuda", generator=gen)).to(dt)
    s["q_weight"], s["k_weight"] = (norm(), norm()) if case["norm"] else (None, None)
    half = case["rotary"] // 2
    turn = torch.arange(case["far"], device="cuda").double()[:, None] * \
        10000.0 ** (-torch.arange(half, device="cuda").double() / half)
    s["cos_sin"] = torch.cat([turn.cos(), turn.sin()], 1).float()
    s["num_pages"] = -(-2 * case["rows"] // page) + 1
    s["slots"] = torch.full((n,), -1, dtype=torch.int64, device="cuda")
    s["slots"][:case["rows"]] = torch.randperm(s["num_pages"] * page, device="cuda", generator=gen)[:case["rows"]]
    s["positions"] = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    s["positions"][:case["rows"]] = torch.randint(case["far"], (case["rows"],), device="cuda", generator=gen).int()
    s["q_out"] = torch.zeros((n, hq, d), dtype=dt, device="cuda")
    s["k_pool"], s["v_pool"] = (torch.zeros((s["num_pages"], page, hkv, d), dtype=dt, device="cuda") for _ in range(2))


def _paged(case, s, gen, lens):
    """A shuffled pool and its block table for sequences of these lengths."""
    page, batch = case["page"], case["batch"]
    held = [-(-n // page) for n in lens]
    s["wide"], s["num_pages"] = max(held), sum(held) + 1
    ids = torch.randperm(s["num_pages"], device="cuda", generator=gen).int()
    s["block_table"] = torch.full((batch, s["wide"]), -1, dtype=torch.int32, device="cuda")
    s["block_table"][torch.arange(s["wide"], device="cuda") < _ints(held)[:, None]] = ids[:sum(held)]
    s["seq_lens"], s["lens_host"], s["batch"] = _ints(lens), lens, batch


def _prepare_chunk(case, s, gen, host):
    hq, hkv, d = HEADS[case["heads"]]
    dt, page = DTYPES[case["dtype"]], case["page"]
    s |= {"hq": hq, "hkv": hkv, "d": d}
    before, new = _lengths(case)
    lens = [a + b for a, b in zip(before, new)]
    _paged(case, s, gen, lens)
    s["pool"] = torch.zeros((s["num_pages"], hkv, page // 16 * _tile_bytes(d)), dtype=torch.uint8, device="cuda")
    _fill(s["pool"], d, gen, dt)
    seq = torch.repeat_interleave(torch.arange(case["batch"], device="cuda"), _ints(new).long())
    pos = torch.cat([torch.arange(a, n, device="cuda") for a, n in zip(before, lens)])
    s["slots"] = s["block_table"].long()[seq, pos // page] * page + pos % page
    s["k"], s["v"] = (torch.randn((sum(new), hkv, d), device="cuda", generator=gen).to(dt) for _ in range(2))
    # expanded pages lie in an order of their own
    s["dst_table"] = torch.full_like(s["block_table"], -1)
    live = s["block_table"] >= 0
    s["dst_table"][live] = torch.randperm(int(live.sum()), device="cuda", generator=gen).int()
    s["dst_pages"] = int(live.sum())
    s["k_pool"], s["v_pool"] = (torch.zeros((s["dst_pages"], page, hkv, d), dtype=dt, device="cuda") for _ in range(2))


def _prepare_step4(case, s, gen, host):
    hq, hkv, d = HEADS[case["heads"]]
    dt, page = DTYPES[case["dtype"]], case["page"]
    s |= {"hq": hq, "hkv": hkv, "d": d}
    lens, _ = _lengths(case)
    _paged(case, s, gen, lens)
    s["pool"] = torch.zeros((s["num_pages"], hkv, page // 16 * _tile_bytes(d)), dtype=torch.uint8, device="cuda")
    _fill(s["pool"], d, gen, dt)
    s["q"] = torch.randn((case["batch"], hq, d), device="cuda", generator=gen).to(dt)
    s["out"] = torch.zeros_like(s["q"])
    s["lse"] = torch.zeros((case["batch"], hq), dtype=torch.float32, device="cuda")


_PREPARE = {"tables": _prepare_tables, "rows": _prepare_rows, "chunk": _prepare_chunk, "step4": _prepare_step4}


def _prepare_own(case, s):
    from paper_2609_37062_b200 import binding as da
    s["da"] = da
    page = case["page"]
    if s["op"] == "tables":
        s["shape"] = da.make_shape(case["batch"], 8, 2, 64, page, s["wide"], s["num_pages"], (page * 128, 128, 64))
        return
    hq, hkv, d = s["hq"], s["hkv"], s["d"]
    kind = da.DA_DTYPE_FP16 if case["dtype"] == "fp16" else da.DA_DTYPE_BF16
    strides = (page * hkv * d, hkv * d, d)
    if s["op"] == "rows":
        s["shape"] = da.make_shape(0, hq, hkv, d, page, 0, s["num_pages"], strides, out_dtype=kind, in_dtype=kind)
        return
    s["shape"] = da.make_kv4_shape(case["batch"], hq, hkv, d, page, s["wide"], s["num_pages"], out_dtype=kind, in_dtype=kind)
    if s["op"] == "chunk":
        s["dst_shape"] = da.make_shape(case["batch"], hq, hkv, d, page, s["wide"], s["dst_pages"], strides,
                                       out_dtype=kind, in_dtype=kind)
        return
    s["plan"] = da.decode_attn_plan(s["shape"], da.make_policy(cache_bits=4), s["lens_host"])
    s["ws"] = torch.empty(max(s["plan"].workspace_bytes, 256), dtype=torch.uint8, device="cuda")


# ------------------------------------------------------------------------------------------------ one pass

def run(s):
    return _RUN[bool(own)][s["op"]](s)


def _own_tables(s):
    s["da"].decode_attn_step_tables(s["shape"], s["seq_lens"], s["gain"], s["seq_lens_out"], s["block_table"], s["free_pages"],
                                    s["free_count"], s["free_count_out"], s["row_starts"], s["page_starts"], s["slots"],
                                    s["positions"], s["row_seq"])
    return {"seq_lens": s["seq_lens_out"], "free_count": s["free_count_out"], "free_pages": s["free_pages"],
            "block_table": s["block_table"], "row_starts": s["row_starts"], "page_starts": s["page_starts"],
            "slots": s["slots"], "positions": s["positions"], "row_seq": s["row_seq"]}


def _own_rows(s):
    c = s["case"]
    s["da"].decode_attn_prepare_rows(s["shape"], s["q"], s["k"], s["v"], s["slots"], s["positions"], s["cos_sin"],
                                     q_out=s["q_out"], k_cache=s["k_pool"], v_cache=s["v_pool"], q_weight=s["q_weight"],
                                     k_weight=s["k_weight"], eps=EPS, interleaved=c["pairs"])
    return {"q": s["q_out"], "k": s["k_pool"], "v": s["v_pool"]}


def _own_chunk(s):
    da = s["da"]
    da.decode_attn_prepare_rows(s["shape"], None, s["k"], s["v"], s["slots"], k_cache=s["pool"], cache_bits=4)
    da.decode_attn_expand_kv(s["dst_shape"], s["shape"], s["pool"], s["block_table"], s["seq_lens"], s["dst_table"],
                              s["k_pool"], s["v_pool"])
    return {"k": s["k_pool"], "v": s["v_pool"]}


def _own_step4(s):
    da = s["da"]
    da.decode_attn_run(s["plan"], s["q"], s["pool"], None, s["block_table"], s["seq_lens"], s["out"], s["lse"], s["ws"])
    da.decode_attn_combine(s["plan"], s["ws"], s["out"], s["lse"])
    return {"out": s["out"], "lse": s["lse"]}


def _plain_tables(s):
    page, rows = s["page"], torch.arange(s["max_rows"], device="cuda")
    old, gain = s["seq_lens"].long(), s["gain"].long()
    new = (old + gain).clamp(min=0)
    held, holds = (old + page - 1) // page, (new + page - 1) // page
    pages = torch.arange(s["wide"], device="cuda")
    # what is given back goes on top of the list, in the order of the sequences and their positions
    back = (pages >= holds[:, None]) & (pages < held[:, None])
    spot = torch.cumsum(back.flatten().long(), 0).view(back.shape) - 1
    count = s["free_count"].long()
    s["free_pages"][(count + spot)[back]] = s["block_table"][back]
    full = count + back.sum()
    # what is needed is taken from the top
    take = (pages >= held[:, None]) & (pages < holds[:, None])
    spot = torch.cumsum(take.flatten().long(), 0).view(take.shape) - 1
    s["block_table"][take] = s["free_pages"][(full - 1 - spot)[take]]
    zero = torch.zeros(1, dtype=torch.int64, device="cuda")
    starts = torch.cat([zero, torch.cumsum(gain.clamp(min=0), 0)])
    page_starts = torch.cat([zero, torch.cumsum((holds - held).clamp(min=0), 0)])
    seq = torch.searchsorted(starts[1:], rows, right=True)
    live = seq < old.numel()
    seq = torch.where(live, seq, 0)
    pos = old[seq] + rows - starts[seq]
    at = torch.where(live, pos, 0)
    slots = s["block_table"].long()[seq, at // page] * page + at % page
    return {"seq_lens": new.int(), "free_count": (full - take.sum()).int(), "free_pages": s["free_pages"],
            "block_table": s["block_table"], "row_starts": starts.int(), "page_starts": page_starts.int(),
            "slots": torch.where(live, slots, -1), "positions": torch.where(live, pos, -1).int(),
            "row_seq": torch.where(live, seq, -1).int()}


def _plain_turn(s, x, weight):
    """Heads [n, heads, d] in 32 bits: normed and rotated."""
    c, half = s["case"], s["case"]["rotary"] // 2
    x = x.float()
    if weight is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * weight.float()
    turn = s["cos_sin"][s["positions"].long().clamp(min=0)][:, None]
    cos, sin = turn[..., :half], turn[..., half:]
    flat, rest = x[..., :2 * half], x[..., 2 * half:]
    a, b = (flat[..., 0::2], flat[..., 1::2]) if c["pairs"] else (flat[..., :half], flat[..., half:])
    a, b = a * cos - b * sin, b * cos + a * sin
    flat = torch.stack([a, b], -1).flatten(-2) if c["pairs"] else torch.cat([a, b], -1)
    return torch.cat([flat, rest], -1)


def _plain_rows(s):
    n, dt = s["case"]["rows"], s["q"].dtype                 # (the rows behind are padding: nothing is written for them)
    q = _plain_turn(s, s["q"], s["q_weight"]).to(dt)
    k = _plain_turn(s, s["k"], s["k_weight"]).to(dt)
    s["q_out"][:n] = q[:n]
    s["k_pool"].view(-1, *k.shape[1:])[s["slots"][:n]] = k[:n]
    s["v_pool"].view(-1, *k.shape[1:])[s["slots"][:n]] = s["v"][:n]
    return {"q": s["q_out"], "k": s["k_pool"], "v": s["v_pool"]}


def _plain_cached(s, pos):
    """K and V values of the logical positions pos [batch, n] in 32 bits: [batch, KV head, n, d]."""
    d, tile = s["d"], _tile_bytes(s["d"])
    at = _places(d, "cuda")
    page = s["block_table"].long().gather(1, pos // s["page"])
    # (batch, KV head, n): the tile of a position and the row of that tile
    tiles = (page[:, None] * s["hkv"] + torch.arange(s["hkv"], device="cuda")[None, :, None]) * (s["page"] // 16) + \
        (pos % s["page"] // 16)[:, None]
    row = (pos % 16)[:, None].expand_as(tiles)
    flat, words = s["pool"].view(-1), s["pool"].view(torch.float16).view(-1)
    read = lambda codes_at, scales_at: _decode(flat[tiles[..., None] * tile + codes_at[row]],
                                               words[tiles[..., None] * (tile // 2) + scales_at[row]])
    return read(at[0], at[2]), read(at[1], at[3])


def _plain_chunk(s):
    d, hkv, page, tile = s["d"], s["hkv"], s["page"], _tile_bytes(s["d"])
    at = _places(d, "cuda")
    tiles = ((s["slots"] // page)[:, None] * hkv + torch.arange(hkv, device="cuda")) * (page // 16) + \
        (s["slots"] % page // 16)[:, None]
    row = (s["slots"] % 16)[:, None].expand_as(tiles)
    flat, words = s["pool"].view(-1), s["pool"].view(torch.float16).view(-1)
    k_codes, k_scale = _encode(s["k"])
    v_codes, v_scale = _encode(s["v"])
    flat[tiles[..., None] * tile + at[0][row]] = k_codes
    flat[tiles[..., None] * tile + at[1][row]] = v_codes
    words[tiles[..., None] * (tile // 2) + at[2][row]] = k_scale
    words[tiles[..., None] * (tile // 2) + at[3][row]] = v_scale
    # every cached position, the last one in the place of those behind a sequence's end (not looked at)
    every = torch.arange(max(s["lens_host"]), device="cuda")
    live = every < s["seq_lens"].long()[:, None]
    pos = torch.where(live, every, s["seq_lens"].long()[:, None] - 1)
    k, v = _plain_cached(s, pos)
    slot = (s["dst_table"].long().gather(1, pos // page) * page + pos % page)[live]
    s["k_pool"].view(-1, hkv, d)[slot] = k.transpose(1, 2)[live].to(s["k_pool"].dtype)
    s["v_pool"].view(-1, hkv, d)[slot] = v.transpose(1, 2)[live].to(s["v_pool"].dtype)
    return {"k": s["k_pool"], "v": s["v_pool"]}


def _plain_step4(s):
    lens, g = s["seq_lens"].long()[:, None], s["hq"] // s["hkv"]
    every = torch.arange(max(s["lens_host"]), device="cuda")
    live = every < lens
    k, v = _plain_cached(s, torch.where(live, every, lens - 1))
    q = s["q"].float().view(s["batch"], s["hkv"], g, s["d"])
    x = torch.where(live[:, None, None], (q @ k.transpose(-1, -2)) / math.sqrt(s["d"]), float("-inf"))
    m = x.amax(-1, keepdim=True)
    p = torch.exp(x - m)
    total = p.sum(-1, keepdim=True)
    out = (p @ v) / total
    return {"out": out.reshape(s["out"].shape).to(s["out"].dtype), "lse": (m + torch.log(total)).reshape(s["lse"].shape)}


_RUN = {False: {"tables": _plain_tables, "rows": _plain_rows, "chunk": _plain_chunk, "step4": _plain_step4},
        True: {"tables": _own_tables, "rows": _own_rows, "chunk": _own_chunk, "step4": _own_step4}}


# ------------------------------------------------------------------------------------------------ the least work

def work(case):
    op = case["op"]
    if op == "tables":
        lens, gain = _lengths(case)
        page, batch = case["page"], case["batch"]
        after = [max(0, n + g) for n, g in zip(lens, gain)]
        moved = sum(abs(-(-m // page) - -(-n // page)) for n, m in zip(lens, after))
        rows = sum(max(0, g) for g in gain) + case["pad"]
        return {"bytes": batch * 20 + moved * 8 + rows * 16 + 16, "flops": 0}
    hq, hkv, d = HEADS[case["heads"]]
    if op == "rows":
        n = case["rows"]
        return {"bytes": n * ((hq + 2 * hkv) * d * 4 + 12) + min(n, case["far"]) * case["rotary"] * 4 +
                (4 * d if case["norm"] else 0), "flops": 0}
    row4 = hkv * _tile_bytes(d) // 16                                          # K and V of a token
    lens, new = _lengths(case)
    if op == "chunk":
        total, n = sum(lens) + sum(new), sum(new)
        return {"bytes": n * (hkv * d * 4 + 8 + row4) + total * (row4 + hkv * d * 4), "flops": 0}
    return {"bytes": sum(lens) * row4 + case["batch"] * hq * (4 * d + 4), "flops": 4 * d * hq * sum(lens)}


# ------------------------------------------------------------------------------------------------ 64 bits

def exact(case, seed):
    return _EXACT[case["op"]](prepare(case, seed))


def _exact_tables(s):
    """Sequence by sequence and page by page, with a list that is a list."""
    page, table = s["page"], s["block_table"].cpu().tolist()
    stack = s["free_pages"].cpu().tolist()
    lens, gain = s["seq_lens"].cpu().tolist(), s["gain"].cpu().tolist()
    count = int(s["free_count"])
    after = [max(0, n + g) for n, g in zip(lens, gain)]
    for b, (n, m) in enumerate(zip(lens, after)):
        for i in range(-(-m // page), -(-n // page)):
            stack[count] = table[b][i]
            count += 1
    starts, page_starts, slots, positions, seqs = [0], [0], [], [], []
    for b, (n, m) in enumerate(zip(lens, after)):
        first = -(-n // page)
        for i in range(first, -(-m // page)):
            count -= 1
            table[b][i] = stack[count]
        for p in range(n, m):
            slots.append(table[b][p // page] * page + p % page)
            positions.append(p)
            seqs.append(b)
        starts.append(starts[-1] + max(0, m - n))
        page_starts.append(page_starts[-1] + max(0, -(-m // page) - first))
    rest = [-1] * (s["max_rows"] - len(slots))
    return {"seq_lens": _ints(after), "free_count": _ints([count]), "free_pages": _ints(stack), "block_table": _ints(table),
            "row_starts": _ints(starts), "page_starts": _ints(page_starts), "slots": _ints(slots + rest, torch.int64),
            "positions": _ints(positions + rest), "row_seq": _ints(seqs + rest)}


def _exact_rows(s):
    c, n, d = s["case"], s["case"]["rows"], s["d"]
    half = c["rotary"] // 2
    first = torch.arange(half, device="cuda") * (2 if c["pairs"] else 1)
    second = first + (1 if c["pairs"] else half)
    turn = s["cos_sin"].double()[s["positions"][:n].long()]
    out = []
    for x, w in ((s["q"][:n], s["q_weight"]), (s["k"][:n], s["k_weight"])):
        x = x.double()
        if w is not None:
            x = x / torch.sqrt(x.square().sum(-1, keepdim=True) / d + EPS) * w.double()
        z = torch.complex(x[..., first], x[..., second]) * torch.complex(turn[:, :half], turn[:, half:])[:, None]
        x = x.clone()
        x[..., first], x[..., second] = z.real, z.imag
        out.append(x)
    q, k, v = (torch.zeros(s[name].shape, dtype=torch.float64, device="cuda") for name in ("q_out", "k_pool", "v_pool"))
    q[:n] = out[0]
    page, slot = s["slots"][:n] // s["page"], s["slots"][:n] % s["page"]
    k[page, slot] = out[1]
    v[page, slot] = s["v"][:n].double()
    return {"q": q, "k": k, "v": v}


def _exact_tile(tile, d, which):
    """Tiles of one head [n, bytes] to values [n, 16, d] in 64 bits, a dim at a time: nothing is taken from the plain form."""
    size = torch.tensor([0, 1, 2, 3, 4, 6, 8, 12], dtype=torch.float64, device="cuda") / 2
    out = torch.zeros((tile.shape[0], 16, d), dtype=torch.float64, device="cuda")
    scales = tile[:, 16 * d:].contiguous().view(torch.float16).double()
    nb, rows = d // 32, torch.arange(16, device="cuda")
    for x in range(d):
        if which == "k":
            byte = rows * (d // 2) + x % 32 // 8 * 4 * nb + x // 32 * 4 + x % 8 // 2
            scale = scales[:, rows * nb + x // 32]
        else:
            byte = 8 * d + rows * (d // 2) + x // 2
            if d == 128:
                byte = byte + torch.where(rows >= 8, 32 if x // 2 % 64 < 32 else -32, 0)
            scale = scales[:, 16 * nb + x // 32 * 16 + rows // 4 * 4 + torch.bitwise_xor(rows % 4, rows // 4)]
        code = tile[:, byte] >> (4 * (x % 2)) & 15
        out[..., x] = size[(code & 7).long()] * torch.where(code > 7, -1.0, 1.0) * scale
    return out


def _exact_quantised(x):
    """Rows [n, hkv, d] to the values that 4 bits hold of them, by the distance to every magnitude."""
    size = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device="cuda")
    y = x.double().unflatten(-1, (-1, 32))
    scale = (y.abs().amax(-1, keepdim=True) / 6).half().double()
    away = (y.abs() / torch.where(scale > 0, scale, 1.0))[..., None] - size
    # the nearest, and of two equally near the one with the even code (the even codes first: the first minimum wins)
    order = torch.tensor([0, 2, 4, 6, 1, 3, 5, 7], device="cuda")
    return (size[order][away.abs()[..., order].argmin(-1)] * y.sign() * scale).flatten(-2)


def _exact_chunk(s):
    d, hkv, page = s["d"], s["hkv"], s["page"]
    fresh = {"k": _exact_quantised(s["k"]), "v": _exact_quantised(s["v"])}
    out = {n: torch.zeros(s[n + "_pool"].shape, dtype=torch.float64, device="cuda") for n in ("k", "v")}
    tiles = s["pool"].view(s["num_pages"], hkv, page // 16, -1)
    for b, n in enumerate(s["lens_host"]):
        at = torch.arange(n, device="cuda")
        src = s["block_table"][b].long()[:-(-n // page)]
        dst = s["dst_table"][b].long()[at // page]
        flat = tiles[src].transpose(1, 2).flatten(0, 2)                        # [tile, head]
        for name in ("k", "v"):
            rows = _exact_tile(flat, d, name).view(-1, hkv, 16, d).transpose(1, 2).flatten(0, 1)
            out[name][dst, at % page] = rows[:n]
    # the new rows lie where their slots say, in the expanded pages' order
    where = torch.full((s["num_pages"],), -1, dtype=torch.int64, device="cuda")
    live = s["block_table"] >= 0
    where[s["block_table"][live].long()] = s["dst_table"][live].long()
    for name in ("k", "v"):
        out[name][where[s["slots"] // page], s["slots"] % page] = fresh[name]
    return out


def _exact_step4(s):
    if sum(s["lens_host"]) * s["hkv"] > 20_000_000:
        return None
    g, page, d = s["hq"] // s["hkv"], s["page"], s["d"]
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device="cuda")
    tiles = s["pool"].view(s["num_pages"], s["hkv"], page // 16, -1)
    for b, n in enumerate(s["lens_host"]):
        src = s["block_table"][b].long()[:-(-n // page)]
        flat = tiles[src].transpose(0, 1).flatten(0, 2)                        # [head, tile]
        k, v = (_exact_tile(flat, d, name).view(s["hkv"], -1, d)[:, :n] for name in ("k", "v"))
        x = s["q"][b].double().view(s["hkv"], g, d) @ k.transpose(1, 2) / math.sqrt(d)
        e = torch.logsumexp(x, -1)
        lse[b] = e.view(-1)
        out[b] = (torch.exp(x - e[..., None]) @ v).view(-1, d)
    return {"out": out, "lse": lse}


_EXACT = {"tables": _exact_tables, "rows": _exact_rows, "chunk": _exact_chunk, "step4": _exact_step4}
