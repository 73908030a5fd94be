"""Repeated calls over a cache in 4 bits repeat their bits, whatever the plan: back to back on one stream, with other inputs between."""
import functools
import random

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from packed_util import KINDS, Cache, da  # noqa: E402

SIZES = {"one": ([2600], 8, 2), "uneven": ([30, 300, 160, 17, 200] * 8, 16, 4), "wide": ([1, 800, 300, 0], 24, 2)}


@functools.cache
def caches(size, dtype):
    lens, hq, hkv = SIZES[size]
    return [Cache(lens, hq, hkv, 64 if size == "uneven" else 128, dtype=dtype, seed=s) for s in (1, 2)]


@pytest.mark.parametrize("size", list(SIZES))
@pytest.mark.parametrize("dtype,out,kw", [("bf16", "bf16", {}), ("fp16", "fp16", {}), ("bf16", "fp32", {"fuse_combine": 1}),
                                          ("bf16", "fp32", {"window_tokens": 400, "sink_tokens": 4}),
                                          ("fp16", "fp32", {"split_mode": da.DA_SPLIT_FIXED_COUNT, "fixed_count": 5})])
def test_same_bits(size, dtype, out, kw):
    lens, (a, b) = SIZES[size][0], caches(size, dtype)
    plan = da.decode_attn_plan(a.shape(out), da.make_policy(cache_bits=4, **kw), lens)
    ws = torch.empty(max(plan.workspace_bytes, 256), dtype=torch.uint8, device="cuda")
    sides = []
    for c in (a, b):
        dev = [torch.from_numpy(c.pool).cuda(), torch.from_numpy(c.table).cuda(), c.q.cuda()]
        sides.append(dev)
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    rng = random.Random(size)
    results = [[], []]
    ws.fill_(0xff)
    for i in range(24):
        side = rng.randrange(2) if i > 1 else i
        pool, table, q = sides[side]
        o = torch.full(a.q.shape, float("nan"), dtype=KINDS[out][1], device="cuda")
        lse = torch.full(a.q.shape[:2], float("nan"), device="cuda")
        da.decode_attn_run(plan, q, pool, None, table, n, o, lse, ws)
        if not kw.get("fuse_combine"):
            da.decode_attn_combine(plan, ws, o, lse)
        results[side].append((o, lse))
    assert da.decode_attn_last_device_status(plan) == da.DA_OK
    plan.destroy()
    for side in results:
        for o, lse in side[1:]:
            assert torch.equal(o, side[0][0]) and torch.equal(lse, side[0][1])
    assert not torch.equal(results[0][0][0], results[1][0][0])
