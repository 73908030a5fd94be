"""Capacity plans of a cache in 4 bits, refreshed and replayed from a graph: fused or not, with windows, masks and limits on pieces."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from packed_util import Cache, check, da  # noqa: E402

WIDE, PAGES, ROWS = 60, 120, 6


@pytest.mark.parametrize("fuse", [0, 1])
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (24, 2, 64), (8, 8, 64)])
@pytest.mark.parametrize("kw", [{}, {"window_tokens": 300, "sink_tokens": 20}, {"split_mode": da.DA_SPLIT_FIXED_COUNT, "fixed_count": 4},
                                {"max_splits": 2, "chunk_tokens": 32}, {"split_mode": da.DA_SPLIT_DETERMINISTIC, "chunk_tokens": 64}])
def test_refreshed_and_replayed(fuse, hq, hkv, d, kw):
    steps = [[40, 900, 3], [500, 0, 17, 333, 1, 64], [], [16], [700, 710]]
    window, sinks = kw.get("window_tokens", 0), kw.get("sink_tokens", 0)
    caches = [Cache(lens, hq, hkv, d, seed=len(lens) + fuse, width=WIDE) for lens in steps if lens]
    for c in caches:
        c.pool, c.num_pages = np.pad(c.pool, ((0, PAGES - len(c.pool)), (0, 0), (0, 0)), constant_values=0xff), PAGES
    policy = da.make_policy(cache_bits=4, capacity_batch=ROWS, capacity_tokens=2000, fuse_combine=fuse, **kw)
    plan = da.decode_attn_plan(caches[0].shape(), policy, caches[0].lens)
    pool = torch.zeros((PAGES, hkv, caches[0].pool.shape[2]), dtype=torch.uint8, device="cuda")
    table, lens = torch.full((ROWS, WIDE), -1, dtype=torch.int32, device="cuda"), torch.zeros(ROWS, dtype=torch.int32, device="cuda")
    mask = torch.ones(ROWS, dtype=torch.uint8, device="cuda")
    q = torch.zeros((ROWS, hq, d), dtype=torch.bfloat16, device="cuda")
    out, lse = torch.zeros((ROWS, hq, d), device="cuda"), torch.zeros((ROWS, hq), device="cuda")
    ws = torch.full((plan.workspace_bytes,), 0xff, dtype=torch.uint8, device="cuda")

    def step():
        da.decode_attn_run(plan, q, pool, None, table, lens, out, lse, ws, run_mask=mask)
        if not fuse:
            da.decode_attn_combine(plan, ws, out, lse)

    def load(c, dead):
        n = len(c.lens)
        pool.copy_(torch.from_numpy(c.pool))
        table[:n].copy_(torch.from_numpy(c.table))
        lens[:n].copy_(torch.tensor(c.lens, dtype=torch.int32))
        q[:n].copy_(c.q)
        mask.fill_(1)
        mask[list(dead)] = 0
        out.fill_(float("nan"))
        lse.fill_(float("nan"))

    load(caches[0], ())
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step()
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i, wanted in enumerate(steps + [steps[1], steps[0]]):
        if not wanted:                                        # nothing is live: nothing is written
            out.fill_(float("nan"))
            da.decode_attn_plan_update(plan, [])
            graph.replay()
            assert torch.isnan(out).all()
            continue
        c = next(c for c in caches if c.lens == wanted)
        dead = (len(wanted) - 1,) if i % 2 else ()
        load(c, dead)
        da.decode_attn_plan_update(plan, c.lens)
        graph.replay()
        assert da.decode_attn_last_device_status(plan) == da.DA_OK
        n = len(wanted)
        check(c, out[:n], lse[:n], f"step {i}", window=window, sinks=sinks, dead=dead)
        assert torch.isnan(out[n:]).all() and torch.isnan(lse[n:]).all()
    del graph
    plan.destroy()
