"""Eviction by attention weight against the oracle: which positions stay (equal), where their rows and totals go (bit
for bit), and that nothing else is written."""
import numpy as np
import pytest
import torch

from bounded_util import Step, oracle_out
from gpu_util import assert_parity, da, to_device
from oracle import bounded_cache as bc
from paper_2609_37062_b200 import workloads as wl

pytestmark = pytest.mark.gpu

LENS = [0, 1, 16, 127, 128, 129, 130, 300, 1000, 4999]


def totals(kind, shape, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.exp(2 * torch.randn(shape, generator=g) - 3)
    if kind == "equal":
        x = torch.full(shape, 0.25)
    elif kind == "zeros":                                     # ties at both zeros, a few totals above them
        x = torch.where(torch.rand(shape, generator=g) < 0.01, x, torch.where(torch.rand(shape, generator=g) < 0.5, 0.0, -0.0))
    elif kind == "steps":                                     # many ties at every value
        x = (x * 4).round() / 4
    elif kind == "any":                                       # any bits: both signs, infinities, NaN, denormals
        x = torch.randint(-2**31, 2**31 - 1, shape, generator=g, dtype=torch.int64).to(torch.int32).view(torch.float32)
        x[..., ::7] = float("inf")
        x[..., 3::11] = float("-inf")
        x[..., 5::13] = float("nan")
    return x


def fresh_pages(w, budget):
    """Destination pages: ids that no sequence holds, in a shuffled order."""
    n = -(-budget // w.page_size)
    held = set(w.block_table[w.block_table >= 0].tolist())
    free = [p for p in range(w.num_pages) if p not in held]
    assert len(free) >= n * w.batch
    g = torch.Generator().manual_seed(5)
    pick = torch.tensor(free)[torch.randperm(len(free), generator=g)[:n * w.batch]]
    return pick.view(w.batch, n).to(torch.int32)


def workload(lens, budget, hq, hkv, d, seed=51, page_size=16, **kw):
    need = sum(-(-n // page_size) for n in lens) + len(lens) * -(-budget // page_size)
    return wl.make_workload("ev", lens, hq, hkv, d, seed=seed, page_size=page_size, pool_pages=need + 3, **kw)


def run(w, dst, budget, sinks, recent, t, in_place, status=None):
    wd = to_device(w)
    before = t.cuda()
    after = before if in_place else torch.full_like(before, 7.0)
    kept = torch.full((w.batch, w.num_kv_heads, budget), -7, dtype=torch.int32, device="cuda")
    lens_out = torch.full((w.batch,), -7, dtype=torch.int32, device="cuda")
    da.decode_attn_evict(da.shape_of_workload(wd), budget, sinks, recent, wd.seq_lens, wd.block_table, dst.cuda(), wd.k_pool,
                         wd.v_pool, before, after, kept, lens_out, status)
    torch.cuda.synchronize()
    return wd, after.cpu(), kept.cpu().numpy(), lens_out.cpu().numpy()


def check(w, dst, budget, sinks, recent, t, in_place):
    wd, after, kept, lens_out = run(w, dst, budget, sinks, recent, t, in_place)
    k, v = w.k_pool.clone(), w.v_pool.clone()
    expect = (t if in_place else torch.full_like(t, 7.0)).clone()
    P = w.page_size
    for b, L in enumerate(w.seq_lens.tolist()):
        assert lens_out[b] == min(L, budget)
        for g in range(w.num_kv_heads):
            stay = bc.kept_positions(t[b, g].numpy(), L, budget, sinks, recent)
            n = len(stay)
            assert n == min(L, budget)
            assert np.array_equal(kept[b, g, :n], stay), (b, g)
            assert (kept[b, g, n:] == -1).all()
            s = torch.from_numpy(stay).long()
            expect[b, g, :L] = 0
            expect[b, g, :n] = t[b, g, s]
            if L > budget:
                page, slot = w.block_table[b, s // P].long(), s % P
                to, to_slot = dst[b, torch.arange(n) // P].long(), torch.arange(n) % P
                for pool in (k, v):
                    if w.layout == "token_major":
                        pool[to, to_slot, g] = pool[page, slot, g]
                    else:
                        pool[to, g, to_slot] = pool[page, g, slot]
    assert torch.equal(after.view(torch.int32), expect.view(torch.int32))     # bits: NaN, and both zeros
    assert torch.equal(wd.k_pool.cpu(), k) and torch.equal(wd.v_pool.cpu(), v)


@pytest.mark.parametrize("kind", ["random", "equal", "zeros", "steps", "any"])
@pytest.mark.parametrize("budget,sinks,recent", [(128, 4, 32), (1, 0, 0), (1, 1, 0), (1, 0, 1), (129, 0, 0), (128, 64, 64),
                                                 (300, 37, 0), (999, 4, 500)])
def test_what_stays(kind, budget, sinks, recent):
    for lens in (LENS, LENS[:-1]):                            # large blocks and a launch of its own for the moves; small ones that move
        w = workload(lens, budget, 8, 2, 64)
        t = totals(kind, (len(lens), 2, max(lens) + 5), seed=budget)
        dst = fresh_pages(w, budget)
        for in_place in (False, True):
            check(w, dst, budget, sinks, recent, t, in_place)


@pytest.mark.parametrize("layout", ["token_major", "head_major"])
@pytest.mark.parametrize("page_size", [16, 64, 256])
@pytest.mark.parametrize("hq,hkv,d,dtype", [(32, 8, 128, "bf16"), (10, 5, 64, "fp16"), (3, 1, 128, "fp16")])
def test_pages_heads_and_layouts(layout, page_size, hq, hkv, d, dtype):
    lens, budget = [700, 90, 401, 400], 400
    w = workload(lens, budget, hq, hkv, d, page_size=page_size, layout=layout, dtype=dtype)
    check(w, fresh_pages(w, budget), budget, 4, 100, totals("random", (4, hkv, 700), 3), False)


@pytest.mark.parametrize("d,budget", [(128, 700), (128, 300), (64, 1500), (64, 300)])
def test_rows_of_some_thousand(d, budget):
    """Blocks of 512 threads: moving by themselves and not."""
    lens = [4000, 2049, 90, 1501]
    w = workload(lens, budget, 8, 4, d, seed=57)
    for in_place in (False, True):
        check(w, fresh_pages(w, budget), budget, 4, 100, totals("steps", (4, 4, 4000), 5), in_place)


def test_rows_longer_than_a_block_holds():
    """Longer rows are shared by a cluster of blocks, the longest walked in runs; compaction in place is the
    delicate case."""
    for lens, budget in (([9000, 4097, 300], 4000), ([49152], 5000), ([49153, 120_000], 100_001), ([100_000], 60_000),
                         ([400_001, 9], 300_000)):
        w = workload(lens, budget, 2, 1, 64, seed=52, page_size=256)
        for kind in ("random", "steps", "equal"):
            t = totals(kind, (len(lens), 1, max(lens)), 9)
            check(w, fresh_pages(w, budget), budget, 4, 1000, t, True)


def test_a_shared_prefix_stays_whole():
    """Rows that share pages: each moves to pages of its own, the shared ones are not touched."""
    lens, budget = [640, 700, 800], 256
    P = 16
    w = wl.make_workload("evs", lens, 8, 2, 64, seed=53, shared_prefix_tokens=512, pool_pages=32 + 40 + 3 * 16)
    check(w, fresh_pages(w, budget), budget, 4, 64, totals("random", (3, 2, 800), 4), False)


def test_bad_pages_and_lengths_are_reported_and_touch_nothing():
    lens, budget = [300, 400], 128
    w = workload(lens, budget, 8, 2, 64, seed=54)
    t = totals("random", (2, 2, 400), 6)
    dst = fresh_pages(w, budget)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    run(w, dst, budget, 4, 32, t, False, status)
    assert int(status) == da.DA_OK
    bad = dst.clone()
    bad[0, 3] = w.num_pages
    wd, _, kept, _ = run(w, bad, budget, 4, 32, t, False, status)
    assert int(status) == da.DA_ERR_BAD_PAGE
    good = run(w, dst, budget, 4, 32, t, False)[0]
    same = torch.ones(w.num_pages, dtype=torch.bool)
    same[dst[0, 3].long()] = False                            # the page that was not reached; all others as they should be
    assert torch.equal(wd.k_pool.cpu()[same], good.k_pool.cpu()[same])
    # longer than the totals, longer than the table, negative
    import dataclasses
    for n in (401, 1 << 20, -5):
        status.zero_()
        wrong = dataclasses.replace(w, seq_lens=torch.tensor([300, n], dtype=torch.int32))
        wd, after, kept, lens_out = run(wrong, dst, budget, 4, 32, t, False, status)
        assert int(status) == da.DA_ERR_STALE_PLAN
        assert lens_out.tolist() == [128, n] and (kept[1] == -1).all() and (after[1] == 7).all()
        assert torch.equal(wd.k_pool.cpu()[dst[1].long()], w.k_pool[dst[1].long()])


def test_a_bounded_generation():
    """Steps that track weights, an eviction, and steps on the shorter cache, all against the oracle."""
    import dataclasses
    lens, budget = [500, 260], 256
    w = workload([n + 1 for n in lens], budget + 16, 32, 8, 128, seed=55)
    w = dataclasses.replace(w, seq_lens=torch.tensor(lens, dtype=torch.int32))
    wd = to_device(w)
    t = torch.zeros((2, 8, 501), device="cuda")
    expect = [np.zeros((8, n + 1)) for n in lens]
    for n_more in (0, 1):
        cur = dataclasses.replace(w, seq_lens=torch.tensor([n + n_more for n in lens], dtype=torch.int32))
        s = Step(to_device(cur), da.make_policy(track_weights=1))
        s()
        da.decode_attn_add_weights(s.plan, s.ws, s.lse, s.w.seq_lens, t)
        s.ok()
        for b, x in enumerate(oracle_out(cur)[2]):
            expect[b][:, :x.shape[1]] += x
    for b, e in enumerate(expect):
        assert (np.abs(t[b, :, :e.shape[1]].cpu().double().numpy() - e) <= 4e-4 * e + 1e-7).all()
    w = cur
    wd = to_device(w)
    dst = fresh_pages(w, budget + 16)
    kept = torch.empty((2, 8, budget), dtype=torch.int32, device="cuda")
    lens_out = torch.empty(2, dtype=torch.int32, device="cuda")
    host_totals = t.cpu().numpy()
    assert da.decode_attn_validate_evict(da.shape_of_workload(wd), budget, 4, 64, w.seq_lens, w.block_table, dst) == da.DA_OK
    da.decode_attn_evict(da.shape_of_workload(wd), budget, 4, 64, wd.seq_lens, wd.block_table, dst.cuda(), wd.k_pool, wd.v_pool,
                         t, None, kept, lens_out)
    # the next step over the kept tokens: the oracle attends over each KV head's own selection
    new_bt = torch.full_like(w.block_table, -1)
    new_bt[:, :dst.shape[1]] = dst
    small = dataclasses.replace(w, k_pool=wd.k_pool.cpu(), v_pool=wd.v_pool.cpu(), seq_lens=lens_out.cpu(), block_table=new_bt)
    s = Step(to_device(small), da.make_policy(track_weights=1))
    out, lse = s()
    s.ok()
    ref, ref_lse, _ = oracle_out(small)
    assert_parity(out, lse, ref, ref_lse)
    for b in range(2):
        for g in range(8):
            stay = bc.kept_positions(host_totals[b, g], int(w.seq_lens[b]), budget, 4, 64)
            assert np.array_equal(kept[b, g].cpu().numpy(), stay)
            q = w.q_bits[b, g * 4].view(torch.bfloat16).double()
            s2 = torch.from_numpy(stay).long()
            pg, sl = w.block_table[b, s2 // 16].long(), s2 % 16
            k = w.k_pool[pg, sl, g].view(torch.bfloat16).double()
            v = w.v_pool[pg, sl, g].view(torch.bfloat16).double()
            o = torch.softmax(k @ q / 128 ** 0.5, 0) @ v
            assert (out[b, g * 4].cpu().double() - o).abs().max() < 2e-3


def test_destination_tables_that_are_columns_of_wider_ones():
    lens, budget = [300, 400], 128
    w = workload(lens, budget, 8, 2, 64, seed=58)
    wd, dst = to_device(w), fresh_pages(w, budget)
    wide = torch.full((2, 20), -1, dtype=torch.int32, device="cuda")
    wide[:, :8] = dst.cuda()
    t = totals("random", (2, 2, 400), 8).cuda()
    out = []
    for table in (dst.cuda(), wide[:, :8], wide):
        x = to_device(w)
        kept = torch.zeros((2, 2, budget), dtype=torch.int32, device="cuda")
        lens_out = torch.zeros(2, dtype=torch.int32, device="cuda")
        da.decode_attn_evict(da.shape_of_workload(x), budget, 4, 32, x.seq_lens, x.block_table, table, x.k_pool, x.v_pool, t,
                             torch.zeros_like(t), kept, lens_out)
        out.append((x.k_pool, x.v_pool, kept))
    for o in out[1:]:
        assert all(torch.equal(a, b) for a, b in zip(o, out[0]))
    kept = torch.zeros((2, 2, budget), dtype=torch.int32, device="cuda")
    for table in (dst[:, :7].cuda(), wide.t().contiguous().t()):               # too few pages; pages not next to each other
        with pytest.raises(da.DecodeAttnError):
            da.decode_attn_evict(da.shape_of_workload(wd), budget, 4, 32, wd.seq_lens, wd.block_table, table, wd.k_pool, wd.v_pool, t,
                                 torch.zeros_like(t), kept, torch.zeros(2, dtype=torch.int32, device="cuda"))


def test_captured_and_replayed():
    lens, budget = [300, 400, 50], 128
    w = workload(lens, budget, 8, 2, 64, seed=56)
    wd = to_device(w)
    dst = fresh_pages(w, budget).cuda()
    t = totals("random", (3, 2, 400), 8).cuda()
    after = torch.zeros_like(t)
    kept = torch.zeros((3, 2, budget), dtype=torch.int32, device="cuda")
    lens_out = torch.zeros(3, dtype=torch.int32, device="cuda")
    call = lambda: da.decode_attn_evict(da.shape_of_workload(wd), budget, 4, 32, wd.seq_lens, wd.block_table, dst, wd.k_pool,
                                        wd.v_pool, t, after, kept, lens_out)
    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for lens in ([300, 400, 50], [129, 128, 3], [0, 399, 50]):
        wd.seq_lens.copy_(torch.tensor(lens, dtype=torch.int32))
        t.copy_(totals("steps", (3, 2, 400), sum(lens)))
        graph.replay()
        for b, L in enumerate(lens):
            assert int(lens_out[b]) == min(L, budget)
            for g in range(2):
                stay = bc.kept_positions(t[b, g].cpu().numpy(), L, budget, 4, 32)
                assert np.array_equal(kept[b, g, :len(stay)].cpu().numpy(), stay)
