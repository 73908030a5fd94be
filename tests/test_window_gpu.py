"""Sliding window with sinks, one new token per sequence, against the fp64 oracle.  Everything the query may not see is
poisoned: NaN in the hidden slots of visible pages, -1 in the block table where a page holds nothing visible."""
import numpy as np
import pytest
import torch

from bounded_util import Step, hide, oracle_out
from gpu_util import assert_parity, da, to_device
from paper_2609_37062_b200 import workloads as wl

pytestmark = pytest.mark.gpu

LENS = [0, 1, 15, 16, 17, 31, 33, 64, 100, 255, 257, 300, 1000, 1025, 2500]


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (16, 4), (17, 16), (100, 37), (256, 4), (777, 200), (4000, 4)])
@pytest.mark.parametrize("hq,hkv,d,dtype", [(8, 2, 64, "bf16"), (32, 8, 128, "fp16"), (10, 2, 128, "bf16"), (24, 2, 64, "bf16")])
def test_window_and_sinks(hq, hkv, d, dtype, window, sinks):
    w = hide(wl.make_workload("win", LENS, hq, hkv, d, seed=31, dtype=dtype), [1] * len(LENS), window, sinks)
    ref, ref_lse, _ = oracle_out(w, window=window, sinks=sinks)
    wd = to_device(w)
    for pol in (dict(), dict(split_mode=da.DA_SPLIT_DETERMINISTIC, chunk_tokens=32), dict(fuse_combine=1, chunk_tokens=64),
                dict(split_mode=da.DA_SPLIT_FIXED_COUNT, fixed_count=3)):
        s = Step(wd, da.make_policy(window_tokens=window, sink_tokens=sinks, **pol))
        out, lse = s()
        s.ok()
        assert_parity(out, lse, ref, ref_lse, str(pol))


@pytest.mark.parametrize("page_size", [32, 64, 256])
@pytest.mark.parametrize("layout", ["token_major", "head_major"])
def test_page_sizes_and_layouts(page_size, layout):
    window, sinks = 300, 20
    w = hide(wl.make_workload("winp", LENS, 16, 4, 128, seed=32, page_size=page_size, layout=layout), [1] * len(LENS), window, sinks)
    ref, ref_lse, _ = oracle_out(w, window=window, sinks=sinks)
    s = Step(to_device(w), da.make_policy(window_tokens=window, sink_tokens=sinks))
    out, lse = s()
    s.ok()
    assert_parity(out, lse, ref, ref_lse)


def test_run_mask_and_new_rows():
    """A masked row reads nothing and emits zero but still writes its K/V; the fused write equals write-then-attend."""
    window, sinks, B = 200, 4, len(LENS)
    w = wl.make_workload("wina", LENS, 32, 8, 128, seed=33)
    new = [wl.normal_bf16_bits(wl.stream_key(33, t, 0), 0, B * 8 * 128).view(B, 8, 128).cuda() for t in (wl.TENSOR_NEW_K, wl.TENSOR_NEW_V)]
    mask = torch.tensor([i % 3 != 1 for i in range(B)], dtype=torch.uint8, device="cuda")
    got = []
    for fused in (False, True):
        wd = to_device(w)
        s = Step(wd, da.make_policy(window_tokens=window, sink_tokens=sinks))
        if fused:
            s(run_mask=mask, new_k=new[0], new_v=new[1])
        else:
            da.decode_attn_append_kv(s.shape, *new, wd.block_table, wd.seq_lens, wd.k_pool, wd.v_pool)
            s(run_mask=mask)
        s.ok()
        got.append((s.out, s.lse, wd.k_pool, wd.v_pool))
    assert all(torch.equal(a, b) for a, b in zip(*got))
    import dataclasses
    after = dataclasses.replace(w, k_pool=got[1][2].cpu(), v_pool=got[1][3].cpu())
    ref, ref_lse, _ = oracle_out(after, window=window, sinks=sinks, run_mask=mask.cpu().numpy())
    assert_parity(got[1][0], got[1][1], ref, ref_lse)


def test_deterministic_bits_do_not_depend_on_the_batch():
    pol = da.make_policy(split_mode=da.DA_SPLIT_DETERMINISTIC, window_tokens=1500, sink_tokens=4)
    lens = [5000, 77, 3001]
    many = Step(to_device(wl.make_workload("wind", lens, 32, 8, 128, seed=34)), pol)
    many()
    for b, L in enumerate(lens):
        one = Step(to_device(wl.make_workload("wind", [L], 32, 8, 128, seed=34, seq_uids=[b])), pol)
        one()
        assert torch.equal(one.out[0], many.out[b]) and torch.equal(one.lse[0], many.lse[b])


def test_a_window_that_hides_nothing_changes_no_bit():
    w = to_device(wl.make_workload("winf", LENS, 32, 8, 128, seed=35))
    a, b = Step(w, da.make_policy()), Step(w, da.make_policy(window_tokens=2500, sink_tokens=4))
    a(), b()
    assert torch.equal(a.out, b.out) and torch.equal(a.lse, b.lse)


def test_capacity_plan_replayed_from_a_graph():
    """One captured graph, refreshed for other lengths and batches; rows behind the live batch stay as they were."""
    window, sinks = 300, 4
    pol = da.make_policy(capacity_batch=6, capacity_tokens=9000, window_tokens=window, sink_tokens=sinks)
    w = wl.make_workload("winc", [2000, 10, 900, 333, 301, 1500], 8, 2, 128, seed=36)
    wd = to_device(w)
    s = Step(wd, pol)
    lens_dev = wd.seq_lens.clone()
    run = lambda: (da.decode_attn_run(s.plan, wd.q_bits, wd.k_pool, wd.v_pool, wd.block_table, lens_dev, s.out, s.lse, s.ws),
                   da.decode_attn_combine(s.plan, s.ws, s.out, s.lse))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for lens in ([2000, 10, 900, 333, 301, 1500], [1999, 1, 300, 16], [0, 5, 850, 299, 77, 1200]):
        da.decode_attn_plan_update(s.plan, lens)
        lens_dev[:len(lens)] = torch.tensor(lens, dtype=torch.int32, device="cuda")
        s.out.fill_(7.0), s.lse.fill_(7.0)
        graph.replay()
        s.ok()
        import dataclasses
        n = len(lens)
        cut = dataclasses.replace(w, batch=n, seq_lens=torch.tensor(lens, dtype=torch.int32), block_table=w.block_table[:n], q_bits=w.q_bits[:n])
        ref, ref_lse, _ = oracle_out(cut, window=window, sinks=sinks)
        assert_parity(s.out[:n], s.lse[:n], ref, ref_lse, str(lens))
        assert (s.out[n:] == 7).all() and (s.lse[n:] == 7).all()


def test_bad_pages_and_stale_lengths_are_reported():
    w = wl.make_workload("wins", [2000, 500], 32, 8, 128, seed=37)
    wd = to_device(w)
    s = Step(wd, da.make_policy(window_tokens=256, sink_tokens=4))
    wd.block_table[0, 60] = 1 << 29                          # hidden: position 960 of 2000
    s()
    s.ok()
    wd.block_table[0, 120] = wd.num_pages                    # visible: position 1920
    s()
    assert da.decode_attn_last_device_status(s.plan) == da.DA_ERR_BAD_PAGE
    wd.block_table.copy_(w.block_table)
    wd.seq_lens[1] = 499
    s()
    assert da.decode_attn_last_device_status(s.plan) == da.DA_ERR_STALE_PLAN
    assert (s.out[1] == 0).all()


def test_helpers_that_know_no_window_refuse():
    w = to_device(wl.make_workload("winh", [2000], 32, 8, 128, seed=38))
    plan = da.decode_attn_plan(da.shape_of_workload(w), da.make_policy(window_tokens=256), w.seq_lens)
    buf = torch.empty((2000, 8, 128), dtype=torch.int16, device="cuda")
    for call in (lambda: da.decode_attn_debug_gather(plan, 0, w.k_pool, w.v_pool, w.block_table, buf, buf),
                 lambda: da.decode_attn_gather_probe(plan, w.k_pool, w.v_pool, w.block_table, buf)):
        with pytest.raises(da.DecodeAttnError) as e:
            call()
        assert e.value.status == da.DA_ERR_UNSUPPORTED
