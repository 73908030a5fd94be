"""RUN masks on windowed plans and on plans that track weights: their units are handed out at run time as those of
ordinary plans are."""
import numpy as np
import pytest
import torch

from bounded_util import Step, hide, oracle_out
from gpu_util import assert_parity, da, to_device
from paper_2609_37062_b200 import workloads as wl
from test_weights_gpu import check, totals

pytestmark = pytest.mark.gpu

# more units than resident blocks: lengths around the window's, its tiles' and a unit's borders
LENS = [0, 1, 16, 17, 100, 255, 256, 257, 300, 511, 512, 513, 700, 1023, 1500, 2047] * 6


def mask_of(fraction, n):
    g = torch.Generator().manual_seed(int(fraction * 100))
    return (torch.rand(n, generator=g) >= fraction).to(torch.uint8).cuda()


@pytest.mark.parametrize("hq,hkv,d,dtype", [(32, 8, 128, "bf16"), (8, 2, 64, "fp16"), (40, 8, 128, "fp16"), (36, 4, 64, "bf16"),
                                            (24, 2, 128, "bf16")])
@pytest.mark.parametrize("pol", [dict(window_tokens=256, sink_tokens=20), dict(track_weights=1),
                                 dict(window_tokens=100, sink_tokens=4, track_weights=1, fuse_combine=1, chunk_tokens=64),
                                 dict(window_tokens=300, split_mode=da.DA_SPLIT_DETERMINISTIC, chunk_tokens=128)])
def test_rows_that_run_have_the_bits_of_an_unmasked_launch(hq, hkv, d, dtype, pol):
    window, sinks, B = pol.get("window_tokens", 0), pol.get("sink_tokens", 0), len(LENS)
    w = wl.make_workload("wm", LENS, hq, hkv, d, seed=91, dtype=dtype)
    if window:
        w = hide(w, [1] * B, window, sinks)
    wd = to_device(w)
    s = Step(wd, da.make_policy(**pol))
    s()
    s.ok()
    out, lse = s.out.clone(), s.lse.clone()
    for fraction in (0.0, 0.5, 0.97, 1.0):
        mask = mask_of(fraction, B)
        on = mask.bool()
        s.ws.fill_(0xFF)                                      # NaN where nothing is written
        for _ in range(2):                                    # (the queue is left as it was found)
            s.out.fill_(float("nan")), s.lse.fill_(float("nan"))
            s(run_mask=mask)
            s.ok()
            assert torch.equal(s.out[on], out[on]) and torch.equal(s.lse[on], lse[on])
            assert (s.out[~on] == 0).all() and torch.isneginf(s.lse[~on]).all()
        if pol.get("track_weights"):
            ref = oracle_out(w, window=window, sinks=sinks, run_mask=mask.cpu().numpy())[2]
            before = totals(wd, 3)
            after = before.clone()
            da.decode_attn_add_weights(s.plan, s.ws, s.lse, wd.seq_lens, after)
            s.ok()
            check(before, after, ref, LENS)
            assert torch.equal(after[~on], before[~on])


def test_masked_rows_write_their_new_keys_and_values():
    window, sinks, B = 128, 4, len(LENS)
    w = wl.make_workload("wmn", LENS, 32, 8, 128, seed=92)
    new = [wl.normal_bf16_bits(wl.stream_key(92, t, 0), 0, B * 8 * 128).view(B, 8, 128).cuda() for t in (wl.TENSOR_NEW_K, wl.TENSOR_NEW_V)]
    for fraction in (0.5, 1.0):
        mask = mask_of(fraction, B)
        got = []
        for fused in (False, True):
            wd = to_device(w)
            s = Step(wd, da.make_policy(window_tokens=window, sink_tokens=sinks))
            if not fused:
                da.decode_attn_append_kv(s.shape, *new, wd.block_table, wd.seq_lens, wd.k_pool, wd.v_pool)
                new_rows = {}
            else:
                new_rows = dict(new_k=new[0], new_v=new[1])
            s(run_mask=mask, **new_rows)
            s.ok()
            got.append((s.out, s.lse, wd.k_pool, wd.v_pool))
        assert all(torch.equal(a, b) for a, b in zip(*got))


def test_a_capacity_plan_under_a_mask_replayed_from_a_graph():
    window, sinks, B = 256, 4, 60
    lens0 = (LENS[1:] * 2)[:B]
    w = wl.make_workload("wmc", lens0, 32, 8, 128, seed=93)
    wd = to_device(w)
    pol = da.make_policy(capacity_batch=B, capacity_tokens=sum(lens0), window_tokens=window, sink_tokens=sinks, track_weights=1)
    s = Step(wd, pol)
    mask = mask_of(0.5, B)
    t = totals(wd, extra=16)
    lens_dev = wd.seq_lens.clone()

    def run():
        da.decode_attn_run(s.plan, wd.q_bits, wd.k_pool, wd.v_pool, wd.block_table, lens_dev, s.out, s.lse, s.ws, run_mask=mask)
        da.decode_attn_combine(s.plan, s.ws, s.out, s.lse)
        da.decode_attn_add_weights(s.plan, s.ws, s.lse, lens_dev, t)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    import dataclasses
    for i, n in enumerate((B, 7, 41)):
        lens = [max(0, L - 3 * i) for L in lens0[:n]]
        da.decode_attn_plan_update(s.plan, lens)
        lens_dev[:n] = torch.tensor(lens, dtype=torch.int32, device="cuda")
        mask.copy_(mask_of(0.3 + 0.2 * i, B))
        before = t.clone()
        graph.replay()
        s.ok()
        cut = dataclasses.replace(w, batch=n, seq_lens=torch.tensor(lens, dtype=torch.int32), block_table=w.block_table[:n], q_bits=w.q_bits[:n])
        ref, ref_lse, ref_w = oracle_out(cut, window=window, sinks=sinks, run_mask=mask[:n].cpu().numpy())
        assert_parity(s.out[:n], s.lse[:n], ref, ref_lse)
        check(before[:n], t[:n], ref_w, lens)
        assert torch.equal(before[n:], t[n:])


def step_us(s, mask, n=30):
    flush = torch.empty(256 << 20, dtype=torch.uint8, device="cuda")
    best = float("inf")
    for _ in range(n):
        flush.zero_()
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        s(run_mask=mask)
        b.record()
        b.synchronize()
        best = min(best, a.elapsed_time(b) * 1e3)
    return best


@pytest.mark.parametrize("pol", [dict(window_tokens=4096, sink_tokens=4), dict(track_weights=1)])
def test_the_time_a_masked_row_saves(pol):
    """Half of 256 rows of 1,024 tokens masked: a windowed or tracking step that the planner packs for all rows takes as
    long as its fullest block, 30 % longer than the ordinary one, whose blocks draw their units."""
    wd = to_device(wl.make_workload("wmt", [1024] * 256, 32, 8, 128, seed=94))
    mask = mask_of(0.5, 256)
    plain, other = Step(wd, da.make_policy()), Step(wd, da.make_policy(**pol))
    for s in (plain, other):
        s(run_mask=mask)
    t_plain, t_other = step_us(plain, mask), step_us(other, mask)
    print(f"{t_plain:.1f} {t_other:.1f}")
    assert t_other <= 1.15 * t_plain, (t_plain, t_other)
