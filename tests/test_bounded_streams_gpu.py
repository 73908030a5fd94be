"""The operators on streams of their own, with every buffer they write looked at, and repeated."""
import dataclasses

import numpy as np
import pytest
import torch

from bounded_util import Step, oracle_out
from gpu_util import assert_parity, da, to_device
from oracle import bounded_cache as bc
from test_evict_gpu import fresh_pages
from test_prompt_gpu import Prompt, compare, prompt
from test_weights_gpu import check

pytestmark = pytest.mark.gpu


def test_every_output_of_calls_on_their_own_streams():
    """A prompt on one stream; attend, count and evict on another; the pools, the totals in both buffers, positions and
    lengths afterwards."""
    lens, budget, sinks, recent = [500, 300], 128, 4, 32
    w = prompt("bs1", [40, 30], [460, 270], 8, 2, 64, 121, pool_pages=120)
    wd = to_device(w)
    steps = dataclasses.replace(wd, q_bits=wd.q_bits[:2].contiguous())
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    pol = da.make_policy(window_tokens=100, sink_tokens=4)
    p = Prompt(wd, [40, 30], pol)
    s = Step(steps, da.make_policy(track_weights=1))
    dst = fresh_pages(w, budget)
    dst_dev, shape = dst.cuda(), da.shape_of_workload(wd)
    before = torch.rand((2, 2, 501), device="cuda")
    total, after = torch.empty_like(before), torch.empty_like(before)
    kept = torch.empty((2, 2, budget), dtype=torch.int32, device="cuda")
    lens_out = torch.empty(2, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    for _ in range(4):
        total.copy_(before)
        after.fill_(7.0)
        a.wait_stream(torch.cuda.current_stream())
        b.wait_stream(torch.cuda.current_stream())
        da.decode_attn_prompt_run(p.plan, wd.q_bits, wd.k_pool, wd.v_pool, wd.block_table, wd.seq_lens, p.out, p.lse, p.ws, stream=a)
        da.decode_attn_run(s.plan, steps.q_bits, wd.k_pool, wd.v_pool, wd.block_table, wd.seq_lens, s.out, s.lse, s.ws, stream=b)
        da.decode_attn_combine(s.plan, s.ws, s.out, s.lse, stream=b)
        da.decode_attn_add_weights(s.plan, s.ws, s.lse, wd.seq_lens, total, stream=b)
        da.decode_attn_evict(shape, budget, sinks, recent, wd.seq_lens, wd.block_table, dst_dev, wd.k_pool, wd.v_pool, total,
                             after, kept, lens_out, stream=b)
        torch.cuda.current_stream().wait_stream(a)
        torch.cuda.current_stream().wait_stream(b)
    torch.cuda.synchronize()
    p.ok(), s.ok()
    compare(p.out, p.lse, w, [40, 30], 100, 4)
    ref, ref_lse, weights = oracle_out(dataclasses.replace(w, q_bits=w.q_bits[:2]))
    assert_parity(s.out, s.lse, ref, ref_lse)
    check(before, total, weights, lens)
    k, v = w.k_pool.clone(), w.v_pool.clone()
    expect = torch.full_like(after, 7.0).cpu()
    t = total.cpu()
    for i, L in enumerate(lens):
        for g in range(2):
            stay = torch.from_numpy(bc.kept_positions(t[i, g].numpy(), L, budget, sinks, recent)).long()
            assert np.array_equal(kept[i, g].cpu().numpy(), stay.numpy())
            expect[i, g, :L] = 0
            expect[i, g, :budget] = t[i, g, stay]
            j = torch.arange(budget)
            for pool in (k, v):
                pool[dst[i, j // 16].long(), j % 16, g] = pool[w.block_table[i, stay // 16].long(), stay % 16, g]
    assert torch.equal(after.cpu(), expect) and lens_out.tolist() == [budget, budget]
    assert torch.equal(wd.k_pool.cpu(), k) and torch.equal(wd.v_pool.cpu(), v)


@pytest.mark.parametrize("new,cached,window,sinks", [([700, 33, 1, 256], [0, 5000, 900, 40], 0, 0), ([512, 400], [3000, 8000], 2000, 4),
                                                     ([16, 3], [30_000, 20_000], 0, 0)])
def test_a_prompt_repeats_its_bits(new, cached, window, sinks):
    wd = to_device(prompt("bs2", new, cached, 32, 8, 128, 122))
    p = Prompt(wd, new, da.make_policy(window_tokens=window, sink_tokens=sinks))
    outs = []
    for i in range(6):
        p.ws.fill_(0xFF if i % 2 else 0)                      # (what the workspace held before plays no part)
        p.out.fill_(float("nan"))
        p()
        outs.append((p.out.clone(), p.lse.clone()))
    p.ok()
    assert all(torch.equal(o, outs[0][0]) and torch.equal(e, outs[0][1]) for o, e in outs[1:])


@pytest.mark.parametrize("pol", [dict(window_tokens=700, sink_tokens=4), dict(track_weights=1), dict(track_weights=1, fuse_combine=1)])
def test_a_step_and_its_totals_repeat_their_bits(pol):
    lens = [0, 1, 900, 5000, 333, 20_000]
    wd = to_device(prompt("bs3", [0] * len(lens), lens, 32, 8, 128, 123))
    from paper_2609_37062_b200 import workloads as wl
    wd = dataclasses.replace(wd, q_bits=wl.normal_bf16_bits(wl.stream_key(123, wl.TENSOR_Q, 1), 0, 6 * 32 * 128).view(6, 32, 128).cuda())
    s = Step(wd, da.make_policy(**pol))
    got = []
    for i in range(6):
        s.ws.fill_(0xFF if i % 2 else 0)
        s()
        t = torch.zeros((6, 8, 20_000), device="cuda")
        if pol.get("track_weights"):
            da.decode_attn_add_weights(s.plan, s.ws, s.lse, wd.seq_lens, t)
        got.append((s.out.clone(), s.lse.clone(), t))
    s.ok()
    assert all(torch.equal(x, y) for g in got[1:] for x, y in zip(g, got[0]))
