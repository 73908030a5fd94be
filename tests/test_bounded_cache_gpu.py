"""Prompts, windowed steps, weights and eviction used together, as an engine would, and their calls on streams of
their own."""
import dataclasses

import numpy as np
import pytest
import torch

from bounded_util import Step, oracle_out
from gpu_util import LSE_ABS, assert_parity, da, to_device
from oracle import bounded_cache as bc
from paper_2609_37062_b200 import workloads as wl
from test_evict_gpu import fresh_pages
from test_prompt_gpu import Prompt, compare, prompt

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("window,sinks", [(0, 0), (200, 4)])
def test_chunks_of_a_prompt_make_the_prompt(window, sinks):
    """Two chunks against the growing cache give what the prompt in one call gives, and its last row is a decode step."""
    L, first = 700, 333
    w = prompt("b1", [L], [0], 32, 8, 128, 111)
    pol = da.make_policy(window_tokens=window, sink_tokens=sinks)
    wd = to_device(w)
    whole = Prompt(wd, [L], pol)
    whole()
    parts = []
    for lo, hi in ((0, first), (first, L)):
        c = dataclasses.replace(wd, seq_lens=torch.tensor([hi], dtype=torch.int32, device="cuda"), q_bits=wd.q_bits[lo:hi].contiguous())
        p = Prompt(c, [hi - lo], pol)
        p()
        p.ok()
        parts.append(p)
    whole.ok()
    out, lse = torch.cat([p.out for p in parts]), torch.cat([p.lse for p in parts])
    compare(out, lse, w, [L], window, sinks)
    compare(whole.out, whole.lse, w, [L], window, sinks)
    step = Step(dataclasses.replace(wd, q_bits=wd.q_bits[-1:].contiguous()), pol)
    o, e = step()
    step.ok()
    # weights of a prompt are rounded to bf16 once: off by at most 2^-8 of sum p |v|, and |v| < 4.5 here
    assert (o[0] - whole.out[-1]).abs().max() < 2.0**-8 * 4.5 and (e[0] - whole.lse[-1]).abs().max() < LSE_ABS


def test_prompt_then_weights_then_eviction_then_steps():
    """A prompt in one call; the weights of its last rows counted as rows that share its pages; the cache cut to its budget;
    decode steps that grow it again."""
    L, n_obs, budget, sinks, recent = 600, 16, 256, 4, 64
    hq, hkv, d, P = 32, 8, 128, 16
    w = prompt("b2", [L], [0], hq, hkv, d, 112, pool_pages=200)
    wd = to_device(w)
    p = Prompt(wd, [L], da.make_policy())
    p()
    p.ok()
    # the last n_obs rows as a batch
    rows = dataclasses.replace(wd, batch=n_obs, q_bits=wd.q_bits[-n_obs:].contiguous(),
                               seq_lens=torch.arange(L - n_obs + 1, L + 1, dtype=torch.int32, device="cuda"),
                               block_table=wd.block_table.expand(n_obs, -1).contiguous())
    s = Step(rows, da.make_policy(track_weights=1))
    out, _ = s()
    totals = torch.zeros((n_obs, hkv, L), device="cuda")
    da.decode_attn_add_weights(s.plan, s.ws, s.lse, rows.seq_lens, totals)
    s.ok()
    assert (out - p.out[-n_obs:]).abs().max() < 2.0**-8 * 4.5
    t = torch.zeros((1, hkv, L + 8), device="cuda")
    t[0, :, :L] = totals.sum(0)
    # eviction to fresh pages with room for a few more tokens
    dst = fresh_pages(w, budget + P)
    kept = torch.empty((1, hkv, budget), dtype=torch.int32, device="cuda")
    lens = torch.empty(1, dtype=torch.int32, device="cuda")
    host = t.cpu().numpy()
    da.decode_attn_evict(da.shape_of_workload(wd), budget, sinks, recent, wd.seq_lens, wd.block_table, dst.cuda(), wd.k_pool,
                         wd.v_pool, t, None, kept, lens)
    assert int(lens) == budget
    for g in range(hkv):
        assert np.array_equal(kept[0, g].cpu().numpy(), bc.kept_positions(host[0, g], L, budget, sinks, recent))
    # steps: write the new row, attend, count
    table = torch.full((1, dst.shape[1]), -1, dtype=torch.int32)
    table[:, :] = dst
    expect = t.cpu().double().numpy()
    for i in range(4):
        n = budget + 1 + i
        q = wl.normal_bf16_bits(wl.stream_key(112, wl.TENSOR_Q, 50 + i), 0, hq * d).view(1, hq, d)
        new = [wl.normal_bf16_bits(wl.stream_key(112, k, 50 + i), 0, hkv * d).view(1, hkv, d).cuda() for k in (wl.TENSOR_NEW_K, wl.TENSOR_NEW_V)]
        cur = dataclasses.replace(wd, q_bits=q.cuda(), seq_lens=torch.tensor([n], dtype=torch.int32, device="cuda"),
                                  block_table=table.cuda(), max_pages_per_seq=table.shape[1])
        s = Step(cur, da.make_policy(track_weights=1))
        out, lse = s(new_k=new[0], new_v=new[1])
        da.decode_attn_add_weights(s.plan, s.ws, s.lse, cur.seq_lens, t)
        s.ok()
        now = dataclasses.replace(cur, k_pool=wd.k_pool.cpu(), v_pool=wd.v_pool.cpu(), q_bits=q, seq_lens=cur.seq_lens.cpu(), block_table=table)
        ref, ref_lse, weights = oracle_out(now)
        assert_parity(out, lse, ref, ref_lse)
        expect[0, :, :n] += weights[0]
    assert (np.abs(t.cpu().double().numpy() - expect) <= 8e-4 * expect + 1e-6).all()


def test_calls_on_streams_of_their_own():
    """Every operator given a stream, two of them at once, ordered by events alone."""
    lens, budget = [500, 300], 128
    w = prompt("b3", [40, 30], [460, 270], 8, 2, 64, 113, pool_pages=120)
    wd = to_device(w)
    steps = dataclasses.replace(wd, q_bits=wd.q_bits[:2].contiguous())
    streams = [torch.cuda.Stream() for _ in range(2)]
    pol = da.make_policy(window_tokens=100, sink_tokens=4)
    p = Prompt(wd, [40, 30], pol)
    s = Step(steps, da.make_policy(track_weights=1))
    t = torch.zeros((2, 2, 500), device="cuda")
    dst = fresh_pages(w, budget).cuda()
    kept = torch.empty((2, 2, budget), dtype=torch.int32, device="cuda")
    lens_out = torch.empty(2, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    shape = da.shape_of_workload(wd)
    for _ in range(3):
        da.decode_attn_prompt_run(p.plan, wd.q_bits, wd.k_pool, wd.v_pool, wd.block_table, wd.seq_lens, p.out, p.lse, p.ws,
                                  stream=streams[0])
        t.zero_()
        streams[1].wait_stream(torch.cuda.current_stream())
        da.decode_attn_run(s.plan, steps.q_bits, wd.k_pool, wd.v_pool, wd.block_table, wd.seq_lens, s.out, s.lse, s.ws,
                           s.plan.workspace_bytes, stream=streams[1].cuda_stream)
        da.decode_attn_combine(s.plan, s.ws, s.out, s.lse, stream=streams[1])
        da.decode_attn_add_weights(s.plan, s.ws, s.lse, wd.seq_lens, t, stream=streams[1])
        da.decode_attn_evict(shape, budget, 4, 32, wd.seq_lens, wd.block_table, dst, wd.k_pool, wd.v_pool, t,
                             torch.zeros_like(t), kept, lens_out, stream=streams[1])
        torch.cuda.synchronize()
    compare(p.out, p.lse, w, [40, 30], 100, 4)
    ref, ref_lse, weights = oracle_out(dataclasses.replace(w, q_bits=w.q_bits[:2]))
    assert_parity(s.out, s.lse, ref, ref_lse)
    for b, L in enumerate(lens):
        assert (np.abs(t[b, :, :L].cpu().double().numpy() - weights[b]) <= 2e-4 * weights[b] + 1e-9).all()
        for g in range(2):
            assert np.array_equal(kept[b, g].cpu().numpy(), bc.kept_positions(t[b, g].cpu().numpy(), L, budget, 4, 32))


def test_one_workspace_for_two_plans_in_turn():
    """A workspace may serve plan after plan on one stream: nothing of an earlier call is read."""
    w = prompt("b4", [70], [2000], 8, 2, 128, 114)
    wd = to_device(w)
    a, b = Prompt(wd, [70], da.make_policy()), Prompt(wd, [70], da.make_policy(window_tokens=600, sink_tokens=10))
    step = dataclasses.replace(wd, q_bits=wd.q_bits[-1:].contiguous())
    s = Step(step, da.make_policy(track_weights=1))
    ws = torch.full((max(a.plan.workspace_bytes, b.plan.workspace_bytes, s.plan.workspace_bytes),), 0xFF, dtype=torch.uint8, device="cuda")
    a.ws = b.ws = s.ws = ws
    t = torch.zeros((1, 2, 2070), device="cuda")
    for _ in range(2):
        a(), b(), s()
        t.zero_()
        da.decode_attn_add_weights(s.plan, ws, s.lse, step.seq_lens, t)
        a(), b()
    a.ok(), b.ok(), s.ok()
    compare(a.out, a.lse, w, [70], 0, 0)
    compare(b.out, b.lse, w, [70], 600, 10)
    weights = oracle_out(dataclasses.replace(w, q_bits=w.q_bits[-1:]))[2][0]
    assert (np.abs(t[0].cpu().double().numpy() - weights) <= 2e-4 * weights + 1e-9).all()


def test_operators_at_once_on_two_plans():
    """Two prompts of different plans in flight together."""
    works = [prompt("b5", [90], [700 + 100 * i], 8, 2, 128, 115 + i) for i in range(2)]
    ps = [Prompt(to_device(w), [90], da.make_policy()) for w in works]
    streams = [torch.cuda.Stream() for _ in ps]
    torch.cuda.synchronize()
    for _ in range(5):
        for p, st in zip(ps, streams):
            with torch.cuda.stream(st):
                p()
    torch.cuda.synchronize()
    for p, w in zip(ps, works):
        p.ok()
        compare(p.out, p.lse, w, [90], 0, 0)
