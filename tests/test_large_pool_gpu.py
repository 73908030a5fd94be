"""Pools of more than 2^31 elements: the operators on pages near their end give the bits they give in a small pool."""
import dataclasses

import pytest
import torch

from bounded_util import Step
from gpu_util import da, to_device
from test_evict_gpu import totals
from test_prompt_gpu import Prompt, prompt

pytestmark = pytest.mark.gpu


def test_pages_beyond_32_bit_offsets():
    window, sinks, budget, hkv, d, P = 300, 4, 128, 8, 128, 16
    w = prompt("lp", [70, 5], [700, 400], 32, hkv, d, 121, pool_pages=100)
    small = to_device(w)
    n = 140_000                                               # pages of 16,384 elements: 2.3e9 in each pool
    shift = n - w.num_pages
    assert n * P * hkv * d > 2**31
    big = {}
    for name in ("k_pool", "v_pool"):
        pool = torch.empty((n, P, hkv, d), dtype=torch.int16, device="cuda")
        pool[shift:] = getattr(small, name)
        big[name] = pool
    table = torch.where(small.block_table >= 0, small.block_table + shift, small.block_table)
    large = dataclasses.replace(small, num_pages=n, block_table=table, **big)
    results = []
    for x in (small, large):
        p = Prompt(x, [70, 5], da.make_policy(window_tokens=window, sink_tokens=sinks))
        p()
        p.ok()
        step = dataclasses.replace(x, q_bits=x.q_bits[:2].contiguous())
        s = Step(step, da.make_policy(window_tokens=window, sink_tokens=sinks, track_weights=1))
        s()
        t = torch.zeros((2, hkv, 770), device="cuda")
        da.decode_attn_add_weights(s.plan, s.ws, s.lse, x.seq_lens, t)
        s.ok()
        used = set(w.block_table[w.block_table >= 0].tolist())
        free = [i for i in range(w.num_pages) if i not in used][:2 * budget // P]
        dst = torch.tensor(free, dtype=torch.int32, device="cuda").view(2, -1) + (x.num_pages - w.num_pages)
        kept = torch.zeros((2, hkv, budget), dtype=torch.int32, device="cuda")
        lens = torch.zeros(2, dtype=torch.int32, device="cuda")
        rank = totals("random", (2, hkv, 770), 3).cuda()
        da.decode_attn_evict(da.shape_of_workload(x), budget, 4, 32, x.seq_lens, x.block_table, dst, x.k_pool, x.v_pool, rank,
                             torch.zeros_like(rank), kept, lens)
        torch.cuda.synchronize()
        results.append((p.out, p.lse, s.out, s.lse, t, kept, lens, x.k_pool[dst.long()].clone(), x.v_pool[dst.long()].clone()))
    assert all(torch.equal(a, b) for a, b in zip(*results))
