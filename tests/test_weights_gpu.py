"""Running totals of attention weights against the fp64 oracle.

Tolerance.  The increment of a token is a sum over the group's heads of 2^(x - e), x and e the logit and the row's
log-sum-exp in the base-2 domain.  x is an fp32 sum of D <= 128 products of 16-bit inputs: its rounding is at most
D * 2^-24 * sum |q k| * scale, about 128 * 6e-8 * 128 * 0.64 / sqrt(128) = 5.5e-5 for N(0, 1) inputs, and e carries at
most the same plus 2^-23 |e|; the exponential adds two ulps.  Together below 2e-4 of the increment; adding it to the
total rounds by half an ulp of the sum (2^-24, doubled here for the sums over heads)."""
import dataclasses

import numpy as np
import pytest
import torch

from bounded_util import Step, hide, oracle_out
from gpu_util import assert_parity, da, to_device
from paper_2609_37062_b200 import workloads as wl

pytestmark = pytest.mark.gpu

LENS = [0, 1, 15, 16, 17, 33, 100, 257, 1000, 2500]


def totals(w, extra=0, seed=0):
    g = torch.Generator().manual_seed(seed)
    return torch.rand((w.batch, w.num_kv_heads, int(w.seq_lens.max()) + extra), generator=g).cuda()


def check(before, after, ref, lens):
    before, after = before.cpu().double().numpy(), after.cpu().double().numpy()
    for b, L in enumerate(lens):
        grown = before[b, :, :L] + ref[b]
        tol = 2e-4 * ref[b] + 2.0**-23 * np.abs(grown)
        assert (np.abs(after[b, :, :L] - grown) <= tol).all(), b
        assert np.array_equal(after[b, :, L:], before[b, :, L:])   # behind the end nothing is written


@pytest.mark.parametrize("hq,hkv,d,dtype", [(8, 2, 64, "bf16"), (32, 8, 128, "bf16"), (8, 8, 128, "fp16"), (10, 2, 128, "bf16"),
                                            (6, 2, 64, "fp16"), (24, 2, 64, "bf16"), (16, 1, 128, "bf16")])
@pytest.mark.parametrize("pol", [dict(), dict(fuse_combine=1, chunk_tokens=64),
                                 dict(split_mode=da.DA_SPLIT_DETERMINISTIC, chunk_tokens=32),
                                 dict(window_tokens=100, sink_tokens=20), dict(window_tokens=16, sink_tokens=0)])
def test_totals_grow_by_the_softmax_weights(hq, hkv, d, dtype, pol):
    window, sinks = pol.get("window_tokens", 0), pol.get("sink_tokens", 0)
    w = wl.make_workload("wt", LENS, hq, hkv, d, seed=41, dtype=dtype)
    if window:
        w = hide(w, [1] * len(LENS), window, sinks)
    ref, ref_lse, ref_w = oracle_out(w, window=window, sinks=sinks)
    wd = to_device(w)
    s = Step(wd, da.make_policy(track_weights=1, **pol))
    s.ws.fill_(0xFF)                                          # NaN where nothing was written
    out, lse = s()
    for extra in (0, 3):                                      # aligned and unaligned rows of totals
        before = totals(wd, extra)
        apart = before.clone()
        da.decode_attn_add_weights(s.plan, s.ws, lse, wd.seq_lens, before, apart)
        s.ok()
        assert_parity(out, lse, ref, ref_lse)
        check(before, apart, ref_w, LENS)
        here = before.clone()
        da.decode_attn_add_weights(s.plan, s.ws, lse, wd.seq_lens, here)
        assert torch.equal(here, apart)                       # in place: the same bits


def test_tracking_changes_no_bit_of_the_output():
    wd = to_device(wl.make_workload("wtb", LENS, 32, 8, 128, seed=42))
    a, b = Step(wd, da.make_policy()), Step(wd, da.make_policy(track_weights=1))
    a(), b()
    assert torch.equal(a.out, b.out) and torch.equal(a.lse, b.lse)


def test_masked_rows_add_nothing():
    wd = to_device(wl.make_workload("wtm", LENS, 32, 8, 128, seed=43))
    s = Step(wd, da.make_policy(track_weights=1))
    s.ws.fill_(0xFF)
    mask = torch.tensor([i % 2 for i in range(len(LENS))], dtype=torch.uint8, device="cuda")
    s(run_mask=mask)
    before = totals(wd)
    after = before.clone()
    da.decode_attn_add_weights(s.plan, s.ws, s.lse, wd.seq_lens, after)
    s.ok()
    assert torch.equal(after[mask == 0], before[mask == 0])
    assert (after[9, :, :2500] > before[9, :, :2500]).any()


def test_prompt_rows_share_pages():
    """The last n tokens of a prompt as n rows over the same pages, each with its own length."""
    n, L = 8, 300
    w = wl.make_workload("wtp", [L], 8, 2, 64, seed=44)
    lens = torch.arange(L - n + 1, L + 1, dtype=torch.int32)
    q = wl.normal_bf16_bits(wl.stream_key(44, wl.TENSOR_Q, 9), 0, n * 8 * 64).view(n, 8, 64)
    rows = dataclasses.replace(w, batch=n, seq_lens=lens, block_table=w.block_table.expand(n, -1).contiguous(), q_bits=q)
    prompt = dataclasses.replace(w, q_bits=q)
    _, _, ref = oracle_out(prompt, new_lens=[n])
    s = Step(to_device(rows), da.make_policy(track_weights=1))
    s()
    t = torch.zeros((n, 2, L), device="cuda")
    da.decode_attn_add_weights(s.plan, s.ws, s.lse, s.w.seq_lens, t)
    s.ok()
    got = t.double().sum(0).cpu().numpy()
    assert (np.abs(got - ref[0]) <= 2e-4 * ref[0] + 1e-9).all()


def test_capacity_plan_and_graph():
    pol = da.make_policy(track_weights=1, capacity_batch=4, capacity_tokens=4000)
    w = wl.make_workload("wtc", [1000, 900, 800, 700], 32, 8, 128, seed=45)
    wd = to_device(w)
    s = Step(wd, pol)
    t = totals(wd, extra=24)
    run = lambda: (s(), da.decode_attn_add_weights(s.plan, s.ws, s.lse, wd.seq_lens, t))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for lens in ([1000, 900, 800, 700], [3, 0, 799, 700], [16, 17]):
        da.decode_attn_plan_update(s.plan, lens)
        n = len(lens)
        wd.seq_lens[:n] = torch.tensor(lens, dtype=torch.int32, device="cuda")
        before = t.clone()
        graph.replay()
        s.ok()
        cut = dataclasses.replace(w, batch=n, seq_lens=torch.tensor(lens, dtype=torch.int32), block_table=w.block_table[:n], q_bits=w.q_bits[:n])
        ref = oracle_out(cut)[2]
        check(before[:n], t[:n], ref, lens)
        assert torch.equal(before[n:], t[n:])


def test_a_graph_captured_while_nothing_is_live():
    """A capacity plan captured with no rows, then with rows of length 0, counts what it is refreshed for."""
    w = wl.make_workload("wtz", [300, 200], 8, 2, 64, seed=47)
    for first in ([], [0, 0]):
        wd = to_device(w)
        s = Step(wd, da.make_policy(track_weights=1, capacity_batch=2, capacity_tokens=600))
        t = torch.zeros((2, 2, 320), device="cuda")
        da.decode_attn_plan_update(s.plan, first)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            s()
            da.decode_attn_add_weights(s.plan, s.ws, s.lse, wd.seq_lens, t)
        da.decode_attn_plan_update(s.plan, [300, 200])
        graph.replay()
        s.ok()
        check(torch.zeros_like(t), t, oracle_out(w)[2], [300, 200])


def test_refusals():
    wd = to_device(wl.make_workload("wtr", [100, 200], 8, 2, 64, seed=46))
    s = Step(wd, da.make_policy(track_weights=1))
    t = totals(wd)
    plain = Step(wd, da.make_policy())
    call = lambda plan=s.plan, ws=s.ws, lse=s.lse, lens=wd.seq_lens, a=t, o=t: da.decode_attn_add_weights(plan, ws, lse, lens, a, o, check=False)
    assert call(plan=plain.plan) == da.DA_ERR_UNSUPPORTED
    assert call(ws=None) == da.DA_ERR_INVALID_ARG
    assert call(lse=None) == da.DA_ERR_INVALID_ARG
    assert call(lens=None) == da.DA_ERR_INVALID_ARG
    assert call(a=t[..., :150].contiguous(), o=t[..., :150].contiguous()) == da.DA_ERR_INVALID_ARG   # rows shorter than a sequence
    with pytest.raises(da.DecodeAttnError):
        da.decode_attn_add_weights(s.plan, s.ws, s.lse, wd.seq_lens, t, t[..., :150])
    rc = da.decode_attn_run(s.plan, wd.q_bits, wd.k_pool, wd.v_pool, wd.block_table, wd.seq_lens, s.out, s.lse, s.ws,
                            s.plan.workspace_bytes - 1, check=False)
    assert rc == da.DA_ERR_WORKSPACE_TOO_SMALL
    s()
    wd.seq_lens[0] = 99
    before = t.clone()
    da.decode_attn_add_weights(s.plan, s.ws, s.lse, wd.seq_lens, t)
    assert da.decode_attn_last_device_status(s.plan) == da.DA_ERR_STALE_PLAN
    assert torch.equal(before[0], t[0])
