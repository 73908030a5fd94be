"""Prompts on the GPU against the fp64 oracle, with NaN in everything no query may see and -1 in the block-table
entries of pages that hold nothing visible.

Tolerance, element by element.  A weight p is rounded once to the 16-bit input type, off by at most u = 2^-8 (bf16) or
2^-11 (fp16) of itself, so an output is off by at most u * sum_t p_t |v_t| (p normalised; the sum is of unrounded
weights).  Logits carry the fp32 rounding of a sum of D products (5.5e-5 at most for these inputs, see
test_weights_gpu.py), which enters the weights twice (numerator and sum): another 1.2e-4 of that sum.  A 16-bit output adds half
a step of its own value.  fp16 weights below 2^-24 of their row's scale vanish and those below 2^-14 lose bits: at most
2^-25 a token, times 2^8 where the scale lags the maximum least: below 2^-11 of the sum up to 5,000 tokens, counted once more."""
import dataclasses

import numpy as np
import pytest
import torch

from bounded_util import hide
from gpu_util import LSE_ABS, LSE_REL, da, to_device
import oracle
from oracle import bounded_cache as bc
from paper_2609_37062_b200 import workloads as wl

pytestmark = pytest.mark.gpu

OUT = {da.DA_DTYPE_FP32: (torch.float32, 0.0), da.DA_DTYPE_BF16: (torch.bfloat16, 2.0**-8), da.DA_DTYPE_FP16: (torch.float16, 2.0**-11)}


def prompt(name, new, cached, hq, hkv, d, seed, **kw):
    """A workload whose last new[b] positions are queries: q has a row for each of them."""
    lens = [n + c for n, c in zip(new, cached)]
    w = wl.make_workload(name, lens, hq, hkv, d, seed=seed, **kw)
    rows = sum(new)
    q = wl.normal_bf16_bits(wl.stream_key(seed, wl.TENSOR_Q, 77), 0, rows * hq * d).view(rows, hq, d)
    if w.dtype == "fp16":
        q = q.view(torch.bfloat16).to(torch.float16).view(torch.int16)
    return dataclasses.replace(w, q_bits=q)


class Prompt:
    def __init__(self, wd, new, policy, out_dtype=da.DA_DTYPE_FP32, scale=0.0):
        self.w = wd
        self.shape = da.shape_of_workload(wd, out_dtype=out_dtype, sm_scale=scale)
        self.plan = da.decode_attn_prompt_plan(self.shape, policy, new, wd.seq_lens)
        rows = max(1, sum(new))
        self.out = torch.full((rows, wd.num_q_heads, wd.head_dim), 7.0, dtype=OUT[out_dtype][0], device="cuda")
        self.lse = torch.full((rows, wd.num_q_heads), 7.0, device="cuda")
        self.ws = torch.full((max(self.plan.workspace_bytes, 256),), 0xFF, dtype=torch.uint8, device="cuda")

    def __call__(self):
        w = self.w
        da.decode_attn_prompt_run(self.plan, w.q_bits, w.k_pool, w.v_pool, w.block_table, w.seq_lens, self.out, self.lse,
                                  self.ws, self.plan.workspace_bytes)
        return self.out, self.lse

    def ok(self):
        assert da.decode_attn_prompt_last_device_status(self.plan) == da.DA_OK


def compare(out, lse, w, new, window, sinks, out_dtype=da.DA_DTYPE_FP32, scale=None, what=""):
    inp = oracle.PagedInputs.from_workload(w)
    ref, ref_lse, _ = bc.attention(inp, new, window, sinks, scale)
    size = bc.attention(inp, new, window, sinks, scale, absolute=True)[0]
    u = 2 * 2.0**-11 if w.dtype == "fp16" else 2.0**-8
    tol = (u + 1.2e-4) * size + OUT[out_dtype][1] * np.abs(ref) + 1e-6
    off = np.abs(out.double().cpu().numpy() - ref)
    assert (off <= tol).all(), (what, float((off / tol).max()))
    got = lse.double().cpu().numpy()
    assert (np.abs(got - ref_lse) <= LSE_ABS + LSE_REL * np.abs(ref_lse)).all(), what


CASES = [  # new tokens, tokens cached before them
    ([1], [0]), ([17], [0]), ([128], [0]), ([300], [0]), ([1, 2, 64, 65, 0, 33], [0, 300, 0, 5, 9, 1000]), ([200, 40], [1111, 3])]


@pytest.mark.parametrize("hq,hkv,d,dtype", [(32, 8, 128, "bf16"), (8, 2, 64, "fp16"), (8, 8, 128, "fp16"), (24, 2, 64, "bf16"),
                                            (10, 2, 128, "bf16"), (16, 1, 64, "bf16")])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (100, 4), (128, 37), (300, 200)])
def test_prompts(hq, hkv, d, dtype, window, sinks):
    for i, (new, cached) in enumerate(CASES):
        w = hide(prompt("p", new, cached, hq, hkv, d, 61 + i, dtype=dtype), new, window, sinks)
        p = Prompt(to_device(w), new, da.make_policy(window_tokens=window, sink_tokens=sinks))
        out, lse = p()
        p.ok()
        compare(out, lse, w, new, window, sinks, what=str((new, cached)))


@pytest.mark.parametrize("out_dtype", list(OUT))
@pytest.mark.parametrize("page_size", [16, 32, 256])
@pytest.mark.parametrize("layout", ["token_major", "head_major"])
def test_pages_layouts_and_output_types(page_size, layout, out_dtype):
    new, cached, window, sinks = [150, 30, 1], [400, 0, 700], 200, 10
    w = hide(prompt("pl", new, cached, 32, 8, 128, 71, page_size=page_size, layout=layout), new, window, sinks)
    p = Prompt(to_device(w), new, da.make_policy(window_tokens=window, sink_tokens=sinks), out_dtype)
    out, lse = p()
    p.ok()
    compare(out, lse, w, new, window, sinks, out_dtype)


@pytest.mark.parametrize("new,cached", [([1], [5000]), ([40], [6000]), ([900], [1500]), ([3, 500], [4100, 0])])
@pytest.mark.parametrize("pol", [dict(), dict(sm_count=5), dict(split_mode=da.DA_SPLIT_DETERMINISTIC, chunk_tokens=256),
                                 dict(window_tokens=1000, sink_tokens=300)])
def test_cut_units(new, cached, pol):
    """Few rows against a long cache: the units are cut along it and their pieces merged."""
    window, sinks = pol.get("window_tokens", 0), pol.get("sink_tokens", 0)
    w = hide(prompt("pc", new, cached, 8, 2, 128, 81), new, window, sinks)
    p = Prompt(to_device(w), new, da.make_policy(**pol))
    if not window and "sm_count" not in pol:
        assert p.plan.workspace_bytes > 0
    out, lse = p()
    p.ok()
    compare(out, lse, w, new, window, sinks)


def test_deterministic_bits_do_not_depend_on_the_batch():
    pol = da.make_policy(split_mode=da.DA_SPLIT_DETERMINISTIC, chunk_tokens=512)
    new, cached = [150, 7, 90], [2000, 0, 700]
    w = prompt("pd", new, cached, 32, 8, 128, 91)
    many = Prompt(to_device(w), new, pol)
    many()
    at = 0
    for b, n in enumerate(new):
        one = dataclasses.replace(w, batch=1, seq_lens=w.seq_lens[b:b + 1], block_table=w.block_table[b:b + 1].contiguous(),
                                  q_bits=w.q_bits[at:at + n].contiguous())
        o = Prompt(to_device(one), [n], pol)
        o()
        assert torch.equal(o.out, many.out[at:at + n]) and torch.equal(o.lse, many.lse[at:at + n])
        at += n
    again = many.out.clone()
    many()
    assert torch.equal(again, many.out)


def test_one_new_token_agrees_with_a_decode_step():
    lens = [300, 17, 1, 2000]
    w = wl.make_workload("po", lens, 32, 8, 128, seed=92)
    wd = to_device(w)
    out, lse = da.run_workload(wd, da.make_policy())
    p = Prompt(wd, [1] * 4, da.make_policy())
    p()
    p.ok()
    compare(p.out, p.lse, w, [1] * 4, 0, 0)
    assert (out - p.out).abs().max() < 2.0**-8 * 4.5 and (lse - p.lse).abs().max() < LSE_ABS


@pytest.mark.parametrize("scale", [0.02, 3.0])
def test_sharp_and_flat_softmax(scale):
    """Logits far apart make the running maximum jump from tile to tile (the rescaled path), flat ones never do."""
    new, cached = [130], [900]
    w = prompt("ps", new, cached, 8, 2, 128, 93)
    p = Prompt(to_device(w), new, da.make_policy(), scale=scale)
    out, lse = p()
    p.ok()
    inp = oracle.PagedInputs.from_workload(w)
    s32 = float(np.float32(scale))
    ref, ref_lse, _ = bc.attention(inp, new, 0, 0, s32)
    size = bc.attention(inp, new, 0, 0, s32, absolute=True)[0]
    # the logits' fp32 rounding grows with the scale: 5.5e-5 is at 1/sqrt(128)
    tol = (2.0**-8 + 1.2e-4 * max(1.0, scale * 128**0.5)) * size + 1e-6
    assert (np.abs(out.double().cpu().numpy() - ref) <= tol).all()
    assert (np.abs(lse.double().cpu().numpy() - ref_lse) <= LSE_ABS + LSE_REL * np.abs(ref_lse)).all()


def test_growing_keys_rescale_every_tile():
    """Keys that grow along the sequence: every tile's maximum is far above the last one's."""
    new, cached = [128], [1024]
    w = prompt("pg", new, cached, 8, 2, 64, 94)
    k = w.k_pool.view(torch.bfloat16).float()
    q = w.q_bits.view(torch.bfloat16).float()
    for t in range(1152):
        pg, sl = int(w.block_table[0, t // 16]), t % 16
        k[pg, sl] = (1 + t // 128) * 0.5
    q = q.abs() * 0.5
    w = dataclasses.replace(w, k_pool=k.to(torch.bfloat16).view(torch.int16), q_bits=q.to(torch.bfloat16).view(torch.int16))
    p = Prompt(to_device(w), new, da.make_policy())
    out, lse = p()
    p.ok()
    compare(out, lse, w, new, 0, 0)


def test_nan_in_a_query_stays_in_its_row():
    """A query that is not a number makes its own row none and no other."""
    for new, cached in (([70], [2000]), ([70], [10])):            # cut units and whole ones
        w = prompt("pq", new, cached, 8, 2, 128, 100)
        good = Prompt(to_device(w), new, da.make_policy())
        good()
        q = w.q_bits.clone()
        q[33, 5, 7] = 0x7FC0
        bad = Prompt(to_device(dataclasses.replace(w, q_bits=q)), new, da.make_policy())
        bad()
        bad.ok()
        assert torch.isnan(bad.out[33, 5]).all() and torch.isnan(bad.lse[33, 5])
        bad.out[33, 5], bad.lse[33, 5] = good.out[33, 5], good.lse[33, 5]
        assert torch.equal(bad.out, good.out) and torch.equal(bad.lse, good.lse)


def test_many_sequences_of_one_token():
    new = [1] * 300
    cached = [(7 * i) % 90 for i in range(300)]
    w = prompt("pm", new, cached, 8, 2, 64, 101)
    p = Prompt(to_device(w), new, da.make_policy(window_tokens=40, sink_tokens=3))
    p()
    p.ok()
    compare(p.out, p.lse, w, new, 40, 3)


def test_capture_and_replay():
    new, cached, window, sinks = [100, 3], [900, 50], 256, 4
    w = prompt("pr", new, cached, 32, 8, 128, 95)
    wd = to_device(w)
    p = Prompt(wd, new, da.make_policy(window_tokens=window, sink_tokens=sinks))
    p()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p()
    for seed in (1, 2):
        q = wl.normal_bf16_bits(wl.stream_key(seed, wl.TENSOR_Q, 5), 0, w.q_bits.numel()).view(w.q_bits.shape)
        wd.q_bits.copy_(q)
        graph.replay()
        p.ok()
        compare(p.out, p.lse, dataclasses.replace(w, q_bits=q), new, window, sinks)


def test_plans_may_go_before_their_kernels_end():
    new, cached = [300], [700]
    w = prompt("pp", new, cached, 32, 8, 128, 96)
    wd = to_device(w)
    outs = []
    for _ in range(20):
        p = Prompt(wd, new, da.make_policy())
        p()
        outs.append(p.out)
        p.plan.destroy()
    torch.cuda.synchronize()
    assert all(torch.equal(o, outs[0]) for o in outs)


def test_bad_pages_and_stale_lengths_are_reported():
    new, cached = [100, 50], [400, 0]
    w = prompt("pb", new, cached, 8, 2, 128, 97)
    wd = to_device(w)
    p = Prompt(wd, new, da.make_policy())
    wd.block_table[0, 3] = w.num_pages
    p()
    assert da.decode_attn_prompt_last_device_status(p.plan) == da.DA_ERR_BAD_PAGE
    assert torch.isfinite(p.out).all()
    wd.block_table[0, 3] = -5
    p()
    assert da.decode_attn_prompt_last_device_status(p.plan) == da.DA_ERR_BAD_PAGE
    wd.block_table.copy_(w.block_table)
    wd.seq_lens[1] = 49
    p()
    assert da.decode_attn_prompt_last_device_status(p.plan) == da.DA_ERR_STALE_PLAN
    assert (p.out[100:] == 0).all() and torch.isneginf(p.lse[100:]).all()
    wd.seq_lens[1] = 50
    p()
    p.ok()
    compare(p.out, p.lse, w, new, 0, 0)


def test_refusals():
    new = [100]
    w = to_device(prompt("pf", new, [3000], 8, 2, 128, 98))
    p = Prompt(w, new, da.make_policy())
    call = lambda q=w.q_bits, k=w.k_pool, bt=w.block_table, lens=w.seq_lens, out=p.out, ws=p.ws, n=p.plan.workspace_bytes: \
        da.decode_attn_prompt_run(p.plan, q, k, w.v_pool, bt, lens, out, p.lse, ws, n, check=False)
    assert call(q=None) == da.DA_ERR_INVALID_ARG
    assert call(k=None) == da.DA_ERR_INVALID_ARG
    assert call(lens=None) == da.DA_ERR_INVALID_ARG
    assert call(out=p.out.data_ptr() + 4) == da.DA_ERR_INVALID_ARG
    assert call(ws=None) == da.DA_ERR_INVALID_ARG
    assert call(n=p.plan.workspace_bytes - 1) == da.DA_ERR_WORKSPACE_TOO_SMALL
    empty = da.decode_attn_prompt_plan(p.shape, da.make_policy(), [0], [3100])
    assert da.decode_attn_prompt_run(empty, None, None, None, None, None, None) == da.DA_OK


def test_no_new_tokens_and_rows_behind_the_last_are_left():
    new, cached = [5, 0, 2], [0, 40, 9]
    w = to_device(prompt("pn", new, cached, 8, 2, 64, 99))
    p = Prompt(w, new, da.make_policy())
    out = torch.full((12, 8, 64), 7.0, device="cuda")
    lse = torch.full((12, 8), 7.0, device="cuda")
    da.decode_attn_prompt_run(p.plan, w.q_bits, w.k_pool, w.v_pool, w.block_table, w.seq_lens, out, lse, p.ws)
    p.ok()
    assert (out[7:] == 7).all() and (lse[7:] == 7).all() and not (out[:7] == 7).any()
