"""How the rows of totals may lie in memory."""
import pytest
import torch

from bounded_util import Step, oracle_out
from gpu_util import da, to_device
from paper_2609_37062_b200 import workloads as wl
from test_weights_gpu import check

pytestmark = pytest.mark.gpu

LENS = [100, 37, 200]


def test_overlapping_rows_are_refused():
    wd = to_device(wl.make_workload("wlo", LENS, 8, 2, 64, seed=71))
    s = Step(wd, da.make_policy(track_weights=1))
    s()
    flat = torch.zeros(4096, device="cuda")
    call = lambda plan, strides: da.decode_attn_add_weights(plan, s.ws, s.lse, wd.seq_lens, flat.as_strided((3, 2, 200), (*strides, 1)),
                                                            check=False)
    for strides in ((200, 200), (400, 400), (199, 800), (400, 199), (200, 400), (400, 800)):
        assert call(s.plan, strides) == da.DA_ERR_INVALID_ARG, strides
    for strides in ((400, 200), (200, 600), (400, 600)):      # sequences first, heads first, interleaved
        assert call(s.plan, strides) == da.DA_OK, strides
    # a capacity plan may be refreshed, and its graph replayed, for more rows than it holds now
    cap = Step(wd, da.make_policy(track_weights=1, capacity_batch=4, capacity_tokens=400))
    for strides, rc in (((208, 3 * 208), da.DA_ERR_INVALID_ARG), ((208, 4 * 208), da.DA_OK), ((416, 208), da.DA_OK)):
        t = flat.as_strided((3, 2, 208), (*strides, 1))
        cap()
        assert da.decode_attn_add_weights(cap.plan, cap.ws, cap.lse, wd.seq_lens, t, check=False) == rc
    cap.ok()


@pytest.mark.parametrize("order", ["sequences", "heads", "interleaved"])
def test_rows_in_any_order(order):
    w = wl.make_workload("wla", LENS, 8, 2, 64, seed=72)
    wd = to_device(w)
    ref = oracle_out(w)[2]
    s = Step(wd, da.make_policy(track_weights=1))
    s()
    strides = {"sequences": (420, 205), "heads": (204, 620), "interleaved": (408, 612)}[order]
    flat = torch.rand(3000, device="cuda")
    t = flat.as_strided((3, 2, 203), (*strides, 1), 8)
    before, all_before = t.clone(), flat.clone()
    da.decode_attn_add_weights(s.plan, s.ws, s.lse, wd.seq_lens, t)
    s.ok()
    check(before, t, ref, LENS)
    t.copy_(before)
    assert torch.equal(flat, all_before)                      # nothing but the rows was written


def test_one_row_of_any_stride():
    w = wl.make_workload("wl1", [150], 4, 1, 64, seed=73)
    wd = to_device(w)
    s = Step(wd, da.make_policy(track_weights=1))
    s()
    for strides in ((0, 0), (1, 1), (150, 7)):
        t = torch.zeros(150, device="cuda").as_strided((1, 1, 150), (*strides, 1))
        da.decode_attn_add_weights(s.plan, s.ws, s.lse, wd.seq_lens, t)
        s.ok()
        check(torch.zeros((1, 1, 150)), t, oracle_out(w)[2], [150])
