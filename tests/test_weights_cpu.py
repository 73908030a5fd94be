"""Totals of attention weights without a GPU: what plans and calls refuse before they reach a device."""
import pytest

from paper_2609_37062_b200 import build as da_build

da_build.build()
from paper_2609_37062_b200 import binding as da  # noqa: E402


def shape(B, mpp=512, hq=32, hkv=8):
    return da.make_shape(B, hq, hkv, 128, 16, mpp, 1 << 20, (16 * hkv * 128, hkv * 128, 128))


def plan_status(sh, policy, lens):
    """DA_OK, or the status a plan is refused with; DA_ERR_CUDA (no device here) counts as accepted."""
    try:
        da.decode_attn_plan(sh, policy, lens).destroy()
    except da.DecodeAttnError as e:
        return da.DA_OK if e.status == da.DA_ERR_CUDA else e.status
    return da.DA_OK


@pytest.mark.parametrize("mode", [da.DA_SPLIT_AUTO, da.DA_SPLIT_DETERMINISTIC, da.DA_SPLIT_FIXED_COUNT])
def test_a_tracking_plan_takes_no_more_than_its_capacity(mode):
    # 64 sequences of 4,000 tokens need no more units or records than 1,024 tokens of capacity allow (none is
    # split), but their logits are 250 times what the workspace has room for
    pol = da.make_policy(split_mode=mode, fixed_count=1, max_splits=1, capacity_batch=64, capacity_tokens=1024, track_weights=1)
    assert plan_status(shape(64), pol, [4000] * 64) == da.DA_ERR_INVALID_ARG
    assert plan_status(shape(1), pol, [1025]) == da.DA_ERR_INVALID_ARG
    assert plan_status(shape(1), pol, [1024]) == da.DA_OK
    assert plan_status(shape(64), pol, [16] * 64) == da.DA_OK
    assert plan_status(shape(64), pol, [16] * 63 + [17]) == da.DA_ERR_INVALID_ARG
    pol.window_tokens = 64                                      # (a window does not change what capacity_tokens counts)
    assert plan_status(shape(1), pol, [1025]) == da.DA_ERR_INVALID_ARG


def test_a_plan_without_totals_is_bounded_by_its_units_alone():
    pol = da.make_policy(capacity_batch=64, capacity_tokens=1024)
    assert plan_status(shape(64), pol, [4000] * 64) == da.DA_OK
