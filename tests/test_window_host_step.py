"""The whole step from host buffers with a window, its hidden pages given back."""
import numpy as np
import pytest
import torch

from bounded_util import hide, oracle_out
from gpu_util import assert_parity, da
from paper_2609_37062_b200 import workloads as wl

LENS = [0, 1, 16, 100, 129, 500, 1000]


def host_step(w, policy):
    """DA_OK or the status; without a device DA_ERR_CUDA says that nothing was refused before one was asked for."""
    out = np.full((w.batch, w.num_q_heads, w.head_dim), np.nan, dtype=np.float32)
    lse = np.full((w.batch, w.num_q_heads), np.nan, dtype=np.float32)
    try:
        da.decode_attn_host_step(da.shape_of_workload(w), policy, w.q_bits, w.k_pool, w.v_pool, w.block_table, w.seq_lens, out, lse)
    except da.DecodeAttnError as e:
        if e.status == da.DA_ERR_CUDA and not torch.cuda.is_available():
            return da.DA_OK, out, lse
        return e.status, out, lse
    return da.DA_OK, out, lse


@pytest.mark.parametrize("page_size", [16, 64, 256])
@pytest.mark.parametrize("window,sinks", [(1, 0), (16, 0), (17, 4), (100, 40), (400, 300)])
def test_only_what_is_looked_up_has_to_lie_in_the_pool(page_size, window, sinks):
    w = wl.make_workload("whs", LENS, 8, 2, 64, seed=81, page_size=page_size)
    pol = da.make_policy(window_tokens=window, sink_tokens=sinks)
    hidden = hide(w, [1] * w.batch, window, sinks)
    assert host_step(hidden, pol)[0] == da.DA_OK
    # each entry that is left, taken away as well, is missed
    for b, i in (hidden.block_table >= 0).nonzero().tolist():
        if i * page_size < LENS[b]:
            missing = hide(w, [1] * w.batch, window, sinks)
            missing.block_table[b, i] = -1
            assert host_step(missing, pol)[0] == da.DA_ERR_BAD_PAGE, (b, i)
    if (hidden.block_table != w.block_table).any():
        assert host_step(hidden, da.make_policy())[0] == da.DA_ERR_BAD_PAGE


@pytest.mark.gpu
@pytest.mark.parametrize("window,sinks", [(1, 0), (17, 4), (100, 40)])
def test_its_results(window, sinks):
    w = hide(wl.make_workload("whr", LENS, 8, 2, 64, seed=82, page_size=32), [1] * len(LENS), window, sinks)
    ref, ref_lse, _ = oracle_out(w, window=window, sinks=sinks)
    status, out, lse = host_step(w, da.make_policy(window_tokens=window, sink_tokens=sinks))
    assert status == da.DA_OK
    assert_parity(torch.from_numpy(out), torch.from_numpy(lse), ref, ref_lse)
