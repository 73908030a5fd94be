"""The room a windowed capacity plan asks for, and that every refresh it allows stays within it."""
import random

import pytest
import torch

from bounded_util import Step, oracle_out
from gpu_util import assert_parity, da, to_device
from paper_2609_37062_b200 import workloads as wl
from test_weights_gpu import check

pytestmark = pytest.mark.gpu

TILE_BYTES = 32 * 16 * 4                                      # logits of a tile: 32 query heads, 16 tokens


def plan(batch, tokens, window, sinks, lens):
    sh = da.make_shape(len(lens), 32, 8, 128, 16, 4096, 1 << 16, (16 * 8 * 128, 8 * 128, 128))
    return da.decode_attn_plan(sh, da.make_policy(capacity_batch=batch, capacity_tokens=tokens, window_tokens=window,
                                                  sink_tokens=sinks, track_weights=1), lens)


def logits_bytes(batch, tokens, window, sinks):
    with_logits = plan(batch, tokens, window, sinks, [])
    sh = with_logits.shape
    records = da.decode_attn_plan(sh, da.make_policy(capacity_batch=batch, capacity_tokens=tokens, window_tokens=window,
                                                     sink_tokens=sinks), [])
    return with_logits.workspace_bytes - (records.workspace_bytes + 255) // 256 * 256


def test_logits_take_no_more_than_what_is_visible():
    assert logits_bytes(256, 256 * 32768, 4096, 4) == 256 * (256 + 1 + 1) * TILE_BYTES      # 135 MB; all tokens: 1.07 GB
    assert logits_bytes(256, 256 * 32768, 0, 0) == (256 * 2048 + 256) * TILE_BYTES
    assert logits_bytes(4, 100, 4096, 4) == (100 // 16 + 4) * TILE_BYTES                    # less than a window


@pytest.mark.parametrize("window,sinks", [(1, 0), (2, 1), (15, 0), (16, 16), (17, 4), (31, 33), (33, 1), (100, 500)])
def test_every_refresh_within_the_capacity_is_taken(window, sinks):
    batch, tokens = 8, 8 * 2000
    p = plan(batch, tokens, window, sinks, [])
    rng = random.Random(window * 1000 + sinks)
    lens = [[w + 16 * k] * batch for w in range(max(1, window - 2), window + 34) for k in (0, 1, 40)]
    lens += [[rng.choice((0, 1, window, window + 1, sinks + window, rng.randint(0, 2000))) for _ in range(batch)] for _ in range(300)]
    for row in lens:
        da.decode_attn_plan_update(p, [min(n, 2000) for n in row])


def test_totals_in_the_smaller_room():
    lens, window, sinks = [1999, 33, 700, 31], 32, 17
    w = wl.make_workload("wcs", lens, 32, 8, 128, seed=95)
    wd = to_device(w)
    s = Step(wd, da.make_policy(capacity_batch=4, capacity_tokens=8000, window_tokens=window, sink_tokens=sinks, track_weights=1))
    n = s.plan.workspace_bytes
    s.ws = torch.full((n + 4096,), 0xAB, dtype=torch.uint8, device="cuda")
    s()
    s.ok()
    ref, ref_lse, ref_w = oracle_out(w, window=window, sinks=sinks)
    assert_parity(s.out, s.lse, ref, ref_lse)
    t = torch.zeros((4, 8, 2000), device="cuda")
    da.decode_attn_add_weights(s.plan, s.ws, s.lse, wd.seq_lens, t)
    s.ok()
    check(torch.zeros_like(t), t, ref_w, lens)
    assert (s.ws[n:] == 0xAB).all()                           # nothing behind the workspace was written
