"""Evictions whose totals do not stand still, or are much wider than their rows."""
import numpy as np
import pytest
import torch

from gpu_util import da, to_device
from test_evict_gpu import check, fresh_pages, totals, workload

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("wide", [2049, 8193, 49_153])
def test_short_rows_in_wide_totals(wide):
    """The width of the totals picks the blocks' size: rows far below it, alone."""
    lens, budget = [0, 1, 130, 300, 65], 64
    w = workload(lens, budget, 8, 2, 64, seed=61, max_pages_per_seq=-(-wide // 16))
    for kind in ("random", "steps", "any"):
        t = totals(kind, (len(lens), 2, wide), seed=8)
        for in_place in (False, True):
            check(w, fresh_pages(w, budget), budget, 4, 16, t, in_place)


def test_totals_that_change_during_the_call():
    """Rows too long for a block are read several times.  A writer on another stream breaks the rules; the call ends all
    the same, writes nothing out of place, and a row is either given up or cut to tokens it holds."""
    L, budget, sinks, recent, guard, n_calls = 60_000, 2000, 4, 100, 4096, 24
    w = workload([L, L], budget, 4, 2, 64, seed=62, page_size=256)
    wd = to_device(w)
    k0, v0 = wd.k_pool.clone(), wd.v_pool.clone()
    dst = fresh_pages(w, budget).cuda()
    kinds = [totals(kind, (2, 2, L), seed=i).cuda() for i, kind in enumerate(("random", "equal", "steps", "any"))]
    t = kinds[0].clone()
    shape = da.shape_of_workload(wd)
    n = 2 * 2 * budget
    kept = torch.full((n_calls, n + guard), -7, dtype=torch.int32, device="cuda")
    after = torch.full((4 * L + guard,), 7.0, device="cuda")
    lens_out = torch.zeros(2, dtype=torch.int32, device="cuda")
    status = torch.zeros(n_calls, dtype=torch.int32, device="cuda")
    k_out, v_out = [], []
    torch.cuda.synchronize()
    writer, caller = torch.cuda.Stream(), torch.cuda.Stream()
    for i in range(n_calls):
        with torch.cuda.stream(writer):
            for j in range(12):
                t.copy_(kinds[(i + j) % 4])
        with torch.cuda.stream(caller):
            wd.k_pool.copy_(k0)
            wd.v_pool.copy_(v0)
            da.decode_attn_evict(shape, budget, sinks, recent, wd.seq_lens, wd.block_table, dst, wd.k_pool, wd.v_pool, t,
                                 after[:4 * L].view(2, 2, L), kept[i, :n].view(2, 2, budget), lens_out, status[i:i + 1])
            k_out.append(wd.k_pool.clone())
            v_out.append(wd.v_pool.clone())
    torch.cuda.synchronize()
    assert (kept[:, n:] == -7).all() and (after[4 * L:] == 7.0).all()
    assert lens_out.tolist() == [budget, budget]
    for i in range(n_calls):
        pos = kept[i, :n].view(2, 2, budget).cpu().numpy()
        k, v = w.k_pool.clone(), w.v_pool.clone()
        given_up = 0
        for b in range(2):
            for g in range(2):
                p = pos[b, g]
                if (p == -1).all():
                    given_up += 1
                    continue
                assert (np.diff(p) > 0).all() and p[0] >= 0 and p[-1] < L
                assert np.array_equal(p[:sinks], np.arange(sinks)) and np.array_equal(p[-recent:], np.arange(L - recent, L))
                s = torch.from_numpy(p).long()
                page, slot = w.block_table[b, s // 256].long(), s % 256
                j = torch.arange(budget)
                to, to_slot = dst[b].cpu()[j // 256].long(), j % 256
                for pool in (k, v):
                    pool[to, to_slot, g] = pool[page, slot, g]
        assert int(status[i]) == (da.DA_ERR_STALE_PLAN if given_up else da.DA_OK)
        assert torch.equal(k_out[i].cpu(), k) and torch.equal(v_out[i].cpu(), v)
