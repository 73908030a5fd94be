"""Helpers shared by the tests of windows, weights, eviction and prompts."""
import dataclasses

import numpy as np
import torch

import oracle
from oracle import bounded_cache as bc
from gpu_util import da, to_device  # noqa: F401


def hide(w, new_lens, window, sinks, poison=0x7FC0):
    """A copy of the workload in which everything no query may see is poisoned: K and V of hidden positions hold NaN,
    and block-table entries of pages that hold no visible position are -1."""
    bt, lens, P = w.block_table.clone(), w.seq_lens.tolist(), w.page_size
    k, v = w.k_pool.clone(), w.v_pool.clone()
    for b, (L, n) in enumerate(zip(lens, new_lens)):
        t = np.arange(L)
        vis = np.zeros(L, dtype=bool)
        if n > 0 and L > 0:
            first = L - n                                     # the oldest query sees the oldest positions
            vis = bc.seen(first, t, window, sinks) | (t > first)
        for p in range(-(-L // P)):
            at = t[p * P:(p + 1) * P]
            page = int(bt[b, p])
            if not vis[at].any():
                bt[b, p] = -1
            for s in np.flatnonzero(~vis[at]):
                if w.layout == "token_major":
                    k[page, s], v[page, s] = poison, poison
                else:
                    k[page, :, s], v[page, :, s] = poison, poison
    return dataclasses.replace(w, block_table=bt, k_pool=k, v_pool=v)


def oracle_out(w, new_lens=None, window=0, sinks=0, run_mask=None, scale=None):
    inp = oracle.PagedInputs.from_workload(w)
    return bc.attention(inp, [1] * w.batch if new_lens is None else new_lens, window, sinks, scale, run_mask)


class Step:
    """One decode step's buffers for a device workload."""

    def __init__(self, w, policy, out_dtype=None, plan=None):
        self.w = w
        self.shape = da.shape_of_workload(w, out_dtype=da.DA_DTYPE_FP32 if out_dtype is None else out_dtype)
        self.plan = plan or da.decode_attn_plan(self.shape, policy, w.seq_lens)
        self.out = torch.full((w.batch, w.num_q_heads, w.head_dim), float("nan"), device="cuda")
        self.lse = torch.full((w.batch, w.num_q_heads), float("nan"), device="cuda")
        self.ws = torch.empty(max(self.plan.workspace_bytes, 256), dtype=torch.uint8, device="cuda")
        self.fused = policy.fuse_combine

    def __call__(self, **kw):
        w = self.w
        da.decode_attn_run(self.plan, w.q_bits, w.k_pool, w.v_pool, w.block_table, w.seq_lens, self.out, self.lse,
                           self.ws, self.plan.workspace_bytes, **kw)
        if not self.fused:
            da.decode_attn_combine(self.plan, self.ws, self.out, self.lse)
        return self.out, self.lse

    def ok(self):
        assert da.decode_attn_last_device_status(self.plan) == da.DA_OK
