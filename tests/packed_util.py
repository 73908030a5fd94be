"""Helpers of the tests of caches in 4 bits: a shuffled packed cache on the CPU with its values, and on the device."""
import numpy as np
import torch

from oracle import packed_cache as ref
from paper_2609_37062_b200 import binding as da

KINDS = {"bf16": (da.DA_DTYPE_BF16, torch.bfloat16), "fp16": (da.DA_DTYPE_FP16, torch.float16),
         "fp32": (da.DA_DTYPE_FP32, torch.float32)}


def rounded(x, dtype):
    """fp64 values as the 16-bit type holds them."""
    return torch.from_numpy(np.asarray(x)).to(KINDS[dtype][1])


class Cache:
    """Sequences of `lens` tokens in a pool in 4 bits whose unused bytes are 0xff (NaN scales) and whose unused block-table
    entries are -1."""

    def __init__(self, lens, hq, hkv, d, page=16, dtype="bf16", seed=0, spare=2, width=None):
        rng = np.random.default_rng(seed)
        self.lens, self.hq, self.hkv, self.d, self.page, self.dtype = list(lens), hq, hkv, d, page, dtype
        held = [-(-n // page) for n in lens]
        self.width = width or max(held + [1])
        self.num_pages = sum(held) + spare
        ids = rng.permutation(self.num_pages)
        self.table = np.full((len(lens), self.width), -1, dtype=np.int32)
        at = 0
        for b, n in enumerate(held):
            self.table[b, :n] = ids[at:at + n]
            at += n
        shape = (self.num_pages, page, hkv, d)
        k, v = (rounded(rng.standard_normal(shape) * rng.uniform(0.3, 3, (1, 1, hkv, d)), dtype).double().numpy() for _ in range(2))
        self.pool = ref.pool_of(k, v, page)
        self.k, self.v = ref.pool_values(self.pool, d, page)
        # what no sequence holds: whole tiles and rows behind an end
        tiles = self.pool.reshape(self.num_pages, hkv, page // 16, -1)
        blank = np.full(ref.tile_bytes(d), 0xff, dtype=np.uint8)
        used = np.zeros((self.num_pages, page), dtype=bool)
        for b, n in enumerate(lens):
            for p in range(n):
                used[self.table[b, p // page], p % page] = True
        for which in ("k", "v"):
            bytes_at, scales_at = ref._index(d, which)
            for pg, place in zip(*np.nonzero(~used)):
                t, r = place // 16, place % 16
                for where in (bytes_at[r], scales_at[r], scales_at[r] + 1):
                    tiles[pg, :, t, where] = blank[0]
        self.q = rounded(rng.standard_normal((len(lens), hq, d)), dtype)

    def shape(self, out="fp32", strides=None):
        return da.make_kv4_shape(len(self.lens), self.hq, self.hkv, self.d, self.page, self.width, self.num_pages, strides,
                                 out_dtype=KINDS[out][0], in_dtype=KINDS[self.dtype][0])

    def expect(self, window=0, sinks=0, scale=None):
        return ref.attend(self.q.double().numpy(), self.k, self.v, self.table, self.lens, self.page, window, sinks, scale)


def bounds(mass, size, lse, n, largest, out="fp32"):
    """How far an output and a log-sum-exp may be off.  Each weight and each value * scale is rounded once to fp16 (2^-11
    relative; weights below 2^-14 of the largest by 2^-25 at most, n of them), logits carry the fp32 sums of 128 products (2^-18 of the
    sum of magnitudes is generous: a product sum of 128 terms has at most 2^-17 / 2 by the worst order), twice because a
    weight is divided by a sum of weights; then the rounding of the output type."""
    dl = size * 2.0 ** -18 + 2.0 ** -18
    err = mass * (2.0 ** -10 + 2.0 ** -20 + 2 * dl[..., None]) + n * 2.0 ** -25 * largest + 1e-6
    half = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8, "fp16": 2.0 ** -11}[out]
    return err + half * (mass + err), dl + np.where(np.isfinite(lse), np.abs(lse), 0) * 2.0 ** -21


def check(cache, out, lse, what="", dtype="fp32", window=0, sinks=0, scale=None, dead=()):
    want, want_lse, mass, size = cache.expect(window, sinks, scale)
    for b in dead:
        want[b], want_lse[b], mass[b], size[b] = 0, -np.inf, 0, 0
    got, got_lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    err, lse_err = bounds(mass, size, want_lse, max(cache.lens + [1]), np.abs(cache.v).max(), dtype)
    assert np.isfinite(got).all(), what
    off = np.abs(got - want)
    assert (off <= err).all(), f"{what}: off by {off.max():.3e}, {(off / err).max():.2f} of the bound"
    assert np.array_equal(np.isneginf(got_lse), np.isneginf(want_lse)), what
    fin = np.isfinite(want_lse)
    assert (np.abs(got_lse[fin] - want_lse[fin]) <= lse_err[fin]).all(), what
    return float((off / err).max()) if off.size else 0.0


def run(cache, policy=None, out="fp32", strides=None, pool=None, run_mask=None, plan=None):
    """plan, run, combine on the current device; returns out, lse and the device status."""
    policy = policy or da.make_policy(cache_bits=4)
    shape = cache.shape(out, strides)
    own = plan is None
    if own:
        plan = da.decode_attn_plan(shape, policy, cache.lens)
    if pool is None:
        pool = torch.from_numpy(cache.pool).cuda()
    table, lens = torch.from_numpy(cache.table).cuda(), torch.tensor(cache.lens, dtype=torch.int32).cuda()
    o = torch.full(cache.q.shape, float("nan"), dtype=KINDS[out][1], device="cuda")
    lse = torch.full(cache.q.shape[:2], float("nan"), dtype=torch.float32, device="cuda")
    ws = torch.empty(max(plan.workspace_bytes, 256), dtype=torch.uint8, device="cuda")
    da.decode_attn_run(plan, cache.q.cuda(), pool, None, table, lens, o, lse, ws, run_mask=run_mask)
    if not policy.fuse_combine:
        da.decode_attn_combine(plan, ws, o, lse)
    status = da.decode_attn_last_device_status(plan)
    if own:
        plan.destroy()
    return o, lse, status
