"""Queries whose dims span what fp16 holds beside a head's largest one, over keys that are large where the query is small."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from oracle import packed_cache as ref  # noqa: E402
from packed_util import Cache, bounds, da, run  # noqa: E402


@pytest.mark.parametrize("span", [10, 17, 20, 24, 30])
@pytest.mark.parametrize("hq,d,dtype", [(8, 128, "bf16"), (8, 64, "bf16"), (8, 128, "fp16"), (24, 128, "bf16")])
@pytest.mark.parametrize("size", [1.0, 300.0])
def test_small_dims_over_large_keys(span, hq, d, dtype, size):
    """Dims 0 .. 31 of a query are of order `size`, the others 2^-span of that; K is 2^(span / 2) and 2^(-span / 2) of order there, so that
    small dims give the larger part of a logit by 2^(span / 2) or so, brought back by the softmax scale.

    A dim is off by half a step of 2^-24 of the head's largest, hence a logit by 2^-25 max|q| sum|k| beside what `bounds` counts."""
    c = Cache([400, 37], hq, 2, d, dtype=dtype, seed=span)
    rng = np.random.default_rng(span + hq)
    grow = np.where(np.arange(d) < 32, 2.0 ** (-span // 2), 2.0 ** ((span + 1) // 2))
    shape = (c.num_pages, 16, 2, d)
    c.pool = ref.pool_of(rng.standard_normal(shape) * grow, c.v, 16)
    c.k, c.v = ref.pool_values(c.pool, d, 16)
    c.q = (c.q.double() * torch.from_numpy(np.where(np.arange(d) < 32, size, size * 2.0 ** -span))).to(c.q.dtype)
    kv4 = c.shape()
    kv4.sm_scale = float(np.float32(0.5 / (size * 2.0 ** ((span + 1) // 2 - span) * np.sqrt(d) + size * 2.0 ** (-span // 2) * np.sqrt(32))))
    plan = da.decode_attn_plan(kv4, da.make_policy(cache_bits=4), c.lens)
    out, lse, status = run(c, plan=plan)
    plan.destroy()
    assert status == da.DA_OK
    want, want_lse, mass, products = c.expect(scale=kv4.sm_scale)
    q = np.abs(c.q.double().numpy()).max(-1)
    keys = np.zeros(q.shape)
    for b, n in enumerate(c.lens):
        at = np.arange(n)
        sums = np.abs(c.k[c.table[b][at // 16], at % 16]).sum(-1).max(0)       # of a KV head
        keys[b] = np.repeat(sums, hq // 2)
    extra = kv4.sm_scale * 2.0 ** -25 * q * keys                               # what a logit is off by
    err, lse_err = bounds(mass, products + extra * 2.0 ** 18, want_lse, max(c.lens), np.abs(c.v).max())
    off = np.abs(out.double().cpu().numpy() - want)
    assert (off <= err).all(), f"{(off / err).max():.2f} of the bound"
    assert (np.abs(lse.double().cpu().numpy() - want_lse) <= lse_err).all()
