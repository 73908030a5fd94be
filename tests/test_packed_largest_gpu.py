"""The largest fp16 values in a cache in 4 bits: written, expanded and attended without becoming infinite."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from oracle import packed_cache as ref  # noqa: E402
from packed_util import KINDS, Cache, check, da, run  # noqa: E402


def written(values, d, dtype, page=16):
    """A pool that decode_attn_prepare_rows wrote of K = V = values [tokens, heads, d], token by token; and what it holds."""
    n, heads, _ = values.shape
    pages = -(-n // page)
    pool = torch.zeros((pages, heads, da.decode_attn_packed_head_bytes(d, page)), dtype=torch.uint8, device="cuda")
    x = values.cuda()
    da.decode_attn_prepare_rows(da.make_kv4_shape(0, heads, heads, d, page, 0, pages, in_dtype=KINDS[dtype][0]), None, x, x,
                                torch.arange(n, device="cuda"), k_cache=pool, cache_bits=4)
    return pool


def large_rows(n, heads, d, dtype, largest, seed):
    """Normal values; in every block of 32 of some rows one or both of +-largest, among smaller ones of that order."""
    gen = torch.Generator().manual_seed(seed)
    x = torch.randn((n, heads, d), generator=gen, dtype=torch.float64)
    x[::3] *= largest / 8
    x.clamp_(-largest, largest)
    x[::3, :, 5::32], x[::6, :, 17::32] = largest, -largest
    x = x.to(KINDS[dtype][1])
    assert x.double().abs().max() == largest
    return x


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype,largest", [("fp16", 65504.0), ("fp16", 65472.0), ("bf16", 65536.0), ("bf16", 65280.0)])
def test_written_and_expanded_to_fp16(d, dtype, largest):
    x = large_rows(50, 2, d, dtype, largest, d)
    pool = written(x, d, dtype)
    want = ref.values(*ref.encode(x.double().numpy()))
    for got in ref.pool_values(pool.cpu().numpy(), d, 16):
        assert np.array_equal(got.reshape(-1, 2, d)[:50], want)
    assert np.abs(want).max() <= 65504
    for to in ("fp16", "bf16"):
        shape = da.make_shape(1, 2, 2, d, 16, 4, 4, (16 * 2 * d, 2 * d, d), in_dtype=KINDS[to][0])
        k, v = (torch.zeros((4, 16, 2, d), dtype=KINDS[to][1], device="cuda") for _ in range(2))
        table = torch.arange(4, dtype=torch.int32, device="cuda")[None].contiguous()
        da.decode_attn_expand_kv(shape, da.make_kv4_shape(1, 2, 2, d, 16, 4, 4), pool, table, torch.tensor([50], dtype=torch.int32).cuda(),
                                 table, k, v)
        for got in (k, v):
            assert torch.isfinite(got).all()
            assert torch.equal(got.flatten(0, 1)[:50].cpu(), torch.from_numpy(want).to(KINDS[to][1]))


@pytest.mark.parametrize("hq", [2, 12, 24])
@pytest.mark.parametrize("dtype,largest", [("fp16", 65504.0), ("bf16", 65536.0)])
def test_attended(hq, dtype, largest):
    """Some of these values have weights that underflow: 0 times a finite value."""
    c = Cache([150, 33], hq, 2, 128, dtype=dtype, seed=hq)
    x = large_rows(c.num_pages * 16, 2, 128, dtype, largest, hq)
    held = ref.values(*ref.encode(x.double().numpy())).reshape(c.num_pages, 16, 2, 128)
    c.pool = ref.pool_of(c.k, x.double().numpy().reshape(held.shape), 16)
    c.v = ref.pool_values(c.pool, 128, 16)[1]
    assert np.array_equal(c.v, held)
    for scale in (0.09, 30.0):
        shape = c.shape()
        shape.sm_scale = scale
        plan = da.decode_attn_plan(shape, da.make_policy(cache_bits=4), c.lens)
        out, lse, status = run(c, plan=plan)
        plan.destroy()
        assert status == da.DA_OK
        check(c, out, lse, f"scale {scale}", scale=scale)
