"""Decode steps over a cache in 4 bits against the fp64 oracle: sizes, groups, types, pages, policies."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from oracle import packed_cache as ref  # noqa: E402
from packed_util import Cache, check, da, run  # noqa: E402

HEADS = [(1, 1), (8, 8), (6, 3), (32, 8), (10, 2), (16, 2), (18, 2), (24, 2), (16, 1)]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv", HEADS)
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_groups(d, hq, hkv, dtype):
    c = Cache([1, 15, 16, 17, 129, 700], hq, hkv, d, dtype=dtype, seed=hq * 7 + d)
    out, lse, status = run(c)
    assert status == da.DA_OK
    check(c, out, lse, f"{hq}/{hkv} heads of {d}")


@pytest.mark.parametrize("lens", [[0], [1], [2, 0, 1], [16], [127, 128, 129], [255, 256, 257, 0], [1023], [4097, 3], [9001]])
@pytest.mark.parametrize("d", [64, 128])
def test_lengths(lens, d):
    c = Cache(lens, 8, 2, d, seed=len(lens) + d)
    out, lse, status = run(c)
    assert status == da.DA_OK
    check(c, out, lse, str(lens))


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("d", [64, 128])
def test_pages(page, d):
    c = Cache([1, page - 1, page, page + 1, 3 * page + 5, 900], 8, 2, d, page=page, seed=page)
    out, lse, status = run(c)
    assert status == da.DA_OK
    check(c, out, lse, f"pages of {page}")


@pytest.mark.parametrize("out", ["fp32", "bf16", "fp16"])
def test_output_types(out):
    c = Cache([37, 400], 32, 8, 128, seed=3)
    o, lse, status = run(c, out=out)
    assert status == da.DA_OK
    check(c, o, lse, out, dtype=out)


def _policies():
    m = da.make_policy
    return {"fixed": m(split_mode=da.DA_SPLIT_FIXED_COUNT, fixed_count=7, cache_bits=4),
            "deterministic": m(split_mode=da.DA_SPLIT_DETERMINISTIC, cache_bits=4),
            "fused": m(fuse_combine=1, cache_bits=4),
            "few blocks": m(sm_count=3, cache_bits=4),
            "one block": m(sm_count=1, ctas_per_sm=1, chunk_tokens=48, cache_bits=4),
            "named kernel": m(kernel=da.DA_KERNEL_PACKED, cache_bits=4)}


@pytest.mark.parametrize("name", list(_policies()))
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (24, 2, 64)])
def test_policies(name, hq, hkv, d):
    c = Cache([1, 0, 80, 1500, 333, 17], hq, hkv, d, seed=11)
    out, lse, status = run(c, _policies()[name])
    assert status == da.DA_OK
    check(c, out, lse, name)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 4), (16, 0), (100, 4), (129, 37), (5000, 3)])
@pytest.mark.parametrize("d", [64, 128])
def test_windows(window, sinks, d):
    c = Cache([1, 90, 200, 1000, 2049], 8, 2, d, seed=window)
    # what no query sees is poisoned, and its pages are gone
    tiles = c.pool.reshape(c.num_pages, c.hkv, c.page // 16, -1)
    for b, n in enumerate(c.lens):
        for i in range(n // 16):
            if (i + 1) * 16 <= n - window and i * 16 >= sinks:
                tiles[c.table[b, i]] = 0xff
                c.table[b, i] = -1
    out, lse, status = run(c, da.make_policy(window_tokens=window, sink_tokens=sinks, cache_bits=4))
    assert status == da.DA_OK
    check(c, out, lse, f"window {window}, sinks {sinks}", window=window, sinks=sinks)


def test_hidden_rows_of_visible_tiles_may_hold_anything():
    c = Cache([100], 4, 1, 128, seed=5)
    tiles = c.pool.reshape(c.num_pages, 1, 1, -1)
    window, sinks = 41, 5                                                      # hides 5 .. 58: parts of tiles 0 and 3
    for p in range(sinks, 100 - window):
        for which in ("k", "v"):
            _, scales = ref._index(128, which)
            tiles[c.table[0, p // 16], :, 0, scales[p % 16]] = 0xff
            tiles[c.table[0, p // 16], :, 0, scales[p % 16] + 1] = 0xff
    out, lse, status = run(c, da.make_policy(window_tokens=window, sink_tokens=sinks, cache_bits=4))
    assert status == da.DA_OK
    check(c, out, lse, "hidden rows", window=window, sinks=sinks)


@pytest.mark.parametrize("scale", [0.01, 1.0, 30.0])
def test_sharp_and_flat_weights(scale):
    c = Cache([2000, 5], 8, 2, 128, seed=9)
    shape = c.shape()
    shape.sm_scale = scale
    plan = da.decode_attn_plan(shape, da.make_policy(cache_bits=4), c.lens)
    out, lse, status = run(c, plan=plan)
    plan.destroy()
    assert status == da.DA_OK
    check(c, out, lse, f"scale {scale}", scale=scale)


@pytest.mark.parametrize("size", [1e-30, 1e-4, 1e4])
def test_queries_of_any_magnitude(size):
    """bf16 queries far outside fp16's range: logits scale with them, the softmax scale brings them back."""
    c = Cache([300], 8, 2, 128, seed=13)
    c.q = (c.q.float() * size).bfloat16()
    shape = c.shape()
    shape.sm_scale = float(torch.tensor(0.09 / size, dtype=torch.float32))
    plan = da.decode_attn_plan(shape, da.make_policy(cache_bits=4), c.lens)
    out, lse, status = run(c, plan=plan)
    plan.destroy()
    assert status == da.DA_OK
    check(c, out, lse, f"queries of {size}", scale=shape.sm_scale)


def test_rising_logits_renew_the_maximum():
    """Keys that grow along the sequence: the running maximum is outrun again and again."""
    c = Cache([1200], 4, 1, 64, seed=2)
    k = np.zeros(c.k.shape)
    for p in range(1200):
        k[c.table[0, p // 16], p % 16] = np.sign(c.q[0, 0].double().numpy()) * (p // 100 + 1) * 0.5
    c.pool = ref.pool_of(k, c.v, 16)
    c.k, c.v = ref.pool_values(c.pool, 64, 16)
    out, lse, status = run(c)
    assert status == da.DA_OK
    check(c, out, lse, "rising")


@pytest.mark.parametrize("fuse", [0, 1])
def test_run_mask(fuse):
    c = Cache([100, 0, 640, 33, 7], 8, 2, 128, seed=21)
    mask = torch.tensor([1, 1, 0, 1, 0], dtype=torch.uint8, device="cuda")
    pages = [int(p) for b in (2, 4) for p in c.table[b] if p >= 0]
    c.pool[pages] = 0xff
    out, lse, status = run(c, da.make_policy(fuse_combine=fuse, cache_bits=4, chunk_tokens=64), run_mask=mask)
    assert status == da.DA_OK
    check(c, out, lse, "masked", dead=(2, 4))


@pytest.mark.parametrize("layout", ["padded", "heads outside"])
def test_strides(layout):
    c = Cache([300, 41], 8, 2, 128, page=32, seed=8)
    head = da.decode_attn_packed_head_bytes(128, 32)
    if layout == "padded":
        strides = (2 * (head + 48) + 16, head + 48)
        pool = torch.full((c.num_pages * strides[0] + 64,), 0xff, dtype=torch.uint8)
    else:
        strides = (head, c.num_pages * head)
        pool = torch.full((2 * c.num_pages * head,), 0xff, dtype=torch.uint8)
    view = pool.as_strided((c.num_pages, 2, head), (strides[0], strides[1], 1))
    view.copy_(torch.from_numpy(c.pool))
    out, lse, status = run(c, strides=strides, pool=pool.cuda())
    assert status == da.DA_OK
    check(c, out, lse, layout)


def test_page_order_and_batch_do_not_change_deterministic_bits():
    pol = da.make_policy(split_mode=da.DA_SPLIT_DETERMINISTIC, cache_bits=4)
    c = Cache([700, 1300, 64], 8, 2, 128, seed=4)
    out, lse, _ = run(c, pol)
    one = Cache([700, 1300, 64], 8, 2, 128, seed=4)
    one.lens, one.table, one.q = [1300], one.table[1:2], one.q[1:2]
    alone, alone_lse, _ = run(one, pol)
    assert torch.equal(out[1:2], alone) and torch.equal(lse[1:2], alone_lse)
    again, again_lse, _ = run(c, pol)
    assert torch.equal(out, again) and torch.equal(lse, again_lse)
    fused, fused_lse, _ = run(c, da.make_policy(split_mode=da.DA_SPLIT_DETERMINISTIC, cache_bits=4, fuse_combine=1))
    assert torch.equal(out, fused) and torch.equal(lse, fused_lse)


@pytest.mark.parametrize("d", [64, 128])
def test_deterministic_bits_beside_many_others(d):
    """A sequence alone and in a batch of more (sequence, KV head) pairs than the device has multiprocessors."""
    pol = da.make_policy(split_mode=da.DA_SPLIT_DETERMINISTIC, cache_bits=4)
    lens = [1300, 700] + [5] * 40
    c, one = Cache(lens, 8, 8, d, seed=4), Cache(lens, 8, 8, d, seed=4)
    out, lse, _ = run(c, pol)
    for b in (0, 1, 20):
        one.lens, one.table, one.q = lens[b:b + 1], c.table[b:b + 1], c.q[b:b + 1]
        alone, alone_lse, _ = run(one, pol)
        assert torch.equal(out[b:b + 1], alone) and torch.equal(lse[b:b + 1], alone_lse)


@pytest.mark.parametrize("lens", [[900] * 20, [100] * 20, [1000, 17, 640] + [33] * 30])
@pytest.mark.parametrize("hq,dtype", [(8, "bf16"), (32, "fp16")])
def test_batches_of_either_size_of_blocks(lens, hq, dtype):
    """As many (sequence, KV head) pairs as the device has multiprocessors, or more, and fewer than it has small blocks."""
    c = Cache(lens, hq, 8, 128, dtype=dtype, seed=len(lens))
    out, lse, status = run(c)
    assert status == da.DA_OK
    check(c, out, lse, "either")
    pol = da.make_policy(cache_bits=4)
    sizes = {da.decode_attn_plan(da.make_kv4_shape(len(x), hq, 8, 128, 16, 70, 2000), pol, x).info().ctas_per_sm
             for x in ([900] * 20, [100] * 20)}
    assert len(sizes) == 2                             # (both kinds occur among these)


def test_capacity_plan_in_a_graph():
    a, b = Cache([40, 900, 3], 8, 2, 128, seed=31, width=70), Cache([1000, 16], 8, 2, 128, seed=32, width=70)
    for c in (a, b):
        c.num_pages = 100
        c.pool = np.pad(c.pool, ((0, 100 - len(c.pool)), (0, 0), (0, 0)))
    pol = da.make_policy(cache_bits=4, capacity_batch=4, capacity_tokens=2000)
    plan = da.decode_attn_plan(a.shape(), pol, a.lens)
    pool = torch.from_numpy(a.pool).cuda()
    table = torch.full((4, 70), -1, dtype=torch.int32, device="cuda")
    lens = torch.zeros(4, dtype=torch.int32, device="cuda")
    q = torch.zeros((4, 8, 128), dtype=torch.bfloat16, device="cuda")
    out, lse = torch.zeros((4, 8, 128), device="cuda"), torch.zeros((4, 8), device="cuda")
    ws = torch.empty(plan.workspace_bytes, dtype=torch.uint8, device="cuda")

    def load(c):
        n = len(c.lens)
        pool.copy_(torch.from_numpy(c.pool))
        table[:n].copy_(torch.from_numpy(c.table))
        lens[:n].copy_(torch.tensor(c.lens, dtype=torch.int32))
        q[:n].copy_(c.q)

    def step():
        da.decode_attn_run(plan, q, pool, None, table, lens, out, lse, ws)
        da.decode_attn_combine(plan, ws, out, lse)

    load(a)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        step()
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for c in (a, b, a):
        load(c)
        da.decode_attn_plan_update(plan, c.lens)
        graph.replay()
        assert da.decode_attn_last_device_status(plan) == da.DA_OK
        check(c, out[:len(c.lens)], lse[:len(c.lens)], "replayed")
    del graph
    plan.destroy()


def test_stale_lengths_void_their_rows():
    c = Cache([200, 100], 8, 2, 128, seed=6)
    plan = da.decode_attn_plan(c.shape(), da.make_policy(cache_bits=4), [200, 90])
    out, lse, status = run(c, plan=plan)
    plan.destroy()
    assert status == da.DA_ERR_STALE_PLAN
    want, _, mass, size = c.expect()
    assert (out[1] == 0).all() and torch.isneginf(lse[1]).all()
    c.lens, c.table, c.q = c.lens[:1], c.table[:1], c.q[:1]
    check(c, out[:1], lse[:1], "the row beside")


@pytest.mark.parametrize("bad", [-1, 1 << 20])
def test_pages_outside_the_pool_are_reported(bad):
    c = Cache([200, 100], 8, 2, 128, seed=6)
    c.table[1, 2] = bad
    out, lse, status = run(c)
    assert status == da.DA_ERR_BAD_PAGE
    c.lens, c.table, c.q = c.lens[:1], c.table[:1], c.q[:1]
    check(c, out[:1], lse[:1], "the row beside")


def test_what_a_packed_plan_refuses_at_a_call():
    c = Cache([100], 8, 2, 128)
    plan = da.decode_attn_plan(c.shape(), da.make_policy(cache_bits=4), c.lens)
    pool, table = torch.from_numpy(c.pool).cuda(), torch.from_numpy(c.table).cuda()
    lens = torch.tensor(c.lens, dtype=torch.int32).cuda()
    q, out = c.q.cuda(), torch.zeros((1, 8, 128), device="cuda")
    rows = torch.zeros((1, 2, 128), dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(max(plan.workspace_bytes, 256), dtype=torch.uint8, device="cuda")
    call = lambda **kw: da.decode_attn_run(plan, q, pool, kw.pop("v", None), table, lens, out, None, ws, check=False, **kw)
    assert call() == da.DA_OK
    assert call(v=pool) == da.DA_ERR_INVALID_ARG
    assert call(new_k=rows, new_v=rows) == da.DA_ERR_UNSUPPORTED
    assert da.decode_attn_append_kv_checked(plan, rows, rows, table, lens, pool, pool, check=False) == da.DA_ERR_UNSUPPORTED
    with pytest.raises(da.DecodeAttnError):
        da.decode_attn_gather_probe(plan, pool, pool, table, torch.zeros(99, dtype=torch.int32, device="cuda"))
    with pytest.raises(da.DecodeAttnError):
        da.decode_attn_debug_gather(plan, 0, pool, pool, table, rows, rows)
    assert da.decode_attn_debug_expire_wait(plan, q, pool, None, table, lens, out, None, ws) == da.DA_ERR_UNSUPPORTED  # (it has no such waits)
    assert da.decode_attn_last_device_status(plan) == da.DA_OK
    plan.destroy()
    plain = da.decode_attn_plan(da.make_shape(1, 8, 2, 128, 16, 7, 9, (16 * 256, 256, 128)), da.make_policy(), [100])
    assert da.decode_attn_run(plain, q, pool, None, table, lens, out, None, ws, check=False) == da.DA_ERR_INVALID_ARG
    plain.destroy()
