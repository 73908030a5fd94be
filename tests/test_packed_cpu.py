"""Refusals of the calls around a cache in 4 bits, step tables and rows, which need no GPU; the planner and the format."""
import ctypes

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import packed_cache as ref  # noqa: E402
from packed_util import Cache, da  # noqa: E402

FAKE = 1 << 20                                                                 # an address that no refused call looks at


def plan_layout(policy, **kw):
    args = dict(batch=2, num_q_heads=8, num_kv_heads=2, head_dim=128, page_size=16, max_pages_per_seq=100, num_pages=300) | kw
    return da.decode_attn_plan_layout(da.make_kv4_shape(**args), policy, [1000, 77][:args["batch"]], 148, 2)


def status_of(call, *a, **kw):
    with pytest.raises(da.DecodeAttnError) as e:
        call(*a, **kw)
    return e.value.status


def test_plans_are_those_of_sixteen_bits():
    lens = [1000, 77]
    for kw in ({}, {"split_mode": da.DA_SPLIT_DETERMINISTIC}, {"window_tokens": 100, "sink_tokens": 4}):
        a = plan_layout(da.make_policy(cache_bits=4, **kw))
        shape = da.make_shape(2, 8, 2, 128, 16, 100, 300, (16 * 256, 256, 128))
        for bits in (0, 16):
            b = da.decode_attn_plan_layout(shape, da.make_policy(cache_bits=bits, **kw), lens, 148, 2)
            assert [bytes(x) for x in a[0]] == [bytes(x) for x in b[0]] and a[3:] == b[3:]


@pytest.mark.parametrize("seed", range(30))
def test_tiles_dealt_evenly_cover_every_token_once(seed):
    """Whatever the mix: every KV head's tokens in order, pieces of at least the smallest chunk, slots of their own, and no
    more records than a capacity plan has room for."""
    rng = np.random.default_rng(seed)
    hkv, group, ctas = int(rng.integers(1, 9)), int(rng.integers(1, 17)), int(rng.choice([2, 4]))
    lens = [int(rng.choice([0, 1, rng.integers(1, 200), rng.integers(1, 40000)])) for _ in range(int(rng.integers(1, 70)))]
    shape = da.make_kv4_shape(len(lens), hkv * group, hkv, 128, 16, 4096, 1 << 20)
    least = int(rng.choice([16, 64, 256]))
    pol = da.make_policy(cache_bits=4, chunk_tokens=least)
    units, splits, base, n_slots, _ = da.decode_attn_plan_layout(shape, pol, lens, 148, ctas)
    per, slots = {}, set()
    for u in units:
        per.setdefault((u.seq, u.kv_head), []).append(u)
        assert u.n_splits == splits[u.seq] and u.seq_len == lens[u.seq]
        assert u.slot == (base[u.seq] + u.split_index if u.n_splits > 1 else -1)
        if u.slot >= 0:
            assert (u.slot, u.kv_head) not in slots and u.slot < n_slots
            slots.add((u.slot, u.kv_head))
    assert len(per) == len(lens) * hkv
    for (b, g), mine in per.items():
        mine.sort(key=lambda u: u.split_index)
        assert [u.split_index for u in mine] == list(range(splits[b]))
        at = 0
        for u in mine:
            assert u.tok_begin % 16 == 0 or u.tok_begin == u.tok_end
            if u.tok_end > u.tok_begin:
                assert u.tok_begin == at
                at = u.tok_end
                assert u.n_splits == 1 or u.tok_end - u.tok_begin > least - 16 or lens[b] <= 2 * least
        assert at == lens[b]
    assert n_slots <= -(-sum(lens) // least) + len(lens)


@pytest.mark.parametrize("kw,want", [
    (dict(cache_bits=8), da.DA_ERR_INVALID_ARG), (dict(cache_bits=-4), da.DA_ERR_INVALID_ARG),
    (dict(cache_bits=4, track_weights=1), da.DA_ERR_UNSUPPORTED), (dict(cache_bits=4, shared_prefix_tokens=64), da.DA_ERR_UNSUPPORTED),
    (dict(cache_bits=4, kernel=da.DA_KERNEL_SIMT), da.DA_ERR_UNSUPPORTED), (dict(cache_bits=4, kernel=da.DA_KERNEL_MMA_TMA), da.DA_ERR_UNSUPPORTED),
    (dict(cache_bits=4, kernel=5), da.DA_ERR_INVALID_ARG)])
def test_policies_refused(kw, want):
    assert status_of(plan_layout, da.make_policy(**kw)) == want


def test_the_packed_kernel_serves_packed_caches_only():
    shape = da.make_shape(2, 8, 2, 128, 16, 100, 300, (16 * 256, 256, 128))
    for bits in (0, 16):
        pol = da.make_policy(kernel=da.DA_KERNEL_PACKED, cache_bits=bits)
        assert status_of(da.decode_attn_plan_layout, shape, pol, [5, 5], 148, 2) == da.DA_ERR_UNSUPPORTED
    pol = da.make_policy(kernel=da.DA_KERNEL_PACKED, shared_prefix_tokens=16)
    assert status_of(da.decode_attn_plan_layout, shape, pol, [50, 50], 148, 2) == da.DA_ERR_UNSUPPORTED


HEAD = 2304                                                                    # bytes of 16 tokens of one head of 128


@pytest.mark.parametrize("strides,want", [
    ((2 * HEAD, HEAD), None), ((HEAD, 300 * HEAD), None), ((2 * HEAD + 16, HEAD + 16), None),
    ((2 * HEAD + 8, HEAD), da.DA_ERR_INVALID_ARG), ((2 * HEAD, HEAD - 16), da.DA_ERR_INVALID_ARG),
    ((HEAD, HEAD), da.DA_ERR_INVALID_ARG), ((0, HEAD), da.DA_ERR_INVALID_ARG), ((2 * HEAD, -HEAD), da.DA_ERR_INVALID_ARG),
    ((HEAD, 299 * HEAD), da.DA_ERR_INVALID_ARG)])
def test_pool_strides(strides, want):
    call = lambda: plan_layout(da.make_policy(cache_bits=4), strides=strides)
    if want is None:
        call()
    else:
        assert status_of(call) == want


def test_shapes_refused():
    pol = da.make_policy(cache_bits=4)
    for kw in (dict(num_q_heads=34), dict(num_pages=0), dict(in_dtype=da.DA_DTYPE_FP32)):
        assert status_of(plan_layout, pol, **kw) in (da.DA_ERR_UNSUPPORTED, da.DA_ERR_INVALID_ARG)
    for d, page in ((96, 16), (256, 16), (128, 8), (128, 48), (128, 512), (0, 16), (128, 0)):
        assert da.decode_attn_packed_head_bytes(d, page) == 0
        shape = da.make_shape(1, 8, 2, d, page, 100, 300, (1 << 20, 1 << 10, 1 << 18))
        assert status_of(da.decode_attn_plan_layout, shape, pol, [5], 148, 2) in (da.DA_ERR_UNSUPPORTED, da.DA_ERR_INVALID_ARG)
    assert da.decode_attn_packed_head_bytes(128, 64) == 4 * HEAD == 4 * ref.tile_bytes(128)
    assert da.decode_attn_packed_head_bytes(64, 16) == ref.tile_bytes(64) == 1152


def test_other_calls_refuse_the_policy():
    shape = da.make_shape(1, 8, 2, 128, 16, 10, 10, (16 * 256, 256, 128))
    pol = da.make_policy(cache_bits=4)
    assert status_of(da.decode_attn_prompt_plan_layout, shape, pol, [4], [9], 148) == da.DA_ERR_UNSUPPORTED
    x = np.zeros(16, dtype=np.int16)
    i = np.zeros(16, dtype=np.int32)
    assert status_of(da.decode_attn_host_step, shape, pol, x, x, x, i, i, x) == da.DA_ERR_UNSUPPORTED


def test_the_oracle_format_round_trips():
    c = Cache([40, 3], 2, 2, 64, page=32, seed=1)
    code, scale = ref.encode(c.k)
    again, scale2 = ref.encode(ref.values(code, scale))
    assert np.array_equal(ref.values(code, scale), ref.values(again, scale2))
    for d in (64, 128):                                                        # every byte of a tile is somebody's, once
        seen = np.zeros(ref.tile_bytes(d), dtype=int)
        for which in ("k", "v"):
            b, s = ref._index(d, which)
            np.add.at(seen, b[:, 0::2].ravel(), 1)
            np.add.at(seen, s.ravel(), 1)
            np.add.at(seen, s.ravel() + 1, 1)
            assert np.array_equal(b[:, 0::2], b[:, 1::2])
        assert (seen == 1).all()


# ------------------------------------------------------------------------------------------------ rows

def rows_args(**kw):
    a = da.RowsArgs()
    a.struct_size = ctypes.sizeof(da.RowsArgs)
    a.rows, a.eps, a.rotary_dim, a.max_positions = 3, 1e-6, 128, 10
    a.q = a.k = a.v = a.q_out = a.k_cache = a.v_cache = a.cos_sin = a.positions = a.slots = a.q_weight = a.k_weight = FAKE
    a.q_stride, a.k_stride, a.v_stride, a.q_out_stride, a.k_out_stride = 1024, 256, 256, 1024, 256
    for name, x in kw.items():
        setattr(a, name, x)
    return a


def rows_status(shape=None, **kw):
    shape = shape or da.make_shape(0, 8, 2, 128, 16, 0, 300, (16 * 256, 256, 128))
    return da._lib.decode_attn_prepare_rows(ctypes.byref(shape), ctypes.byref(rows_args(**kw)), None)


@pytest.mark.parametrize("kw", [
    dict(struct_size=8), dict(flags=1), dict(rows=-1), dict(cache_bits=8), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")),
    dict(interleaved=2), dict(rotary_dim=4), dict(rotary_dim=132), dict(rotary_dim=136), dict(rotary_dim=0), dict(max_positions=0),
    dict(cos_sin=None), dict(cos_sin=FAKE + 4), dict(v_cache=None), dict(k_cache=None), dict(q_out=None), dict(q=None),
    dict(k=None), dict(v=None), dict(positions=None), dict(slots=None), dict(q_stride=1016), dict(q_stride=1028), dict(k_stride=255),
    dict(v_stride=0), dict(q_out_stride=1016), dict(k_out=FAKE, k_out_stride=0), dict(q=FAKE + 8), dict(k=FAKE + 2), dict(q_weight_stride=64),
    dict(k_weight=FAKE + 8), dict(k_weight_stride=-128), dict(positions=FAKE + 2), dict(slots=FAKE + 4), dict(status=FAKE + 1),
    dict(k_cache=FAKE + 8), dict(cache_bits=4), dict(q=None, q_out=None, k=None, v=None, k_cache=None, v_cache=None)])
def test_rows_refused(kw):
    assert rows_status(**kw) == da.DA_ERR_INVALID_ARG


def test_rows_with_a_packed_pool_refused():
    shape = da.make_kv4_shape(0, 8, 2, 128, 16, 0, 300)
    assert rows_status(shape) == da.DA_ERR_INVALID_ARG                         # (not its strides)
    assert rows_status(shape, cache_bits=4) == da.DA_ERR_INVALID_ARG           # v_cache
    assert rows_status(shape, cache_bits=4, v_cache=None, k_cache=None, v=None, k_out=FAKE) == da.DA_ERR_INVALID_ARG
    assert rows_status(shape, cache_bits=4, v_cache=None, rows=0) == da.DA_OK


def test_groups_that_no_attention_serves_refused():
    assert rows_status(da.make_shape(0, 17, 1, 128, 16, 0, 300, (16 * 128, 128, 128)), q_stride=17 * 128, q_out_stride=17 * 128) == \
        da.DA_ERR_UNSUPPORTED


def test_nothing_to_prepare():
    assert rows_status(rows=0) == da.DA_OK


def test_rows_binding_refuses():
    shape = da.make_shape(0, 8, 2, 128, 16, 0, 300, (16 * 256, 256, 128))
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)
    slots, pos = torch.zeros(4, dtype=torch.int64), torch.zeros(4, dtype=torch.int32)
    good = dict(q=bf(4, 8, 128), k=bf(4, 2, 128), v=bf(4, 2, 128), slots=slots, positions=pos, q_out=bf(4, 8, 128), k_cache=bf(1), v_cache=bf(1),
                rows=4)
    for bad in (dict(q=bf(4, 8, 64)), dict(q=bf(3, 8, 128)), dict(k=bf(4, 2, 128).half()), dict(v=bf(4, 4, 128)[:, ::2]),
                dict(q=bf(4, 8, 256)[..., ::2]), dict(slots=slots.int()), dict(slots=slots[:3]), dict(positions=pos.long()),
                dict(cos_sin=torch.zeros(9, 128).double()), dict(cos_sin=torch.zeros(9)), dict(q_weight=bf(64)), dict(q_weight=bf(8, 128).T),
                dict(status=torch.zeros(1)), dict(k_weight=bf(4, 128))):
        args = good | bad
        assert status_of(da.decode_attn_prepare_rows, shape, args.pop("q"), args.pop("k"), args.pop("v"), **args) == da.DA_ERR_INVALID_ARG


# ------------------------------------------------------------------------------------------------ tables

def tables_status(shape=None, **kw):
    shape = shape or da.make_shape(4, 8, 2, 64, 16, 10, 99, (16 * 128, 128, 64))
    a = da.TablesArgs()
    a.struct_size = ctypes.sizeof(da.TablesArgs)
    a.max_rows, a.free_capacity = 5, 9
    for name in ("seq_lens", "gains", "seq_lens_out", "block_table", "free_pages", "free_count", "free_count_out", "row_starts", "page_starts",
                 "slots", "positions", "row_seq", "status"):
        setattr(a, name, FAKE)
    for name, x in kw.items():
        setattr(a, name, x)
    return da._lib.decode_attn_step_tables(ctypes.byref(shape), ctypes.byref(a), None)


@pytest.mark.parametrize("kw", [dict(struct_size=4), dict(flags=2), dict(max_rows=-1), dict(free_capacity=-1)] +
                         [{n: None} for n in ("seq_lens", "gains", "seq_lens_out", "block_table", "free_pages", "free_count", "free_count_out",
                                              "row_starts", "page_starts", "slots", "positions")] +
                         [{n: FAKE + 2} for n in ("seq_lens", "gains", "seq_lens_out", "block_table", "free_pages", "free_count",
                                                  "free_count_out", "row_starts", "page_starts", "positions", "row_seq", "status")] +
                         [dict(slots=FAKE + 4)])
def test_tables_refused(kw):
    assert tables_status(**kw) == da.DA_ERR_INVALID_ARG


def test_table_shapes_refused():
    make = lambda **kw: da.make_shape(**(dict(batch=4, num_q_heads=8, num_kv_heads=2, head_dim=64, page_size=16, max_pages_per_seq=10,
                                             num_pages=99, k_strides=(16 * 128, 128, 64)) | kw))
    assert tables_status(make(batch=-1)) == da.DA_ERR_INVALID_ARG
    assert tables_status(make(num_pages=0)) == da.DA_ERR_INVALID_ARG
    assert tables_status(make(max_pages_per_seq=-1)) == da.DA_ERR_INVALID_ARG
    for page in (0, 8, 24, 512):
        assert tables_status(make(page_size=page)) == da.DA_ERR_UNSUPPORTED


def test_tables_binding_refuses():
    shape = da.make_shape(4, 8, 2, 64, 16, 10, 99, (16 * 128, 128, 64))
    i = lambda *s: torch.zeros(s, dtype=torch.int32)
    good = dict(seq_lens=i(4), gains=i(4), seq_lens_out=i(4), block_table=i(4, 10), free_pages=i(9), free_count=i(1), free_count_out=i(1),
                row_starts=i(5), page_starts=i(5), slots=torch.zeros(6, dtype=torch.int64), positions=i(6), row_seq=i(6), status=i(1))
    for bad in (dict(seq_lens=i(3)), dict(gains=i(4).long()), dict(block_table=i(4, 9)), dict(block_table=i(10, 4).T), dict(row_starts=i(4)),
                dict(page_starts=i(4)), dict(slots=i(6)), dict(positions=i(5)), dict(row_seq=i(5)), dict(free_count=i(0)),
                dict(slots=torch.zeros(12, dtype=torch.int64)[::2]), dict(status=torch.zeros(1))):
        assert status_of(da.decode_attn_step_tables, shape, **(good | bad)) == da.DA_ERR_INVALID_ARG


# ------------------------------------------------------------------------------------------------ expand

def expand_status(shape=None, packed=None, **kw):
    shape = shape or da.make_shape(2, 8, 2, 128, 16, 10, 30, (16 * 256, 256, 128))
    packed = packed or da.make_kv4_shape(2, 8, 2, 128, 16, 12, 40)
    p = dict(pool=FAKE, table=FAKE, lens=FAKE, dst=FAKE, k=FAKE, v=FAKE, status=None) | kw
    return da._lib.decode_attn_expand_kv(ctypes.byref(shape), ctypes.byref(packed), p["pool"], p["table"], p["lens"], p["dst"], p["k"], p["v"],
                                         p["status"], None)


def test_expanding_refused():
    for name in ("pool", "table", "lens", "dst", "k", "v"):
        assert expand_status(**{name: None}) == da.DA_ERR_INVALID_ARG
        assert expand_status(**{name: FAKE + 2}) == da.DA_ERR_INVALID_ARG
    assert expand_status(status=FAKE + 1) == da.DA_ERR_INVALID_ARG
    kv4 = lambda **kw: da.make_kv4_shape(**(dict(batch=2, num_q_heads=8, num_kv_heads=2, head_dim=128, page_size=16, max_pages_per_seq=12,
                                                num_pages=40) | kw))
    for kw in (dict(batch=3), dict(num_kv_heads=4), dict(head_dim=64), dict(page_size=32), dict(strides=(HEAD, HEAD))):
        assert expand_status(packed=kv4(**kw)) == da.DA_ERR_INVALID_ARG
    assert expand_status(packed=kv4(max_pages_per_seq=0)) == da.DA_OK           # no table, nothing to do
