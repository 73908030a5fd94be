"""Eviction without a GPU: the host check of its pages, and the numbers it refuses."""
import numpy as np
import pytest

from paper_2609_37062_b200 import build as da_build

da_build.build()
from paper_2609_37062_b200 import binding as da  # noqa: E402


def shape(B=2, page=16, mpp=8, pages=32, d=64):
    return da.make_shape(B, 8, 2, d, page, mpp, pages, (page * 2 * d, 2 * d, d))


BT = np.arange(16, dtype=np.int32).reshape(2, 8)
DST = np.array([[20, 21], [22, 23]], dtype=np.int32)


def validate(budget=32, sinks=4, recent=8, lens=(100, 20), bt=BT, dst=DST, sh=None):
    return da.decode_attn_validate_evict(sh or shape(), budget, sinks, recent, lens, bt, dst)


def test_fresh_pages_are_accepted():
    assert validate() == da.DA_OK
    assert validate(lens=(0, 0)) == da.DA_OK
    assert da.decode_attn_validate_evict(shape(B=0), 32, 0, 0, [], np.zeros((0, 8)), np.zeros((0, 2))) == da.DA_OK


@pytest.mark.parametrize("kw", [dict(budget=0), dict(budget=-1), dict(sinks=-1), dict(recent=-1), dict(sinks=30, recent=3),
                                dict(sinks=2**31 - 1, recent=2**31 - 1), dict(budget=33), dict(lens=(-1, 5)), dict(lens=(129, 5))])
def test_bad_numbers_are_refused(kw):
    assert validate(**kw) == da.DA_ERR_INVALID_ARG


def test_bad_pages_are_refused():
    def with_entry(a, i, j, v):
        a = a.copy()
        a[i, j] = v
        return a
    assert validate(bt=with_entry(BT, 0, 2, 32)) == da.DA_ERR_BAD_PAGE        # outside the pool
    assert validate(bt=with_entry(BT, 0, 7, -1)) == da.DA_OK                  # 100 tokens: seven pages
    assert validate(dst=with_entry(DST, 0, 1, -1)) == da.DA_ERR_BAD_PAGE
    assert validate(dst=with_entry(DST, 0, 1, 20)) == da.DA_ERR_BAD_PAGE      # named twice
    assert validate(dst=with_entry(DST, 0, 1, 9)) == da.DA_ERR_BAD_PAGE       # read by the other row
    assert validate(dst=with_entry(DST, 0, 1, 15)) == da.DA_OK                # behind that row's end: nobody's
    assert validate(dst=with_entry(DST, 1, 0, -1)) == da.DA_OK                # that row is within the budget
    assert validate(dst=with_entry(DST, 1, 0, -1), lens=(100, 33)) == da.DA_ERR_BAD_PAGE


def test_calls_are_refused_before_they_reach_a_device():
    import ctypes
    sh = shape()
    a = da._evict_args(32, 4, 8, 2)
    call = lambda: da._lib.decode_attn_evict(ctypes.byref(sh), ctypes.byref(a), None)
    assert call() == da.DA_ERR_INVALID_ARG                                    # no pointers
    fake = 1 << 20
    for name in ("seq_lens", "block_table", "dst_block_table", "k_cache", "v_cache", "weights", "weights_out", "kept"):
        setattr(a, name, fake)
    a.seq_lens_out = fake
    a.weight_tokens = a.stride_seq = a.stride_head = 128
    assert call() == da.DA_ERR_INVALID_ARG                                    # the new lengths over the old ones
    a.seq_lens_out = fake + 64
    for name, bad in (("weight_tokens", 0), ("stride_head", 100), ("stride_seq", 100), ("k_cache", fake + 8), ("struct_size", 8),
                      ("flags", 1), ("dst_max_pages", 1), ("status", fake + 2), ("kept", fake + 1)):
        good = getattr(a, name)
        setattr(a, name, bad)
        assert call() == da.DA_ERR_INVALID_ARG, name
        setattr(a, name, good)


def layout_status(T, stride_seq, stride_head, batch=1 << 30, heads=2):
    """What the call says to rows of totals laid out like this.  Of some 2^31 rows with budgets of 512 tokens, more than a
    launch takes: a layout that is accepted is answered with DA_ERR_UNSUPPORTED, before any device is asked."""
    import ctypes
    sh = da.make_shape(batch, heads, heads, 64, 16, 8, 32, (16 * heads * 64, heads * 64, 64))
    a = da._evict_args(512, 4, 8, 32)
    for i, name in enumerate(("seq_lens", "block_table", "dst_block_table", "k_cache", "v_cache", "weights", "weights_out", "kept",
                              "seq_lens_out")):
        setattr(a, name, (i + 1) << 20)
    a.weight_tokens, a.stride_seq, a.stride_head = T, stride_seq, stride_head
    assert batch * heads * (512 // 32) // 8 > 2**31 - 1
    return da._lib.decode_attn_evict(ctypes.byref(sh), ctypes.byref(a), None)


@pytest.mark.parametrize("T", [1, 128, 1000])
def test_overlapping_rows_of_totals_are_refused(T):
    B = 1 << 30
    for stride_seq, stride_head in ((2 * T, T), (3 * T, T), (2 * T + 1, T + 1), (T, B * T), (T + 3, B * (T + 3)),
                                    (2 * T, 3 * T), (2 * T, 7 * T), (5 * T, 3 * T),
                                    (2**60, 2**61 + 2**59), (2**62, T)):      # interleaved rows lie apart too
        assert layout_status(T, stride_seq, stride_head) == da.DA_ERR_UNSUPPORTED, (stride_seq, stride_head)
    for stride_seq, stride_head in ((T, T), (2 * T, 2 * T), (2 * T, 4 * T), (T, 7 * T), (2 * T - 1, T), (T, (B - 1) * T),
                                    (2 * T + 2, T - 1), (T - 1, B * T), (0, T), (T, 0), (-2 * T, T), (2**62, 2**62)):
        assert layout_status(T, stride_seq, stride_head) == da.DA_ERR_INVALID_ARG, (stride_seq, stride_head)
    # one KV head, or one sequence: its stride does not matter
    for any_stride in (0, 1, T, -5):
        assert layout_status(T, T, any_stride, batch=2**31 - 1, heads=1) == da.DA_ERR_UNSUPPORTED
        assert layout_status(T, any_stride, T, batch=1, heads=2**31 - 1) == da.DA_ERR_UNSUPPORTED
    assert layout_status(T, T - 1, 0, batch=2**31 - 1, heads=1) == da.DA_ERR_INVALID_ARG
    assert layout_status(T, 0, T - 1, batch=1, heads=2**31 - 1) == da.DA_ERR_INVALID_ARG


def test_rows_lie_apart_exactly_when_no_two_share_a_value():
    """All small layouts against the definition, through the host-only check that both entry points share."""
    import itertools
    T = 3
    for stride_seq, stride_head, heads in itertools.product(range(1, 22), range(1, 22), (2, 3, 5)):
        # (a batch so large that a launch refuses it has every row of a smaller one: the definition needs some 2 * heads * 21 / T)
        rows = np.arange(200)[:, None] * stride_seq + np.arange(heads)[None, :] * stride_head
        values = (rows.reshape(-1, 1) + np.arange(T)).ravel()
        apart = len(np.unique(values)) == len(values)
        got = layout_status(T, stride_seq, stride_head, batch=(1 << 31) // heads + 1, heads=heads)
        assert got == (da.DA_ERR_UNSUPPORTED if apart else da.DA_ERR_INVALID_ARG), (stride_seq, stride_head, heads)
