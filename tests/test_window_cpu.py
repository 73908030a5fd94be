"""Windowed plans without a GPU: what they refuse, and that their units cover exactly the visible tiles."""
import numpy as np
import pytest

from paper_2609_37062_b200 import build as da_build

da_build.build()
from paper_2609_37062_b200 import binding as da  # noqa: E402
from oracle import bounded_cache as bc  # noqa: E402


def shape(B, page=16, mpp=8192):
    return da.make_shape(B, 32, 8, 128, page, mpp, 1 << 20, (page * 8 * 128, 8 * 128, 128))


def layout(lens, policy, page=16):
    return da.decode_attn_plan_layout(shape(len(lens), page), policy, lens, 148, 2)


@pytest.mark.parametrize("kw", [dict(window_tokens=-1), dict(sink_tokens=-4, window_tokens=64), dict(sink_tokens=4),
                                dict(track_weights=2), dict(track_weights=-1)])
def test_bad_window_arguments_are_refused(kw):
    with pytest.raises(da.DecodeAttnError) as e:
        layout([100], da.make_policy(**kw))
    assert e.value.status == da.DA_ERR_INVALID_ARG


@pytest.mark.parametrize("kw", [dict(window_tokens=64), dict(track_weights=1)])
def test_windows_and_weights_are_refused_where_they_are_not_built(kw):
    for other in (dict(kernel=da.DA_KERNEL_SIMT), dict(shared_prefix_tokens=64)):
        with pytest.raises(da.DecodeAttnError) as e:
            layout([100], da.make_policy(**kw, **other))
        assert e.value.status == da.DA_ERR_UNSUPPORTED


def visible_tiles(L, window, sinks):
    t = np.arange(L)
    return sorted(set((t[bc.seen(L - 1, t, window, sinks)] // 16).tolist()))


@pytest.mark.parametrize("window,sinks", [(1, 0), (15, 0), (16, 1), (17, 4), (64, 37), (100, 16), (256, 4), (1024, 128),
                                          (5000, 4), (1, 5000), (1 << 30, 4), (2**31 - 1, 2**31 - 1)])
@pytest.mark.parametrize("mode", [da.DA_SPLIT_AUTO, da.DA_SPLIT_DETERMINISTIC, da.DA_SPLIT_FIXED_COUNT])
def test_units_cover_the_visible_tiles_once(window, sinks, mode):
    lens = [0, 1, 15, 16, 17, 31, 32, 33, 64, 100, 255, 256, 257, 300, 1000, 1024, 1025, 5003, 100_000]
    pol = da.make_policy(split_mode=mode, fixed_count=3, window_tokens=window, sink_tokens=sinks)
    units, splits, _, n_slots, _ = layout(lens, pol)
    per = {}
    for u in units:
        assert u.seq_len == lens[u.seq] and u.tok_begin % 16 == 0
        per.setdefault((u.seq, u.kv_head), []).append((u.tok_begin, u.tok_end))
    for b, L in enumerate(lens):
        tiles = visible_tiles(L, window, sinks) if L else []
        # visible positions: the visible tiles side by side, the last one as ragged as the sequence's end
        n = 16 * len(tiles) - ((-L) % 16 if tiles else 0)
        for g in range(8):
            spans = sorted(s for s in per[(b, g)] if s[1] > s[0])
            at = 0
            for lo, hi in spans:
                assert lo == at
                at = hi
            assert at == n, (b, L, at, n)


def test_a_window_as_long_as_the_sequences_changes_nothing():
    lens = [0, 17, 300, 4096, 32768]
    a = layout(lens, da.make_policy())
    b = layout(lens, da.make_policy(window_tokens=32768, sink_tokens=4))
    key = lambda us: [(u.seq, u.kv_head, u.tok_begin, u.tok_end, u.slot) for u in us]
    assert key(a[0]) == key(b[0]) and a[3] == b[3]


def test_deterministic_cuts_depend_on_the_sequence_alone():
    pol = da.make_policy(split_mode=da.DA_SPLIT_DETERMINISTIC, window_tokens=2000, sink_tokens=4)
    alone = [(u.kv_head, u.tok_begin, u.tok_end) for u in layout([9000], pol)[0]]
    among = [(u.kv_head, u.tok_begin, u.tok_end) for u in layout([5, 9000, 700, 30000], pol)[0] if u.seq == 1]
    assert sorted(alone) == sorted(among)
