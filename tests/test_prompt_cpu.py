"""The prompt planner without a GPU: its units cover every (query, visible position) once, blocks get equal shares,
and what is not built is refused."""
import random

import numpy as np
import pytest

from paper_2609_37062_b200 import build as da_build

da_build.build()
from paper_2609_37062_b200 import binding as da  # noqa: E402
from oracle import bounded_cache as bc  # noqa: E402


def shape(B, hq=32, hkv=8, page=16, mpp=1 << 16):
    return da.make_shape(B, hq, hkv, 128, page, mpp, 1 << 20, (page * hkv * 128, hkv * 128, 128))


def tile_list(u):
    """The whole tile list of a unit's tokens, from its fields."""
    return [i if i < u.sink_tiles else i - u.sink_tiles + u.window_tile for i in range(u.tile_begin, u.tile_end)]


def check(new, lens, policy, window=0, sinks=0, hq=32, hkv=8, sm=148):
    units, begin = da.decode_attn_prompt_plan_layout(shape(len(new), hq, hkv), policy, new, lens, sm)
    per_unit = 2 * (128 // (hq // hkv))
    assert begin[0] == 0 and begin[-1] == len(units) and (np.diff(begin) >= 0).all() and len(begin) - 1 <= sm
    rows = np.concatenate([[0], np.cumsum(new)])
    tiles, slots = {}, []
    for u in units:
        assert 1 <= u.n_tok <= per_unit and u.seq_len == lens[u.seq] and u.tile_begin < u.tile_end
        assert u.pos - u.row == lens[u.seq] - new[u.seq] - rows[u.seq]
        tiles.setdefault((u.seq, u.kv_head, u.row, u.n_tok, u.pos), []).append(u)
        if u.slot >= 0:
            slots.append(u.slot)
    assert sorted(slots) == list(range(len(slots)))
    seen_rows = {}
    for (b, g, row, n, pos), group in tiles.items():
        assert all(u.n_pieces == len(group) for u in group) and (len(group) > 1) == (group[0].slot >= 0)
        assert [u.slot for u in group] == [group[0].slot + i if len(group) > 1 else -1 for i in range(len(group))]
        listed = [t for u in group for t in tile_list(u)]
        t = np.arange(pos + n)
        seen = np.zeros(pos + n, dtype=bool)
        for i in (pos, pos + n - 1):
            seen |= bc.seen(i, t, window, sinks)
        seen |= (t >= pos)
        assert len(set(listed)) == len(listed) and listed == sorted(listed)
        assert set((t[seen] // 128).tolist()) <= set(listed)
        assert max(listed) == (pos + n - 1) // 128
        if window:                                            # nothing is listed that no query sees
            low = max(0, pos - window + 1)
            assert all(x * 128 < sinks or x * 128 + 127 >= low for x in listed)
        seen_rows.setdefault((b, g), []).append((row, n))
    for b in range(len(new)):
        for g in range(hkv):
            got = sorted(seen_rows.get((b, g), []))
            at = rows[b]
            for row, n in got:
                assert row == at
                at += n
            assert at == rows[b + 1]
    return units, begin


@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (100, 4), (128, 128), (1000, 300), (5000, 4), (2**31 - 1, 2**31 - 1)])
@pytest.mark.parametrize("mode", [da.DA_SPLIT_AUTO, da.DA_SPLIT_DETERMINISTIC])
def test_every_pair_is_covered_once(window, sinks, mode):
    pol = da.make_policy(window_tokens=window, sink_tokens=sinks, split_mode=mode)
    for new, lens in (([1], [1]), ([0], [0]), ([0], [77]), ([64], [64]), ([65, 0, 3], [65, 9, 4000]), ([1], [100_000]),
                      ([4096], [16384]), ([5, 700, 0, 1, 129], [5, 2000, 0, 8000, 129])):
        for hq, hkv in ((32, 8), (8, 8), (48, 4), (10, 2), (16, 1)):
            for sm in (148, 3):
                check(new, lens, pol, window, sinks, hq, hkv, sm)


@pytest.mark.parametrize("seed", range(6))
def test_random_batches(seed):
    rng = random.Random(seed)
    for _ in range(25):
        B = rng.randint(1, 9)
        new = [rng.choice([0, 1, 7, 64, 65, rng.randint(1, 3000)]) for _ in range(B)]
        lens = [n + rng.choice([0, 0, 1, rng.randint(1, 20_000)]) for n in new]
        window = rng.choice([0, 1, rng.randint(1, 5000)])
        sinks = rng.choice([0, 4, rng.randint(0, 500)]) if window else 0
        hq, hkv = rng.choice([(32, 8), (8, 8), (48, 4), (10, 2), (16, 1)])
        pol = da.make_policy(window_tokens=window, sink_tokens=sinks, split_mode=rng.choice([0, 2]), chunk_tokens=rng.choice([0, 128, 1024]))
        check(new, lens, pol, window, sinks, hq, hkv, rng.choice([148, 148, 20]))


def test_long_work_is_spread_evenly():
    for new, lens, kw in (([4096], [16384], dict(window_tokens=4096, sink_tokens=4)), ([1], [131072], {}), ([8192], [8192], {}),
                          ([300, 512, 450, 480], [2000, 9000, 5000, 7000], {})):
        units, begin = check(new, lens, da.make_policy(**kw), **{"window": kw.get("window_tokens", 0), "sinks": kw.get("sink_tokens", 0)})
        load = [sum(u.tile_end - u.tile_begin + 1 for u in units[a:b]) for a, b in zip(begin[:-1], begin[1:])]
        mean = sum(load) / len(load)
        assert max(load) <= 1.1 * mean + 8, (max(load), mean)
        assert len(load) == 148


def test_deterministic_pieces_depend_on_the_sequence_alone():
    pol = da.make_policy(split_mode=da.DA_SPLIT_DETERMINISTIC, chunk_tokens=512)
    key = lambda us, b: sorted((u.kv_head, u.pos, u.n_tok, u.tile_begin, u.tile_end) for u in us if u.seq == b)
    alone = da.decode_attn_prompt_plan_layout(shape(1), pol, [200], [3000], 148)[0]
    among = da.decode_attn_prompt_plan_layout(shape(3), pol, [9, 200, 4000], [9, 3000, 5000], 148)[0]
    assert key(alone, 0) == key(among, 1)


@pytest.mark.parametrize("kw,status", [
    (dict(kernel=da.DA_KERNEL_MMA_TMA), da.DA_ERR_UNSUPPORTED), (dict(fuse_combine=1), da.DA_ERR_UNSUPPORTED),
    (dict(capacity_batch=4, capacity_tokens=100), da.DA_ERR_UNSUPPORTED), (dict(track_weights=1), da.DA_ERR_UNSUPPORTED),
    (dict(shared_prefix_tokens=16), da.DA_ERR_UNSUPPORTED),
    (dict(split_mode=da.DA_SPLIT_FIXED_COUNT, fixed_count=2), da.DA_ERR_UNSUPPORTED),
    (dict(max_splits=4), da.DA_ERR_UNSUPPORTED), (dict(ctas_per_sm=1), da.DA_ERR_UNSUPPORTED),
    (dict(split_mode=da.DA_SPLIT_DETERMINISTIC, chunk_tokens=16), da.DA_ERR_INVALID_ARG),
    (dict(sink_tokens=4), da.DA_ERR_INVALID_ARG), (dict(window_tokens=-1), da.DA_ERR_INVALID_ARG)])
def test_policies_that_are_refused(kw, status):
    with pytest.raises(da.DecodeAttnError) as e:
        da.decode_attn_prompt_plan_layout(shape(1), da.make_policy(**kw), [10], [100], 148)
    assert e.value.status == status


def test_work_lists_too_long_to_make_are_refused():
    sh = da.make_shape(1, 16, 1, 64, 256, 1 << 23, 1 << 30, (256 * 64, 64, 64))
    for pol, new in ((da.make_policy(), 1 << 30), (da.make_policy(split_mode=da.DA_SPLIT_DETERMINISTIC, chunk_tokens=128), 1 << 20)):
        with pytest.raises(da.DecodeAttnError) as e:
            da.decode_attn_prompt_plan_layout(sh, pol, [new], [1 << 30], 148)
        assert e.value.status == da.DA_ERR_UNSUPPORTED


@pytest.mark.parametrize("new,lens", [([-1], [10]), ([11], [10]), ([1], [16 * 65536 + 1])])
def test_lengths_that_are_refused(new, lens):
    with pytest.raises(da.DecodeAttnError) as e:
        da.decode_attn_prompt_plan_layout(shape(1), da.make_policy(), new, lens, 148)
    assert e.value.status == da.DA_ERR_INVALID_ARG
