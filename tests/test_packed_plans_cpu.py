"""Plans of caches in 4 bits under small limits on the pieces of a sequence, by the thousand and without a GPU."""
import ctypes

import numpy as np
import pytest

pytest.importorskip("torch")

from packed_util import da  # noqa: E402

UNIT = np.dtype([(name, np.int32) for name, _ in da.Unit._fields_])


def layout(hkv, group, lens, policy, ctas, head_dim=128):
    """Units, pieces and first record of every sequence, and the number of records, as arrays."""
    shape = da.make_kv4_shape(len(lens), hkv * group, hkv, head_dim, 16, 4096, 1 << 20)
    lens = np.asarray(lens, dtype=np.int32)
    room = 300000 // 8
    units, n, slots, chunk = np.zeros(room, dtype=UNIT), ctypes.c_int64(), ctypes.c_int64(), ctypes.c_int32()
    splits, base = np.zeros(len(lens), dtype=np.int32), np.zeros(len(lens), dtype=np.int32)
    rc = da._lib.decode_attn_plan_layout(ctypes.byref(shape), ctypes.byref(policy), lens.ctypes.data, 148, ctas, units.ctypes.data, room,
                                         ctypes.byref(n), splits.ctypes.data, base.ctypes.data, ctypes.byref(slots), ctypes.byref(chunk))
    assert rc == da.DA_OK
    return units[:n.value], splits, base, slots.value


def check(hkv, lens, limit, units, splits, base, n_slots):
    """Every KV head's tokens once, in order; pieces and records as the tables of the sequences say."""
    lens = np.asarray(lens)
    assert ((splits >= 1) & (splits <= limit)).all()
    cut = splits > 1
    assert n_slots == splits[cut].sum() and (base[~cut] == -1).all()
    assert np.array_equal(base[cut], np.concatenate([[0], np.cumsum(splits[cut])[:-1]])[:cut.sum()])
    u = units[np.lexsort((units["split_index"], units["kv_head"], units["seq"]))]
    seq = np.repeat(np.arange(len(lens)), splits * hkv)
    assert np.array_equal(u["seq"], seq) and np.array_equal(u["n_splits"], splits[seq]) and np.array_equal(u["seq_len"], lens[seq])
    assert np.array_equal(u["kv_head"], np.concatenate([np.repeat(np.arange(hkv), s) for s in splits]))
    assert np.array_equal(u["split_index"], np.concatenate([np.tile(np.arange(s), hkv) for s in splits]))
    assert np.array_equal(u["slot"], np.where(cut[seq], base[seq] + u["split_index"], -1))
    # a piece begins where the one before it ended (empty ones lie at the end), the last ends with the sequence
    first = u["split_index"] == 0
    assert (u["tok_begin"][first] == 0).all()
    assert np.array_equal(u["tok_begin"][~first], u["tok_end"][:-1][~first[1:]])
    assert (u["tok_end"] >= u["tok_begin"]).all() and np.array_equal(u["tok_end"][np.append(first[1:], True)], lens[seq[np.append(first[1:], True)]])


@pytest.mark.parametrize("limit", [1, 2, 3, 4, 5, 6, 8])
@pytest.mark.parametrize("ctas", [2, 4])
def test_limits_on_the_pieces_of_a_sequence(limit, ctas):
    rng = np.random.default_rng(10 * limit + ctas)
    for i in range(600):
        hkv, chunk, most = (8, 0, 2000) if i % 2 else (int(rng.integers(1, 9)), int(rng.choice([0, 16, 48])), 6000)
        lens = rng.integers(1, most, size=int(rng.integers(40 if i % 2 else 20, 71)))
        policy = da.make_policy(cache_bits=4, max_splits=limit, chunk_tokens=chunk)
        check(hkv, lens, limit, *layout(hkv, 4, lens, policy, ctas))


@pytest.mark.parametrize("limit", [2, 3])
def test_a_share_that_no_trial_has_seen(limit):
    lens = [1662, 1955, 1732, 927, 334, 1066, 2537, 1769, 1539, 802, 2269, 2192, 1102, 2799, 1291, 2091, 2170, 1427, 198, 2687, 1235, 792, 397,
            65, 2428, 2123, 1124, 2006, 847, 2162, 797, 1965, 2779, 2456]
    for ctas in (2, 4):
        policy = da.make_policy(cache_bits=4, max_splits=limit, chunk_tokens=16)
        check(6, lens, limit, *layout(6, 4, lens, policy, ctas))
