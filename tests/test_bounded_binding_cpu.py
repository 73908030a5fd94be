"""What the binding refuses of an eviction's and the totals' tensors, before the library sees their addresses."""
import pytest
import torch

from paper_2609_37062_b200 import build as da_build

da_build.build()
from paper_2609_37062_b200 import binding as da  # noqa: E402

B, HKV, BUDGET, TOKENS = 3, 2, 40, 100


def tensors():
    return dict(seq_lens=torch.zeros(B, dtype=torch.int32), block_table=torch.zeros((B, 8), dtype=torch.int32),
                dst_block_table=torch.zeros((B, 4), dtype=torch.int32), k_cache=torch.zeros(1 << 16, dtype=torch.int16),
                v_cache=torch.zeros(1 << 16, dtype=torch.int16), weights=torch.zeros((B, HKV, TOKENS)), weights_out=None,
                kept=torch.zeros((B, HKV, BUDGET), dtype=torch.int32), seq_lens_out=torch.zeros(B, dtype=torch.int32),
                status=torch.zeros(1, dtype=torch.int32))


@pytest.fixture
def passed_on(monkeypatch):
    """The arguments that reach the library; nothing is called."""
    calls = []

    class Library:
        decode_attn_strerror = da._lib.decode_attn_strerror

        def __getattr__(self, name):
            return lambda *a: calls.append((name, a)) or 0
    monkeypatch.setattr(da, "_lib", Library())
    return calls


def evict(batch=B, **change):
    sh = da.make_shape(batch, 8, HKV, 64, 16, 8, 32, (16 * HKV * 64, HKV * 64, 64))
    t = tensors()
    t.update(change)
    return da.decode_attn_evict(sh, BUDGET, 4, 8, **t, stream=1)


def stride_of(calls):
    return calls[-1][1][1]._obj.dst_max_pages


def test_tables_that_are_columns_of_wider_ones(passed_on):
    evict()
    assert stride_of(passed_on) == 4
    evict(dst_block_table=torch.zeros((B, 9), dtype=torch.int32)[:, 2:6])
    assert stride_of(passed_on) == 9
    for one in (torch.zeros((1, 4), dtype=torch.int32), torch.zeros(4, dtype=torch.int32).as_strided((1, 4), (0, 1)),
                torch.zeros(64, dtype=torch.int32).as_strided((1, 4), (2, 1))):
        evict(batch=1, dst_block_table=one)
        assert stride_of(passed_on) == 4


@pytest.mark.parametrize("change", [
    dict(dst_block_table=torch.zeros(4, dtype=torch.int32).expand(B, 4)),               # one row for all: rows would be read behind it
    dict(dst_block_table=torch.zeros(12, dtype=torch.int32).as_strided((B, 4), (3, 1))),
    dict(dst_block_table=torch.zeros((4, B), dtype=torch.int32).t()),
    dict(dst_block_table=torch.zeros((B, 2), dtype=torch.int32)),                       # fewer pages than the budget
    dict(dst_block_table=torch.zeros((B - 1, 4), dtype=torch.int32)),
    dict(dst_block_table=torch.zeros((B, 4), dtype=torch.int64)),
    dict(kept=torch.zeros((B, HKV, BUDGET - 1), dtype=torch.int32)),
    dict(kept=torch.zeros((B, HKV, BUDGET), dtype=torch.int16)),
    dict(kept=torch.zeros((B, BUDGET, HKV), dtype=torch.int32).transpose(1, 2)),
    dict(seq_lens_out=torch.zeros(B - 1, dtype=torch.int32)),
    dict(seq_lens_out=torch.zeros(2 * B, dtype=torch.int32)[::2]),
    dict(seq_lens_out=torch.zeros(B, dtype=torch.int16)),
    dict(status=torch.zeros(1, dtype=torch.int16)),
    dict(weights=torch.zeros((B, HKV, TOKENS), dtype=torch.float16)),
    dict(weights=torch.zeros((B, HKV, TOKENS), dtype=torch.float64)),
    dict(weights=torch.zeros((B, HKV * TOKENS))),
    dict(weights=torch.zeros((B, HKV + 1, TOKENS))),
    dict(weights_out=torch.zeros((B, HKV, TOKENS), dtype=torch.bfloat16)),
    dict(weights_out=torch.zeros((B, TOKENS, HKV)).transpose(1, 2)),
], ids=lambda c: next(iter(c)))
def test_what_the_library_could_not_read_is_refused(passed_on, change):
    with pytest.raises(da.DecodeAttnError) as e:
        evict(**change)
    assert e.value.status == da.DA_ERR_INVALID_ARG and not passed_on


def test_totals_of_another_type_are_refused(passed_on):
    sh = da.make_shape(B, 8, HKV, 64, 16, 8, 32, (16 * HKV * 64, HKV * 64, 64))
    plan = da.Plan(0, 0, sh, da.make_policy(track_weights=1))
    add = lambda *w: da.decode_attn_add_weights(plan, 256, 256, 256, *w, stream=1)
    add(torch.zeros((B, HKV, TOKENS)))
    assert len(passed_on) == 1
    for bad in (torch.zeros((B, HKV, TOKENS), dtype=torch.float16), torch.zeros((B, HKV, TOKENS), dtype=torch.int32),
                torch.zeros((B, TOKENS))):
        with pytest.raises(da.DecodeAttnError):
            add(bad)
    with pytest.raises(da.DecodeAttnError):
        add(torch.zeros((B, HKV, TOKENS)), torch.zeros((B, HKV, TOKENS), dtype=torch.float64))
    assert len(passed_on) == 1
