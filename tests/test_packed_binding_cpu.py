"""Tables that the expansion would misread are refused ahead of the library."""
import pytest

torch = pytest.importorskip("torch")

from packed_util import da  # noqa: E402


def test_expanding_refuses_tables_of_other_types_sizes_and_strides():
    shape, packed = da.make_shape(3, 8, 2, 128, 16, 10, 30, (16 * 256, 256, 128)), da.make_kv4_shape(3, 8, 2, 128, 16, 12, 40)
    i = lambda *s: torch.zeros(s, dtype=torch.int32)
    pools = [torch.zeros(64, dtype=torch.uint8) for _ in range(3)]
    good = dict(block_table=i(3, 12), seq_lens=i(3), dst_block_table=i(3, 10), status=i(1))
    for bad in (dict(block_table=i(3, 12).long()), dict(block_table=i(3, 20)[:, :12]), dict(block_table=i(3, 11)), dict(block_table=i(12, 3).T),
                dict(seq_lens=i(3).long()), dict(seq_lens=i(2)), dict(seq_lens=i(6)[::2]), dict(dst_block_table=i(3, 9)),
                dict(dst_block_table=i(3, 20)[:, 5:15]), dict(dst_block_table=i(3, 10).short()), dict(status=torch.zeros(1)), dict(status=i(0))):
        args = good | bad
        with pytest.raises(da.DecodeAttnError) as e:
            da.decode_attn_expand_kv(shape, packed, pools[0], args["block_table"], args["seq_lens"], args["dst_block_table"], *pools[1:],
                                     args["status"], stream=0)
        assert e.value.status == da.DA_ERR_INVALID_ARG
