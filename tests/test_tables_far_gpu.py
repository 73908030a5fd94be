"""Step tables asked for more rows than 32 bits count."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from packed_util import da  # noqa: E402


@pytest.mark.parametrize("many,gain", [(4, 1 << 30), (5, (1 << 30) + 7), (1024, 1 << 22), (1030, 1 << 22), (2048, 1 << 21), (4096, 1 << 20)])
@pytest.mark.parametrize("max_rows", [100, 9000])
def test_sums_of_rows_beyond_32_bits(many, gain, max_rows):
    """Sequences that ask for 2^32 tokens together and more, with pages for all of them, behind one and ahead of two that ask for a token
    each: the first is served, all others are refused."""
    page, n = 256, many + 3
    width, pages = (gain + 5 + page - 1) // page, many * ((gain + 5) // page + 1) + 10
    i32 = dict(dtype=torch.int32, device="cuda")
    shape = da.make_shape(n, 8, 2, 64, page, width, pages + n, (page * 128, 128, 64))
    lens, gains = torch.full((n,), 5, **i32), torch.full((n,), gain, **i32)
    gains[0] = gains[-2:] = 1
    table = torch.full((n, width), -1, **i32)
    table[:, 0] = pages + torch.arange(n, **i32)
    before = table.clone()
    free, count, left = torch.arange(pages, **i32), torch.tensor([pages], **i32), torch.zeros(1, **i32)
    starts, page_starts = torch.zeros(n + 1, **i32), torch.zeros(n + 1, **i32)
    slots = torch.zeros(max_rows, dtype=torch.int64, device="cuda")
    positions, seq, status, after = torch.zeros(max_rows, **i32), torch.zeros(max_rows, **i32), torch.zeros(1, **i32), torch.zeros(n, **i32)
    da.decode_attn_step_tables(shape, lens, gains, after, table, free, count, left, starts, page_starts, slots, positions, seq, status)
    assert int(status) == da.DA_ERR_WORKSPACE_TOO_SMALL
    assert after[0] == 6 and (after[1:] == 5).all() and int(left) == pages
    assert starts[0] == 0 and (starts[1:] == 1).all() and (page_starts == 0).all()
    assert torch.equal(table, before) and torch.equal(free, torch.arange(pages, **i32))
    assert (int(slots[0]), int(positions[0]), int(seq[0])) == (pages * page + 5, 5, 0)
    assert (slots[1:] == -1).all() and (positions[1:] == -1).all() and (seq[1:] == -1).all()
