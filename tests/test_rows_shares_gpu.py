"""Rows whose heads are shared out unevenly among warps that go round more than once: 8 tasks in three shares of 2, 3 and 3, with
rows left out anywhere among them."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from packed_util import da  # noqa: E402
from test_rows_gpu import Rows, close, of_slots  # noqa: E402


def with_rows_left_out(n, seed, *args, **kw):
    """Rows of which a tenth is padding and some lie behind the table, and which ones are live."""
    r = Rows(n, *args, far=700, page=64, seed=seed, **kw)
    gen = torch.Generator().manual_seed(seed)
    dead, lost = torch.rand(n, generator=gen) < 0.1, torch.rand(n, generator=gen) < 0.02
    r.positions[lost] = 700 + 5
    r.positions[dead] = -1
    return r, ~dead & ~lost


@pytest.mark.parametrize("hq,hkv,d", [(16, 8, 128), (24, 4, 128), (24, 3, 128), (48, 8, 64)])
@pytest.mark.parametrize("n", [1185, 1200, 1500, 1578])
@pytest.mark.parametrize("interleaved", [False, True])
def test_uneven_shares(hq, hkv, d, n, interleaved):
    r, live = with_rows_left_out(n, n + hq, hq, hkv, d, interleaved=interleaved)
    q_out, (k_pool, v_pool), k_out = r.q_out(7.0), r.pools(7.0), torch.full((n, hkv, d), 7.0, dtype=r.dtype, device="cuda")
    r.call(q_out=q_out, k_out=k_out, k_cache=k_pool, v_cache=v_pool)
    r.positions[~live] = 0
    q, k, _ = r.expect()
    close(q_out[live.cuda()], q[live.numpy()], r.dtype, "q")
    close(k_out[live.cuda()], k[live.numpy()], r.dtype, "k")
    assert (q_out[~live.cuda()] == 7.0).all() and (k_out[~live.cuda()] == 7.0).all()
    assert torch.equal(of_slots(k_pool, r.slots[live]), k_out[live.cuda()])
    assert torch.equal(of_slots(v_pool, r.slots[live]).cpu(), list(r.split(r.qkv))[2][live])


@pytest.mark.parametrize("n", [1200, 1578])
def test_uneven_shares_of_queries_alone(n):
    r, live = with_rows_left_out(n, n, 32, 8, 128)
    q_out = r.q_out(7.0)
    r.call(k=None, v=None, k_weight=None, slots=None, q_out=q_out)
    r.positions[~live] = 0
    close(q_out[live.cuda()], r.expect()[0][live.numpy()], r.dtype)
    assert (q_out[~live.cuda()] == 7.0).all()


@pytest.mark.parametrize("hq,hkv,d,rotary", [(16, 8, 128, 128), (24, 4, 128, 64), (48, 8, 64, 64)])
@pytest.mark.parametrize("n", [1200, 1578])
@pytest.mark.parametrize("interleaved", [False, True])
def test_uneven_shares_to_4_bits(hq, hkv, d, rotary, n, interleaved):
    """The same bytes as from the call's 16-bit keys written by a call that turns nothing."""
    r, live = with_rows_left_out(n, n + d, hq, hkv, d, rotary=rotary, interleaved=interleaved)
    pool = lambda: torch.zeros((r.num_pages, hkv, da.decode_attn_packed_head_bytes(d, r.page)), dtype=torch.uint8, device="cuda")
    fused, apart, q_out = pool(), pool(), r.q_out()
    k_out = torch.zeros((n, hkv, d), dtype=r.dtype, device="cuda")
    r.call(4, q_out=q_out, k_out=k_out, k_cache=fused)
    slots = torch.where(live, r.slots, -1).cuda()
    r.call(4, q=None, q_weight=None, k=k_out, k_weight=None, positions=None, cos_sin=None, slots=slots, k_cache=apart)
    assert torch.equal(fused, apart)
    r.positions[~live] = 0
    q, k, _ = r.expect()
    close(q_out[live.cuda()], q[live.numpy()], r.dtype, "q")
    close(k_out[live.cuda()], k[live.numpy()], r.dtype, "k")
