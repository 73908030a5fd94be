"""Rows of new tokens (norms, rotation, cache write) against the fp64 oracle, and the cache in 4 bits that they are
written to and expanded from."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from oracle import packed_cache as ref  # noqa: E402
from packed_util import KINDS, da  # noqa: E402


def turn_table(far, rotary, base=10000.0):
    half = rotary // 2
    x = torch.arange(far).double()[:, None] * base ** (-torch.arange(half).double() / half)
    return torch.cat([x.cos(), x.sin()], 1).float()


class Rows:
    def __init__(self, n, hq, hkv, d, dtype="bf16", page=16, rotary=None, norm=True, per_head=False, interleaved=False, far=5000,
                 seed=0, size=1.0):
        gen = torch.Generator().manual_seed(seed)
        dt = KINDS[dtype][1]
        self.n, self.hq, self.hkv, self.d, self.dtype, self.page, self.interleaved = n, hq, hkv, d, dt, page, interleaved
        self.qkv = (torch.randn((n, (hq + 2 * hkv) * d), generator=gen) * size).to(dt)
        weight = lambda h: (1 + 0.2 * torch.randn((h, d) if per_head else (d,), generator=gen)).to(dt) if norm else None
        self.q_weight, self.k_weight = weight(hq), weight(hkv)
        rotary = d if rotary is None else rotary
        self.cos_sin = turn_table(far, rotary) if rotary else None
        self.positions = torch.randint(far, (n,), generator=gen).int()
        self.num_pages = -(-2 * n // page) + 1
        self.slots = torch.randperm(self.num_pages * page, generator=gen)[:n]
        self.kind = KINDS[dtype][0]

    def split(self, qkv):
        a, b = self.hq * self.d, self.hkv * self.d
        return (x.unflatten(1, (-1, self.d)) for x in qkv.split([a, b, b], 1))

    def shape(self):
        row = self.hkv * self.d
        return da.make_shape(0, self.hq, self.hkv, self.d, self.page, 0, self.num_pages, (self.page * row, row, self.d),
                             in_dtype=self.kind)

    def kv4_shape(self):
        return da.make_kv4_shape(0, self.hq, self.hkv, self.d, self.page, 0, self.num_pages, in_dtype=self.kind)

    def expect(self):
        q, k, v = (x.double().numpy() for x in self.split(self.qkv))
        turn = None if self.cos_sin is None else self.cos_sin.double().numpy()[self.positions.numpy()]
        w = lambda x: None if x is None else x.double().numpy()
        return (ref.rows(q, w(self.q_weight), 1e-6, turn, self.interleaved), ref.rows(k, w(self.k_weight), 1e-6, turn, self.interleaved), v)

    def call(self, cache_bits=16, shape=None, **kw):
        dev = lambda x: None if x is None else x.cuda()
        q, k, v = self.split(self.qkv.cuda())
        args = dict(slots=self.slots.cuda(), positions=dev(self.positions), cos_sin=dev(self.cos_sin), q_weight=dev(self.q_weight),
                    k_weight=dev(self.k_weight), interleaved=self.interleaved, cache_bits=cache_bits)
        args |= kw
        return da.decode_attn_prepare_rows(shape or (self.kv4_shape() if cache_bits == 4 else self.shape()), args.pop("q", q),
                                           args.pop("k", k), args.pop("v", v), **args)

    def pools(self, fill=0.0):
        return [torch.full((self.num_pages, self.page, self.hkv, self.d), fill, dtype=self.dtype, device="cuda") for _ in range(2)]

    def q_out(self, fill=0.0):
        return torch.full((self.n, self.hq, self.d), fill, dtype=self.dtype, device="cuda")


def close(got, want, dtype, what=""):
    """One rounding of the 16-bit type, and fp32 arithmetic of a sum of 128 squares (2^-17 relative by the worst order), a
    reciprocal root (2 steps) and two products of a rotation (relative to the pair, not to the difference)."""
    half = torch.finfo(dtype).eps / 2
    got = got.double().cpu().numpy()
    size = np.abs(want) + np.abs(want).max(-1, keepdims=True) * 2.0 ** -16
    tiny = torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps          # (a subnormal's step)
    assert (np.abs(got - want) <= half * size + np.abs(want).max(-1, keepdims=True) * 2.0 ** -16 + tiny).all(), what


def of_slots(pool, slots):
    return pool.flatten(0, 1)[slots.to(pool.device)]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rotary", ["all", "half", 8, 24, 0])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_rows(d, rotary, interleaved, norm, dtype):
    rotary = {"all": d, "half": d // 2}.get(rotary, rotary)
    r = Rows(37, 10, 2, d, dtype, rotary=rotary, interleaved=interleaved, norm=norm, seed=d + rotary)
    q_out, (k_pool, v_pool) = r.q_out(), r.pools()
    k_out = torch.zeros((37, 2, d), dtype=r.dtype, device="cuda")
    r.call(q_out=q_out, k_out=k_out, k_cache=k_pool, v_cache=v_pool)
    q, k, v = r.expect()
    close(q_out, q, r.dtype, "q")
    close(k_out, k, r.dtype, "k")
    assert torch.equal(of_slots(k_pool, r.slots), k_out)
    assert torch.equal(of_slots(v_pool, r.slots).cpu(), list(r.split(r.qkv))[2])
    untouched = torch.ones(r.num_pages * r.page, dtype=torch.bool)
    untouched[r.slots] = False
    assert (k_pool.flatten(0, 1)[untouched.cuda()] == 0).all() and (v_pool.flatten(0, 1)[untouched.cuda()] == 0).all()


@pytest.mark.parametrize("hq,hkv", [(1, 1), (8, 8), (32, 8), (48, 4), (3, 3), (16, 1)])
@pytest.mark.parametrize("n", [1, 2, 513])
def test_heads_and_rows(hq, hkv, n):
    r = Rows(n, hq, hkv, 128, per_head=True, page=64, seed=n + hq)
    q_out, (k_pool, v_pool) = r.q_out(), r.pools()
    r.call(q_out=q_out, k_cache=k_pool, v_cache=v_pool)
    q, k, _ = r.expect()
    close(q_out, q, r.dtype)
    close(of_slots(k_pool, r.slots), k, r.dtype)


@pytest.mark.parametrize("normed", ["q", "k"])
@pytest.mark.parametrize("rotary", [128, 0])
@pytest.mark.parametrize("n", [3, 1500])
def test_one_of_the_norms_alone(normed, rotary, n):
    r = Rows(n, 10, 2, 128, rotary=rotary, seed=n)
    if normed == "q":
        r.k_weight = None
    else:
        r.q_weight = None
    q_out, (k_pool, v_pool) = r.q_out(), r.pools()
    r.call(q_out=q_out, k_cache=k_pool, v_cache=v_pool)
    q, k, _ = r.expect()
    close(q_out, q, r.dtype, "q")
    close(of_slots(k_pool, r.slots), k, r.dtype, "k")


@pytest.mark.parametrize("size", [0.0, 1e-4, 300.0])
def test_magnitudes(size):
    r = Rows(5, 4, 2, 64, seed=1, size=size)
    q_out, (k_pool, v_pool) = r.q_out(), r.pools()
    r.call(q_out=q_out, k_cache=k_pool, v_cache=v_pool)
    q, k, _ = r.expect()
    close(q_out, q, r.dtype)
    close(of_slots(k_pool, r.slots), k, r.dtype)


def test_far_positions_turn_by_the_table():
    r = Rows(9, 4, 2, 128, far=131072, seed=3)
    r.positions[:3] = torch.tensor([0, 131071, 131070])
    q_out, (k_pool, v_pool) = r.q_out(), r.pools()
    r.call(q_out=q_out, k_cache=k_pool, v_cache=v_pool)
    close(q_out, r.expect()[0], r.dtype)


@pytest.mark.parametrize("cache_bits", [16, 4])
def test_padding_rows_and_rows_without_a_slot(cache_bits):
    r = Rows(12, 8, 2, 128, seed=4)
    keep, slots = r.positions.clone(), r.slots.clone()
    r.positions[[2, 11]] = -1                                                  # padding: nothing of them
    r.slots[5] = -1                                                            # no slot: q alone
    q_out = r.q_out(7.0)
    if cache_bits == 4:
        k_pool = torch.full((r.num_pages, 2, da.decode_attn_packed_head_bytes(128, 16)), 0xff, dtype=torch.uint8, device="cuda")
        r.call(4, q_out=q_out, k_cache=k_pool)
        before = (k_pool == 0xff).all()
        assert not before
    else:
        k_pool, v_pool = r.pools(7.0)
        r.call(q_out=q_out, k_cache=k_pool, v_cache=v_pool)
        for pool in (k_pool, v_pool):
            for b in (2, 5, 11):
                assert (of_slots(pool, slots)[b] == 7.0).all()
    live = [i for i in range(12) if i not in (2, 11)]
    r.positions, r.slots = keep, slots
    close(q_out[live], r.expect()[0][live], r.dtype)
    assert (q_out[[2, 11]] == 7.0).all()


def test_in_place_and_strided():
    r = Rows(50, 8, 2, 128, seed=5)
    qkv = r.qkv.cuda()
    q, k, v = r.split(qkv)
    k_pool, v_pool = r.pools()
    r.call(q=q, k=k, v=v, q_out=q, k_out=k, k_cache=k_pool, v_cache=v_pool)
    want_q, want_k, _ = r.expect()
    close(q, want_q, r.dtype)
    close(k, want_k, r.dtype)
    assert torch.equal(v.cpu(), list(r.split(r.qkv))[2]) and torch.equal(of_slots(v_pool, r.slots), v)
    assert torch.equal(of_slots(k_pool, r.slots), k)


def test_parts_alone():
    r = Rows(20, 8, 2, 64, seed=6)
    q_out, k_out = r.q_out(), torch.zeros((20, 2, 64), dtype=r.dtype, device="cuda")
    want_q, want_k, _ = r.expect()
    r.call(k=None, v=None, k_weight=None, slots=None, q_out=q_out)
    close(q_out, want_q, r.dtype)
    r.call(q=None, v=None, q_weight=None, slots=None, k_out=k_out)
    close(k_out, want_k, r.dtype)
    k_pool, v_pool = r.pools()
    _, k, v = r.split(r.qkv.cuda())
    r.call(q=None, q_weight=None, k_weight=None, positions=None, cos_sin=None, k_cache=k_pool, v_cache=v_pool)
    assert torch.equal(of_slots(k_pool, r.slots), k) and torch.equal(of_slots(v_pool, r.slots), v)


@pytest.mark.parametrize("layout", ["head-major", "padded"])
def test_pool_strides(layout):
    r = Rows(40, 4, 4, 64, page=32, seed=7)
    if layout == "head-major":
        strides = (4 * 32 * 64, 64, 32 * 64)
        size = r.num_pages * 4 * 32 * 64
    else:
        strides = (32 * 4 * 72 + 40, 4 * 72, 72)
        size = r.num_pages * strides[0]
    k_flat, v_flat = (torch.zeros(size, dtype=r.dtype, device="cuda") for _ in range(2))
    view = lambda x: x.as_strided((r.num_pages, 32, 4, 64), (strides[0], strides[1], strides[2], 1))
    shape = da.make_shape(0, 4, 4, 64, 32, 0, r.num_pages, strides)
    q_out = r.q_out()
    r.call(shape=shape, q_out=q_out, k_cache=k_flat, v_cache=v_flat)
    _, k, v = r.expect()
    close(of_slots(view(k_flat), r.slots), k, r.dtype)
    assert np.array_equal(of_slots(view(v_flat), r.slots).double().cpu().numpy(), v)


def test_slots_and_positions_outside_are_reported():
    r = Rows(6, 4, 2, 64, seed=8)
    r.slots[2] = r.num_pages * 16
    r.slots[3] = 1 << 40
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    q_out, (k_pool, v_pool) = r.q_out(), r.pools()
    r.call(q_out=q_out, k_cache=k_pool, v_cache=v_pool, status=status)
    assert int(status) == da.DA_ERR_BAD_PAGE
    q, k, _ = r.expect()
    close(q_out, q, r.dtype)
    close(of_slots(k_pool, r.slots[[0, 1, 4, 5]]), k[[0, 1, 4, 5]], r.dtype)
    r = Rows(6, 4, 2, 64, seed=8)
    q = r.expect()[0]
    r.positions[1] = 5000
    q_out, status = r.q_out(7.0), torch.zeros(1, dtype=torch.int32, device="cuda")
    r.call(q_out=q_out, k_cache=k_pool, v_cache=v_pool, status=status)
    assert int(status) == da.DA_ERR_STALE_PLAN and (q_out[1] == 7.0).all()
    close(q_out[[0, 2, 3, 4, 5]], q[[0, 2, 3, 4, 5]], r.dtype)


# ------------------------------------------------------------------------------------------------ in 4 bits

def stored(r, pool):
    """K and V values that a packed pool holds at the rows' slots."""
    k, v = ref.pool_values(pool.cpu().numpy(), r.d, r.page)
    s = r.slots.numpy()
    return k[s // r.page, s % r.page], v[s // r.page, s % r.page]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_quantised_rows_are_the_nearest(d, page, dtype):
    r = Rows(83, 4, 2, d, dtype, page=page, norm=False, rotary=0, seed=9)
    pool = torch.zeros((r.num_pages, 2, da.decode_attn_packed_head_bytes(d, page)), dtype=torch.uint8, device="cuda")
    r.call(4, q=None, positions=None, k_cache=pool)
    _, k, v = r.split(r.qkv)
    got_k, got_v = stored(r, pool)
    for got, x in ((got_k, k), (got_v, v)):
        code, scale = ref.encode(x.double().numpy())
        assert np.array_equal(got, ref.values(code, scale))


@pytest.mark.parametrize("rotary,interleaved", [(128, False), (128, True), (64, False), (24, False), (8, True), (0, False)])
def test_quantised_on_the_way_as_by_a_second_call(rotary, interleaved):
    """The same bytes from the fused call as from its 16-bit K quantised by a call of its own."""
    r = Rows(61, 6, 2, 128, rotary=rotary, interleaved=interleaved, seed=10 + rotary)
    pool = lambda: torch.zeros((r.num_pages, 2, da.decode_attn_packed_head_bytes(128, 16)), dtype=torch.uint8, device="cuda")
    fused, apart, q_out = pool(), pool(), r.q_out()
    k_out = torch.zeros((61, 2, 128), dtype=r.dtype, device="cuda")
    r.call(4, q_out=q_out, k_out=k_out, k_cache=fused)
    r.call(4, q=None, q_weight=None, k=k_out, k_weight=None, positions=None, cos_sin=None, k_cache=apart)
    assert torch.equal(fused, apart)
    close(k_out, r.expect()[1], r.dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_quotients_at_and_beside_the_ties(dtype):
    """Scales of many mantissas and exponents; values at the ties between codes and one step of the type to either side."""
    dt = KINDS[dtype][1]
    bits = 11 if dtype == "fp16" else 8
    mantissas = torch.arange(2 ** (bits - 4), 2 ** (bits - 3)).double() / 2 ** (bits - 4)     # 3 * m and 7 * m are values of the type
    scales = torch.cat([mantissas * 2.0 ** e for e in (-9, -1, 0, 5)])
    ties = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]).double()
    at = (scales[:, None] * ties).to(dt)
    assert torch.equal(at.double(), scales[:, None] * ties) and torch.equal((6 * scales).to(dt).double(), 6 * scales)
    near = [torch.nextafter(at, torch.full_like(at, to)) for to in (float("inf"), 0.0)]
    x = torch.zeros((len(scales), 64), dtype=dt)
    for i, part in enumerate([at, *near]):
        x[:, 8 * i:8 * i + 7] = part
        x[:, 32 + 8 * i:32 + 8 * i + 7] = -part
    x[:, 7], x[:, 39] = (6 * scales).to(dt), (-6 * scales).to(dt)
    r = Rows(len(scales), 1, 1, 64, dtype, norm=False, rotary=0, seed=2)
    pool = torch.zeros((r.num_pages, 1, da.decode_attn_packed_head_bytes(64, 16)), dtype=torch.uint8, device="cuda")
    r.call(4, q=None, k=x[:, None].cuda(), v=x[:, None].cuda(), positions=None, k_cache=pool)
    code, scale = ref.encode(x.double().numpy())
    assert np.array_equal(scale.astype(np.float64), np.repeat(scales[:, None].numpy(), 2, 1).reshape(scale.shape))
    want = ref.values(code, scale)
    for got in stored(r, pool):
        assert np.array_equal(got[:, 0], want)


@pytest.mark.parametrize("rotary", [64, 32])
def test_quantised_on_the_way_small_heads(rotary):
    r = Rows(45, 6, 3, 64, "fp16", rotary=rotary, page=32, seed=rotary)
    pool = lambda: torch.zeros((r.num_pages, 3, da.decode_attn_packed_head_bytes(64, 32)), dtype=torch.uint8, device="cuda")
    fused, apart, q_out = pool(), pool(), r.q_out()
    k_out = torch.zeros((45, 3, 64), dtype=r.dtype, device="cuda")
    r.call(4, q_out=q_out, k_out=k_out, k_cache=fused)
    r.call(4, q=None, q_weight=None, k=k_out, k_weight=None, positions=None, cos_sin=None, k_cache=apart)
    assert torch.equal(fused, apart)
    close(k_out, r.expect()[1], r.dtype)


def test_values_at_the_borders():
    """Ties between codes, zeros, tiny and huge blocks, infinities."""
    r = Rows(6, 1, 1, 64, "fp16", norm=False, rotary=0, seed=1)
    ties = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0])
    x = torch.zeros((6, 64), dtype=torch.float16)
    x[0, :8], x[0, 8:16], x[0, 32] = ties, -ties, 6.0
    x[1, :8] = ties * 2.0 ** -14
    x[2, :4] = torch.tensor([65504.0, -65504.0, 30000.0, 1.0])
    x[3, :2] = torch.tensor([6e-8, -6e-8])                                     # below 6 * 2^-25: zeros
    x[4, 0], x[4, 1] = float("inf"), 3.0
    k = x[:, None]
    pool = torch.zeros((r.num_pages, 1, da.decode_attn_packed_head_bytes(64, 16)), dtype=torch.uint8, device="cuda")
    r.call(4, q=None, k=k.cuda(), v=k.cuda(), positions=None, k_cache=pool)
    got_k, got_v = stored(r, pool)
    assert np.array_equal(got_k, got_v)
    code, scale = ref.encode(x[:4].double().numpy())
    assert np.array_equal(got_k[:4, 0], ref.values(code, scale))
    assert (got_k[3, 0, :32] == 0).all()
    assert got_k[4, 0, 0] == 6 * 65504.0 and got_k[4, 0, 1] == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("d,page", [(64, 16), (64, 128), (128, 16), (128, 32)])
def test_expanded_pages(d, page, dtype):
    from packed_util import Cache
    c = Cache([1, 0, 16, 17, 333, page, page + 1], 4, 2, d, page=page, dtype=dtype, seed=d)
    rng = np.random.default_rng(1)
    wide = c.width + 3
    dst = np.full((len(c.lens), wide), -1, dtype=np.int32)
    live = c.table >= 0
    n = int(live.sum())
    dst[:, :c.width][live] = rng.permutation(n + 5)[:n]
    dt = KINDS[dtype][1]
    k, v = (torch.full((n + 5, page, 2, d), 7.0, dtype=dt, device="cuda") for _ in range(2))
    row = 2 * d
    shape = da.make_shape(len(c.lens), 4, 2, d, page, wide, n + 5, (page * row, row, d), in_dtype=KINDS[dtype][0])
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    da.decode_attn_expand_kv(shape, c.shape(), torch.from_numpy(c.pool).cuda(), torch.from_numpy(c.table).cuda(),
                             torch.tensor(c.lens, dtype=torch.int32).cuda(), torch.from_numpy(dst).cuda(), k, v, status)
    assert int(status) == da.DA_OK
    want_k, want_v = torch.full(k.shape, 7.0, dtype=dt), torch.full(k.shape, 7.0, dtype=dt)
    for b, length in enumerate(c.lens):
        at = np.arange(length)
        src, to = c.table[b][at // page], dst[b][at // page]
        want_k[to, at % page] = torch.from_numpy(c.k[src, at % page]).to(dt)
        want_v[to, at % page] = torch.from_numpy(c.v[src, at % page]).to(dt)
    assert torch.equal(k.cpu(), want_k) and torch.equal(v.cpu(), want_v)


@pytest.mark.parametrize("n,hkv,d,page", [(700, 3, 64, 16), (257, 1, 128, 16), (256, 8, 128, 64)])
def test_expanding_many_sequences(n, hkv, d, page):
    """More sequences than one block sums up at a time, some of them empty, read from a few pages that they share."""
    gen = torch.Generator().manual_seed(n)
    lens = torch.randint(3 * page + 1, (n,), generator=gen).int()
    lens[torch.randint(n, (n // 5,), generator=gen)] = 0
    expand_shared(lens, hkv, d, page, 3, gen)


def test_expanding_more_tiles_than_a_round_of_all_warps():
    gen = torch.Generator().manual_seed(0)
    expand_shared(torch.tensor([7400 * 256 - 3, 1, 7377 * 256] + [7400 * 256 - 129] * 6).int(), 1, 64, 256, 7400, gen)


def expand_shared(lens, hkv, d, page, width, gen):
    """Sequences whose source pages are drawn from eight; expected: those eight, expanded one sequence each."""
    n, few = len(lens), 8
    head = da.decode_attn_packed_head_bytes(d, page)
    pool = torch.randint(256, (few, hkv, head), generator=gen, dtype=torch.uint8)
    tiles = pool.view(few, hkv, page // 16, -1)
    scales = (0.5 + torch.rand(tiles[..., 16 * d:].shape[:-1] + (d // 16 * 16,), generator=gen)).half()
    tiles[..., 16 * d:] = scales.contiguous().view(torch.uint8)
    pool = pool.cuda()
    table = torch.randint(few, (n, width), generator=gen).int().cuda()
    held = (lens + page - 1) // page
    live = (torch.arange(width)[None] < held[:, None]).cuda()
    total = int(held.sum())
    dst = torch.full((n, width), -1, dtype=torch.int32, device="cuda")
    dst[live] = torch.randperm(total, generator=gen).int().cuda()
    row = hkv * d
    pages = lambda m: [torch.full((m, page, hkv, d), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    shapes = lambda b, w, m: (da.make_shape(b, hkv, hkv, d, page, w, m, (page * row, row, d)), da.make_kv4_shape(b, hkv, hkv, d, page, w, few))
    one = torch.arange(few, dtype=torch.int32, device="cuda")[:, None].contiguous()
    few_kv, kv = pages(few), pages(total)
    da.decode_attn_expand_kv(*shapes(few, 1, few), pool, one, torch.full((few,), page, dtype=torch.int32, device="cuda"), one, *few_kv)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    da.decode_attn_expand_kv(*shapes(n, width, total), pool, table, lens.cuda(), dst, *kv, status)
    assert int(status) == da.DA_OK
    src = torch.empty(total, dtype=torch.long, device="cuda")
    src[dst[live].long()] = table[live].long()
    rows = torch.empty(total, dtype=torch.long, device="cuda")                 # of every destination page
    rows[dst[live].long()] = (lens.cuda()[:, None] - torch.arange(width, device="cuda") * page).clamp(max=page)[live].long()
    for got, of in zip(kv, few_kv):
        for at in range(0, total, 4096):
            want = of[src[at:at + 4096]]
            want[torch.arange(page, device="cuda")[None] >= rows[at:at + 4096, None]] = 7.0
            assert torch.equal(got[at:at + 4096], want)


def test_expanding_reports_what_does_not_fit():
    from packed_util import Cache
    c = Cache([40, 40, 40], 2, 1, 64, seed=3)
    c.table[0, 1] = 99
    dst = torch.arange(9, dtype=torch.int32).view(3, 3)
    dst[1, 2] = 9
    k, v = (torch.full((9, 16, 1, 64), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    shape = da.make_shape(3, 2, 1, 64, 16, 3, 9, (16 * 64, 64, 64))
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    lens = torch.tensor(c.lens, dtype=torch.int32).cuda()
    call = lambda: da.decode_attn_expand_kv(shape, c.shape(), torch.from_numpy(c.pool).cuda(), torch.from_numpy(c.table).cuda(), lens,
                                            dst.cuda(), k, v, status)
    call()
    assert int(status) == da.DA_ERR_BAD_PAGE
    assert (k[1] == 7).all() and (k[5] == 7).all() and not (k[0] == 7).all() and not (k[8, :8] == 7).all() and (k[8, 8:] == 7).all()
    status.zero_()
    c.table[0, 1], dst[1, 2] = c.table[0, 0], 5
    lens[2] = 49                                                               # more than the three pages of its tables
    lens[1] = -1
    k.fill_(7.0)
    call()
    assert int(status) == da.DA_ERR_STALE_PLAN
    assert (k[3:] == 7).all() and not (k[0] == 7).all()


# ------------------------------------------------------------------------------------------------ many rows

@pytest.mark.parametrize("hq,hkv,d,parts", [(4, 1, 128, "q"), (1, 1, 64, "qkv"), (9, 1, 128, "qkv"), (32, 8, 128, "qkv"), (2, 2, 64, "kv")])
@pytest.mark.parametrize("n", [2367, 2369, 9001])
def test_more_rows_than_warps(hq, hkv, d, parts, n):
    """Warps go from row to row: few and many tasks a row, rows of padding and bad positions among them."""
    r = Rows(n, hq, hkv, d, far=700, page=64, seed=n + hq)
    gen = torch.Generator().manual_seed(n)
    dead = torch.rand(n, generator=gen) < 0.1
    r.positions[dead] = -1
    lost = torch.rand(n, generator=gen) < 0.02
    r.positions[lost & ~dead] = 700 + 5
    q_out, (k_pool, v_pool), k_out = r.q_out(7.0), r.pools(7.0), torch.full((n, hkv, d), 7.0, dtype=r.dtype, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    args = dict(status=status)
    args |= dict(q_out=q_out) if "q" in parts else dict(q=None, q_weight=None)
    args |= dict(k_out=k_out, k_cache=k_pool, v_cache=v_pool) if "kv" in parts else dict(k=None, v=None, k_weight=None, slots=None)
    r.call(**args)
    assert int(status) == da.DA_ERR_STALE_PLAN
    live = ~dead & ~lost
    r.positions[~live] = 0
    q, k, v = r.expect()
    keep = live.numpy()
    if "q" in parts:
        close(q_out[live.cuda()], q[keep], r.dtype, "q")
        assert (q_out[~live.cuda()] == 7.0).all()
    if "kv" in parts:
        close(k_out[live.cuda()], k[keep], r.dtype, "k")
        assert torch.equal(of_slots(k_pool, r.slots[live]), k_out[live.cuda()])
        assert torch.equal(of_slots(v_pool, r.slots[live]).cpu(), list(r.split(r.qkv))[2][live])
        assert (of_slots(v_pool, r.slots[~live]) == 7.0).all()


def test_fewer_rows_than_the_tensors_hold():
    r = Rows(40, 8, 2, 128, seed=12)
    q_out, (k_pool, v_pool) = r.q_out(7.0), r.pools(7.0)
    r.call(q_out=q_out, k_cache=k_pool, v_cache=v_pool, rows=17)
    close(q_out[:17], r.expect()[0][:17], r.dtype)
    assert (q_out[17:] == 7.0).all() and (of_slots(v_pool, r.slots[17:]) == 7.0).all()


@pytest.mark.parametrize("cache_bits", [16, 4])
def test_pools_beyond_32_bits(cache_bits):
    """Slots whose bytes lie past 2^32 (and whose elements lie past 2^31)."""
    r = Rows(30, 4, 2, 128, page=16, seed=13)
    head = da.decode_attn_packed_head_bytes(128, 16)
    r.num_pages = (5 << 30) // (2 * head) if cache_bits == 4 else (5 << 30) // (16 * 2 * 128 * 2)
    r.slots = torch.arange(30) * 7 + (r.num_pages - 20) * 16
    q_out = r.q_out()
    k_out = torch.zeros((30, 2, 128), dtype=r.dtype, device="cuda")
    if cache_bits == 4:
        pool = torch.empty((r.num_pages, 2, head), dtype=torch.uint8, device="cuda")
        pool[-20:] = 0
        r.call(4, q_out=q_out, k_out=k_out, k_cache=pool)
        r.slots -= (r.num_pages - 20) * 16
        got_k, got_v = stored(r, pool[-20:])
        code, scale = ref.encode(k_out.double().cpu().numpy())
        assert np.array_equal(got_k, ref.values(code, scale))
        # the same pages expanded, through a table that names them
        table = torch.arange(r.num_pages - 20, r.num_pages, dtype=torch.int32, device="cuda")[None]
        k, v = (torch.zeros((20, 16, 2, 128), dtype=r.dtype, device="cuda") for _ in range(2))
        shape = da.make_shape(1, 4, 2, 128, 16, 20, 20, (16 * 256, 256, 128))
        packed = da.make_kv4_shape(1, 4, 2, 128, 16, 20, r.num_pages)
        da.decode_attn_expand_kv(shape, packed, pool, table, torch.tensor([320], dtype=torch.int32).cuda(),
                                 torch.arange(20, dtype=torch.int32, device="cuda")[None].contiguous(), k, v)
        assert torch.equal(of_slots(k, r.slots).cpu(), torch.from_numpy(got_k).to(r.dtype))
        assert torch.equal(of_slots(v, r.slots).cpu(), torch.from_numpy(got_v).to(r.dtype))
    else:
        k_pool, v_pool = (torch.empty((r.num_pages, 16, 2, 128), dtype=r.dtype, device="cuda") for _ in range(2))
        r.call(q_out=q_out, k_out=k_out, k_cache=k_pool, v_cache=v_pool)
        assert torch.equal(of_slots(k_pool, r.slots), k_out)
        assert torch.equal(of_slots(v_pool, r.slots).cpu(), list(r.split(r.qkv))[2])
    close(k_out, r.expect()[1], r.dtype)
