"""Step tables, rows of new tokens, the cache in 4 bits and its attention used together, as a serving step uses them: on
streams of their own, captured and replayed, with prompts through expanded pages, sharing a workspace."""
import random

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from oracle import packed_cache as ref  # noqa: E402
from packed_util import Cache, bounds, check, da, run  # noqa: E402
from test_rows_gpu import close, turn_table  # noqa: E402

HQ, HKV, D, PAGE, WIDE, PAGES, ROWS = 8, 2, 128, 16, 40, 300, 512


class Engine:
    """What a serving loop holds on the device; every step is tables, rows (norm, rotation, write), then attention."""

    def __init__(self, batch, seed=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        i32 = dict(dtype=torch.int32, device="cuda")
        self.batch, self.gen = batch, gen
        self.lens = torch.zeros(batch, **i32)
        self.gains = torch.zeros(batch, **i32)
        self.table = torch.full((batch, WIDE), -1, **i32)
        self.free = torch.randperm(PAGES, device="cuda", generator=gen).int()
        self.count = torch.tensor([PAGES], **i32)
        self.starts, self.page_starts = torch.zeros(batch + 1, **i32), torch.zeros(batch + 1, **i32)
        self.slots = torch.zeros(ROWS, dtype=torch.int64, device="cuda")
        self.positions, self.row_seq, self.status = torch.zeros(ROWS, **i32), torch.zeros(ROWS, **i32), torch.zeros(1, **i32)
        self.pool = torch.full((PAGES, HKV, da.decode_attn_packed_head_bytes(D, PAGE)), 0xff, dtype=torch.uint8, device="cuda")
        self.qkv = torch.zeros((ROWS, (HQ + 2 * HKV) * D), dtype=torch.bfloat16, device="cuda")
        self.q, self.k, self.v = (x.unflatten(1, (-1, D)) for x in self.qkv.split([HQ * D, HKV * D, HKV * D], 1))
        self.q_out = torch.zeros((ROWS, HQ, D), dtype=torch.bfloat16, device="cuda")
        self.k_out = torch.zeros((ROWS, HKV, D), dtype=torch.bfloat16, device="cuda")
        self.weights = [(1 + 0.1 * torch.randn(D, device="cuda", generator=gen)).bfloat16() for _ in range(2)]
        self.cos_sin = turn_table(WIDE * PAGE, D).cuda()
        self.shape = da.make_kv4_shape(batch, HQ, HKV, D, PAGE, WIDE, PAGES)

    def write(self):
        da.decode_attn_step_tables(self.shape, self.lens, self.gains, self.lens, self.table, self.free, self.count, self.count, self.starts,
                                   self.page_starts, self.slots, self.positions, self.row_seq, self.status)
        da.decode_attn_prepare_rows(self.shape, self.q, self.k, self.v, self.slots, self.positions, self.cos_sin, q_out=self.q_out,
                                    k_out=self.k_out, k_cache=self.pool, q_weight=self.weights[0], k_weight=self.weights[1], cache_bits=4,
                                    status=self.status)

    def fresh(self, gains):
        self.gains.copy_(torch.tensor(gains, dtype=torch.int32))
        self.qkv.copy_(torch.randn(self.qkv.shape, device="cuda", generator=self.gen).bfloat16())

    def cache(self, lens, q):
        """The oracle's view of what the pool holds now."""
        c = Cache.__new__(Cache)
        c.lens, c.hq, c.hkv, c.d, c.page, c.dtype = lens, HQ, HKV, D, PAGE, "bf16"
        c.table, c.pool, c.q = self.table.cpu().numpy(), self.pool.cpu().numpy(), q.cpu()
        used = np.unique(c.table[c.table >= 0])
        k, v = np.zeros((PAGES, PAGE, HKV, D)), np.zeros((PAGES, PAGE, HKV, D))
        k[used], v[used] = ref.pool_values(c.pool[used], D, PAGE)
        c.k, c.v = np.nan_to_num(k), np.nan_to_num(v)
        return c

    def check_rows(self, n):
        """Queries and keys of the last step's n rows, and what the pool holds of its keys and values."""
        turn = self.cos_sin.double().cpu().numpy()[self.positions[:n].cpu().numpy()]
        w = [x.double().cpu().numpy() for x in self.weights]
        close(self.q_out[:n], ref.rows(self.q[:n].double().cpu().numpy(), w[0], 1e-6, turn, False), torch.bfloat16)
        close(self.k_out[:n], ref.rows(self.k[:n].double().cpu().numpy(), w[1], 1e-6, turn, False), torch.bfloat16)
        k, v = ref.pool_values(self.pool.cpu().numpy(), D, PAGE)
        s = self.slots[:n].cpu().numpy()
        for got, x in ((k, self.k_out[:n]), (v, self.v[:n])):
            assert np.array_equal(got[s // PAGE, s % PAGE], ref.values(*ref.encode(x.double().cpu().numpy())))


def last_rows(e, batch):
    """Rows of the step's last token of every sequence (all have one)."""
    return (e.starts[1:batch + 1] - 1).long()


def test_a_serving_loop():
    e, batch = Engine(5, seed=1), 5
    rng = random.Random(2)
    lens = [0] * batch
    for step in range(12):
        if step == 0:
            gains = [40, 1, 17, 100, 16]
        elif step == 6:
            gains = [-lens[0], 1, -3, 60, 1]                                   # one ends, one loses rejected tokens, one takes a chunk
        else:
            gains = [rng.randint(1, 5) for _ in range(batch)]
        e.fresh(gains)
        e.write()
        lens = [max(0, n + g) for n, g in zip(lens, gains)]
        assert e.lens.tolist() == lens and int(e.status) == da.DA_OK
        n = sum(max(0, g) for g in gains)
        assert (e.positions[n:] == -1).all()
        e.check_rows(n)
        if step == 6:
            continue
        q = e.q_out[last_rows(e, batch)]
        out, lse, status = run_on(e, lens, q)
        assert status == da.DA_OK
        check(e.cache(lens, q), out, lse, f"step {step}")
    # all pages are in a table or in the list, once
    held = [int(p) for row, n in zip(e.table.tolist(), lens) for p in row[:-(-n // PAGE)]]
    assert sorted(held + e.free[:int(e.count)].tolist()) == list(range(PAGES))


def run_on(e, lens, q, plan=None, ws=None, policy=None):
    shape = e.shape
    shape.batch = len(lens)
    own = plan is None
    if own:
        plan = da.decode_attn_plan(shape, policy or da.make_policy(cache_bits=4), lens)
    ws = ws if ws is not None else torch.empty(max(plan.workspace_bytes, 256), dtype=torch.uint8, device="cuda")
    out = torch.full((len(lens), HQ, D), float("nan"), device="cuda")
    lse = torch.full((len(lens), HQ), float("nan"), device="cuda")
    da.decode_attn_run(plan, q.contiguous(), e.pool, None, e.table, e.lens, out, lse, ws)
    da.decode_attn_combine(plan, ws, out, lse)
    status = da.decode_attn_last_device_status(plan)
    if own:
        plan.destroy()
    return out, lse, status


def test_two_loops_on_two_streams():
    """Each on a stream of its own, nothing waited for in between; the workspaces are their own."""
    streams = [torch.cuda.Stream() for _ in range(2)]
    engines, outs, lens = [], [], [[30, 200, 7], [90, 16, 41]]
    for i, st in enumerate(streams):
        st.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(st):
            e = Engine(3, seed=10 + i)
            e.fresh(lens[i])
            engines.append(e)
    torch.cuda.synchronize()
    plans = [da.decode_attn_plan(e.shape, da.make_policy(cache_bits=4, chunk_tokens=32), n) for e, n in zip(engines, lens)]
    ws = [torch.empty(max(p.workspace_bytes, 256), dtype=torch.uint8, device="cuda") for p in plans]
    for i, st in enumerate(streams):
        outs.append((torch.zeros((3, HQ, D), device="cuda"), torch.zeros((3, HQ), device="cuda"),
                     torch.zeros((3, HQ, D), dtype=torch.bfloat16, device="cuda")))
    torch.cuda.synchronize()
    for _ in range(3):
        for e, p, w, (out, lse, q), st in zip(engines, plans, ws, outs, streams):
            with torch.cuda.stream(st):
                e.lens.zero_()
                e.count.fill_(PAGES)
                e.write()
                q.copy_(e.q_out[last_rows(e, 3)])
                da.decode_attn_run(p, q, e.pool, None, e.table, e.lens, out, lse, w)
                da.decode_attn_combine(p, w, out, lse)
    torch.cuda.synchronize()
    for e, p, n, (out, lse, q) in zip(engines, plans, lens, outs):
        assert da.decode_attn_last_device_status(p) == da.DA_OK and int(e.status) == da.DA_OK
        e.check_rows(sum(n))
        check(e.cache(n, q), out, lse, "a stream")
        p.destroy()


def test_captured_steps_that_share_a_workspace():
    """Two captured steps of two plans on one stream, replayed in turn with new rows; gains, lengths and tables change on the
    device alone."""
    e, batch = Engine(4, seed=3), 4
    lens = [50, 3, 120, 31]
    e.fresh(lens)
    e.write()
    torch.cuda.synchronize()
    policies = [da.make_policy(cache_bits=4, capacity_batch=4, capacity_tokens=2000), da.make_policy(cache_bits=4, capacity_batch=4,
                capacity_tokens=2000, split_mode=da.DA_SPLIT_DETERMINISTIC, chunk_tokens=32)]
    plans = [da.decode_attn_plan(e.shape, pol, lens) for pol in policies]
    ws = torch.empty(max(p.workspace_bytes for p in plans), dtype=torch.uint8, device="cuda")
    out, lse = torch.zeros((batch, HQ, D), device="cuda"), torch.zeros((batch, HQ), device="cuda")
    q = torch.zeros((batch, HQ, D), dtype=torch.bfloat16, device="cuda")

    def step(plan):
        e.write()
        q.copy_(e.q_out[:batch])                                               # one new token each: rows are the sequences
        da.decode_attn_run(plan, q, e.pool, None, e.table, e.lens, out, lse, ws)
        da.decode_attn_combine(plan, ws, out, lse)

    stream, graphs = torch.cuda.Stream(), []
    e.gains.zero_()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        for plan in plans:
            step(plan)                                                         # (a step that gains nothing)
    stream.synchronize()
    for plan in plans:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=stream):
            step(plan)
    for i in range(6):
        e.fresh([1] * batch)
        lens = [n + 1 for n in lens]
        da.decode_attn_plan_update(plans[i % 2], lens)
        graphs[i % 2].replay()
        assert da.decode_attn_last_device_status(plans[i % 2]) == da.DA_OK and int(e.status) == da.DA_OK
        assert e.lens.tolist() == lens
        e.check_rows(batch)
        check(e.cache(lens, q), out, lse, f"replay {i}")
    graphs.clear()
    for plan in plans:
        plan.destroy()


def test_a_prompt_over_a_cache_in_4_bits():
    """A chunk of 37 new tokens behind 100: written in 4 bits, expanded, attended by the prompt kernel; then a decode step."""
    e = Engine(2, seed=5)
    before, new = [100, 5], [37, 64]
    e.fresh(before)
    e.write()
    e.fresh(new)
    e.write()
    lens = [a + b for a, b in zip(before, new)]
    n = sum(new)
    e.check_rows(n)
    row = HKV * D
    shape = da.make_shape(2, HQ, HKV, D, PAGE, WIDE, 2 * WIDE, (PAGE * row, row, D))
    k, v = (torch.full((2 * WIDE, PAGE, HKV, D), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    dst = torch.arange(2 * WIDE, dtype=torch.int32, device="cuda").view(2, WIDE).flip(1).contiguous()
    da.decode_attn_expand_kv(shape, e.shape, e.pool, e.table, e.lens, dst, k, v, e.status)
    plan = da.decode_attn_prompt_plan(shape, da.make_policy(), new, lens)
    out, lse = torch.zeros((n, HQ, D), device="cuda"), torch.zeros((n, HQ), device="cuda")
    ws = torch.empty(max(plan.workspace_bytes, 256), dtype=torch.uint8, device="cuda")
    da.decode_attn_prompt_run(plan, e.q_out[:n].contiguous(), k, v, dst, e.lens, out, lse, ws)
    assert da.decode_attn_prompt_last_device_status(plan) == da.DA_OK and int(e.status) == da.DA_OK
    plan.destroy()
    # every new token is a row of a batch whose sequence ends with it
    c = e.cache(lens, e.q_out[:n])
    seq = [b for b in range(2) for _ in range(new[b])]
    c.table, c.lens = c.table[seq], [before[b] + i + 1 for b in range(2) for i in range(new[b])]
    want, want_lse, mass, size = c.expect()
    err, lse_err = bounds(mass, size, want_lse, max(lens), np.abs(c.v).max())
    # (the prompt kernel multiplies values rounded to bf16, keys too: half a step of 2^-8 of every product of a logit)
    err = err + mass * (2.0 ** -8 * 2 + 2 * size[..., None] * 2.0 ** -8)
    assert (np.abs(out.double().cpu().numpy() - want) <= err).all()
    assert (np.abs(lse.double().cpu().numpy() - want_lse) <= lse_err + size * 2.0 ** -8).all()
    # the same last rows by a decode step over the 4 bits
    last = last_rows(e, 2)
    out4, lse4, status = run_on(e, lens, e.q_out[last])
    assert status == da.DA_OK
    check(e.cache(lens, e.q_out[last]), out4, lse4, "the last token")


@pytest.mark.parametrize("seed", range(24))
def test_random_cases(seed):
    rng = random.Random(seed)
    hkv = rng.choice([1, 2, 3, 8])
    group, d, page = rng.randint(1, 16), rng.choice([64, 128]), rng.choice([16, 32, 64, 128, 256])
    lens = [rng.choice([0, 1, rng.randint(1, 60), rng.randint(1, 3000)]) for _ in range(rng.randint(1, 9))]
    c = Cache(lens, hkv * group, hkv, d, page=page, dtype=rng.choice(["bf16", "fp16"]), seed=seed)
    window = rng.choice([0, 0, rng.randint(1, 500)])
    sinks = rng.choice([0, 4, 33]) if window else 0
    mode = rng.choice([da.DA_SPLIT_AUTO, da.DA_SPLIT_AUTO, da.DA_SPLIT_DETERMINISTIC, da.DA_SPLIT_FIXED_COUNT])
    pol = da.make_policy(cache_bits=4, split_mode=mode, fixed_count=rng.randint(1, 9), window_tokens=window, sink_tokens=sinks,
                         chunk_tokens=rng.choice([0, 16, 64, 256]), sm_count=rng.choice([0, 0, 3, 20]), fuse_combine=rng.choice([0, 0, 1]))
    mask = [rng.random() < 0.8 for _ in lens] if rng.random() < 0.4 else None
    out = rng.choice(["fp32", "bf16", "fp16"])
    o, lse, status = run(c, pol, out=out, run_mask=None if mask is None else torch.tensor(mask, dtype=torch.uint8, device="cuda"))
    assert status == da.DA_OK
    dead = () if mask is None else tuple(b for b, m in enumerate(mask) if not m)
    check(c, o, lse, f"seed {seed}", dtype=out, window=window, sinks=sinks, dead=dead)


def test_a_pool_beyond_32_bits():
    head = da.decode_attn_packed_head_bytes(128, 16)
    c = Cache([300, 90], 8, 2, 128, seed=7)
    far = (5 << 30) // (2 * head)
    pool = torch.empty((far + c.num_pages, 2, head), dtype=torch.uint8, device="cuda")
    pool[far:] = torch.from_numpy(c.pool).cuda()
    near = c.table
    c.table = np.where(near >= 0, near + far, near).astype(np.int32)
    pages, c.num_pages = c.num_pages, far + c.num_pages
    out, lse, status = run(c, pool=pool)
    assert status == da.DA_OK
    c.table, c.num_pages = near, pages
    check(c, out, lse, "far pages")
