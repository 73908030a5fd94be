"""Step tables against the plain loops of the oracle: every output, every refusal, in place and in a graph."""
import random

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from oracle import packed_cache as ref  # noqa: E402
from packed_util import da  # noqa: E402


class Step:
    def __init__(self, lens, gains, page=16, width=None, spare=5, max_rows=None, capacity=None, num_pages=None, seed=0, free=None):
        rng = random.Random(seed)
        self.lens, self.gains, self.page = list(lens), list(gains), page
        pages = lambda n: -(-max(0, n) // page)
        after = [max(0, a + b) for a, b in zip(lens, gains)]
        self.width = width if width is not None else max([pages(n) for n in self.lens + after] + [1])
        held = [min(pages(n), self.width) for n in self.lens]
        lack = sum(max(0, pages(m) - pages(n)) for m, n in zip(after, lens))
        back = sum(max(0, pages(n) - pages(m)) for m, n in zip(after, lens))
        self.count = lack + spare if free is None else free
        self.num_pages = num_pages or sum(held) + self.count + 3
        ids = list(range(sum(held) + self.count + 3))
        rng.shuffle(ids)
        self.table, at = [], 0
        for h in held:
            self.table.append(ids[at:at + h] + [-1] * (self.width - h))
            at += h
        self.capacity = self.count + back if capacity is None else capacity
        self.free = ids[at:at + self.count] + [-1] * (self.capacity - self.count)
        self.free = self.free[:self.capacity]
        self.max_rows = sum(max(0, g) for g in gains) if max_rows is None else max_rows

    def expect(self):
        return ref.step_tables(self.lens, self.gains, self.table, self.free, self.count, self.capacity, self.page, self.num_pages,
                               self.max_rows)

    def put(self):
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
        n = len(self.lens)
        self.shape = da.make_shape(n, 8, 2, 64, self.page, self.width, self.num_pages, (self.page * 128, 128, 64))
        self.t = dict(seq_lens=i32(self.lens), gains=i32(self.gains), seq_lens_out=torch.full((n,), 77, dtype=torch.int32, device="cuda"),
                      block_table=i32(self.table).view(n, self.width), free_pages=i32(self.free), free_count=i32([self.count]),
                      free_count_out=i32([77]), row_starts=torch.full((n + 1,), 77, dtype=torch.int32, device="cuda"),
                      page_starts=torch.full((n + 1,), 77, dtype=torch.int32, device="cuda"),
                      slots=torch.full((self.max_rows,), 77, dtype=torch.int64, device="cuda"),
                      positions=torch.full((self.max_rows,), 77, dtype=torch.int32, device="cuda"),
                      row_seq=torch.full((self.max_rows,), 77, dtype=torch.int32, device="cuda"), status=i32([0]))
        return self

    def call(self, **kw):
        da.decode_attn_step_tables(self.shape, **(self.t | kw))
        return self

    def check(self, lens="seq_lens_out", count="free_count_out", row_seq=True):
        want, t = self.expect(), self.t
        got = {"lens": t[lens], "count": t[count], "free": t["free_pages"], "table": t["block_table"], "row_starts": t["row_starts"],
               "page_starts": t["page_starts"], "slots": t["slots"], "positions": t["positions"], "status": t["status"]}
        if row_seq:
            got["row_seq"] = t["row_seq"]
        for name, x in got.items():
            assert np.array_equal(x.cpu().numpy().ravel(), np.array(want[name], dtype=np.int64).ravel()), name
        return want


def mixed(n, seed, most=300, grow=70):
    rng = random.Random(seed)
    lens = [rng.choice([0, 1, 15, 16, 17, rng.randint(0, most)]) for _ in range(n)]
    gains = [rng.choice([0, 1, 1, 1, rng.randint(0, grow), -rng.randint(0, 20), -l, -1 << 30]) for l in lens]
    return lens, gains


@pytest.mark.parametrize("page", [16, 32, 256])
@pytest.mark.parametrize("n", [1, 2, 31, 64, 257, 1023, 1024, 1025, 2500])
def test_steps(n, page):
    s = Step(*mixed(n, n + page), page=page, seed=n)
    s.max_rows += n % 7
    want = s.put().call().check()
    assert want["status"] == da.DA_OK


@pytest.mark.parametrize("rows", [8189, 8192, 8193, 70001])
def test_one_launch_and_two(rows):
    gains = [rows // 3, 0, 1, rows - rows // 3 - 2, -40, 1]
    s = Step([5, 0, 16, 100, 640, 3], gains, seed=rows)
    assert s.put().call().check()["status"] == da.DA_OK
    s.max_rows += 1000                                                         # padding behind
    assert s.put().call().check()["status"] == da.DA_OK


def test_nothing_to_do():
    assert Step([], []).put().call().check()["status"] == da.DA_OK
    assert Step([0, 40], [0, 0], max_rows=9).put().call().check()["status"] == da.DA_OK
    assert Step([33], [-33]).put().call().check()["status"] == da.DA_OK


def test_in_place():
    s = Step(*mixed(300, 5), seed=2).put()
    s.call(seq_lens_out=s.t["seq_lens"], free_count_out=s.t["free_count"]).check("seq_lens", "free_count")


def test_without_row_seq_and_unaligned():
    s = Step(*mixed(90, 6), seed=3).put()
    n = s.max_rows
    slots, positions = torch.zeros(n + 1, dtype=torch.int64, device="cuda")[1:], torch.zeros(n + 3, dtype=torch.int32, device="cuda")[3:]
    s.t |= {"slots": slots, "positions": positions, "row_seq": None}
    s.call().check(row_seq=False)


@pytest.mark.parametrize("seed", range(12))
@pytest.mark.parametrize("n", [40, 1500])
def test_short_of_pages_rows_and_room(n, seed):
    rng = random.Random(seed)
    lens, gains = mixed(n, seed + 50)
    rows = sum(max(0, g) for g in gains)
    s = Step(lens, gains, seed=seed, free=rng.randint(0, 2 * n), max_rows=rng.choice([rows, rng.randint(0, rows)]))
    s.capacity = rng.choice([s.capacity, rng.randint(s.count, max(s.count, s.capacity))])
    s.free = s.free[:s.capacity]
    if rng.random() < 0.5:                                                     # lengths that no table row can hold, or none at all
        s.lens[rng.randrange(n)] = s.width * s.page + 1
        s.lens[rng.randrange(n)] = -3
        s.gains[rng.randrange(n)] = (1 << 31) - 1
    s.put().call().check()


def test_each_shortage_is_told():
    assert Step([0, 0], [16, 17], spare=-1).put().call().check()["status"] == da.DA_ERR_NO_PAGES
    assert Step([0, 5], [16, 17], max_rows=32).put().call().check()["status"] == da.DA_ERR_WORKSPACE_TOO_SMALL
    assert Step([160, 5], [-160, 1], capacity=12).put().call().check()["status"] == da.DA_ERR_NO_PAGES
    assert Step([160], [1], width=10).put().call().check()["status"] == da.DA_ERR_STALE_PLAN
    bad = Step([0, 16], [5, 1], num_pages=1)
    assert bad.put().call().check()["status"] == da.DA_ERR_BAD_PAGE
    for count in (-1, 1000):
        s = Step([0, 16], [5, 1])
        s.count = count
        assert s.put().call().check()["status"] == da.DA_ERR_STALE_PLAN


def test_many_steps_in_a_graph_lose_no_page():
    """A captured step, in place, with the gains changing from replay to replay: the pages in tables and list stay the same set."""
    rng = random.Random(1)
    n, page, width = 24, 16, 40
    s = Step([0] * n, [3] * n, page=page, width=width, spare=400, max_rows=700, seed=1)
    s.capacity += 100
    s.free += [-1] * 100
    s.put()
    t = s.t | {"seq_lens_out": s.t["seq_lens"], "free_count_out": s.t["free_count"]}
    every = sorted(s.free[:s.count])
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        da.decode_attn_step_tables(s.shape, **t)
    lens = [0] * n
    for _ in range(60):
        gains = [rng.choice([1, 1, 1, rng.randint(0, 60), -rng.randint(0, 30), -l]) for l in lens]
        gains = [min(g, width * page - l) for g, l in zip(gains, lens)]
        t["gains"].copy_(torch.tensor(gains, dtype=torch.int32))
        graph.replay()
        lens = [max(0, a + b) for a, b in zip(lens, gains)]
        assert t["seq_lens"].tolist() == lens
        table, count = t["block_table"].tolist(), int(t["free_count"])
        held = [p for row, m in zip(table, lens) for p in row[:-(-m // page)]]
        assert sorted(held + t["free_pages"].tolist()[:count]) == every
        starts = t["row_starts"].tolist()
        for b in (0, n - 1):
            for i in range(max(0, gains[b])):
                p = lens[b] - gains[b] + i
                assert int(t["slots"][starts[b] + i]) == table[b][p // page] * page + p % page
    assert int(t["status"]) == da.DA_OK
    del graph


@pytest.mark.parametrize("rows", [500, 20000])
def test_nothing_is_written_beside_the_buffers(rows):
    s = Step(*mixed(200, 9, grow=rows // 60), seed=4)
    s.max_rows += 13
    s.put()
    held = {}
    for name in ("seq_lens_out", "block_table", "free_pages", "free_count_out", "row_starts", "page_starts", "slots", "positions",
                 "row_seq", "status"):
        x = s.t[name]
        big = torch.full((x.numel() + 64,), 1234567, dtype=x.dtype, device="cuda")
        big[32:32 + x.numel()] = x.reshape(-1)
        held[name] = big
        s.t[name] = big[32:32 + x.numel()].view(x.shape)
    s.call().check()
    for name, big in held.items():
        assert (big[:32] == 1234567).all() and (big[-32:] == 1234567).all(), name


def test_a_batch_larger_than_shared_memory():
    n = 5000
    rng = random.Random(3)
    lens = [rng.randint(0, 90) for _ in range(n)]
    for rows, gains in ((0, [rng.choice([0, 1, 1, 3]) for _ in range(n)]), (20000, [rng.randint(0, 9) for _ in range(n)])):
        s = Step(lens, gains, seed=rows)
        s.max_rows += rows
        assert s.put().call().check()["status"] == da.DA_OK
