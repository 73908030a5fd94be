"""Decode steps over a cache in 4 bits whose plans limit the pieces of a sequence."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from packed_util import Cache, check, da, run  # noqa: E402

UNEVEN = [1662, 1955, 1732, 927, 334, 1066, 2537, 1769, 1539, 802, 2269, 2192, 1102, 2799, 1291, 2091, 2170, 1427, 198, 2687, 1235, 792, 397, 65,
          2428, 2123, 1124, 2006, 847, 2162, 797, 1965, 2779, 2456]


@pytest.mark.parametrize("limit", [1, 2, 3])
def test_every_row_is_attended(limit):
    c = Cache(UNEVEN, 6, 6, 64, seed=limit)
    for kw in ({}, {"fuse_combine": 1}, {"chunk_tokens": 16}, {"chunk_tokens": 16, "sm_count": 74}):
        out, lse, status = run(c, da.make_policy(cache_bits=4, max_splits=limit, **kw))
        assert status == da.DA_OK
        check(c, out, lse, str(kw))
