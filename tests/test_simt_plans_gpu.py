"""What AUTO plans of the CUDA-core kernel are cut for: its resident blocks, which its registers decide."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2609_37062_b200 import binding as da  # noqa: E402


@pytest.mark.parametrize("d", [64, 128])
def test_resident_blocks_by_group(d):
    """With one more at groups of 4, 64 rows of 30 to 900 tokens (32/8 heads of 128) take 70 us instead of 47."""
    blocks = []
    for group in range(1, 9):
        shape = da.make_shape(1, group, 1, d, 16, 9, 9, (16 * d, d, d))
        plan = da.decode_attn_plan(shape, da.make_policy(kernel=da.DA_KERNEL_SIMT), [100])
        blocks.append(plan.info().ctas_per_sm)
        plan.destroy()
    assert blocks == [4, 4, 4, 3, 3, 2, 2, 2]
