"""kv_group_attn at the ends of what its arguments may be."""
import pytest
import torch

from batchcase import Batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("layout", ["bhsd", "paged"])
@pytest.mark.parametrize("D,cap", [(64, 0.0), (128, 9.0)])
@pytest.mark.parametrize("ends", [(1, -1), (-1, 1)])
def test_positions_as_far_apart_as_they_may_be(ends, D, cap, layout):
    """2^31 between a token and those that it sees, and a token of the same rows some 1000 behind or ahead of it. With slopes of this size the distances are biases of 0.02 to 4."""
    a, b = (e * 2 ** 30 for e in ends)
    for near in (0, 700, 1000):
        positions = [a, a, b, b - ends[1] * near]
        batch = Batch([70], [4], 1, 8, D, torch.bfloat16, "16", layout, seed=D, slopes=[2.0e-9, 1.0e-9, 1.0e-10, 1.0e-11, 1.5e-9, 0.0, -1.0e-9, -1.0e-10], positions=positions, cap=cap)
        for n_splits in (0, 1, 2):
            batch.check(batch.attend(n_splits=n_splits))
