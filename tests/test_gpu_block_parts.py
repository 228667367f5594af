"""Products in 32 bits that are cut into more parts than they have steps: the parts without a step add nothing."""
import pytest
import torch

from tests.test_gpu_block import ACTS, block, step  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu

# at 256 compute units: both projections and the derivative by h of 3 steps in 4 parts; x's gradient of 22 and 12 steps in 32 and 16; y of 11 and 7 in 16 and 8
SIZES = [(5, 192, 704), (5, 192, 384), (40, 192, 704), (70, 192, 448), (130, 192, 704), (66, 704, 192)]


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("save", [None, "full", "packed"])
@pytest.mark.parametrize("n,hidden,inner", SIZES)
def test_more_parts_than_steps(block, n, hidden, inner, save, act):  # noqa: F811
    step(block, n, hidden, inner, torch.float32, act, save, n % 2 == 0)
