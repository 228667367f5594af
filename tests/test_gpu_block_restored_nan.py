"""What the feed-forward block keeps in 8 bits, read back by `restore` and as x's checkpoint: a group of 32 that held a sum that is not
finite has NaN as its scale and comes back as NaN, all others as codes * scales."""
import math

import pytest
import torch

from tests import block_reference as R
from tests.test_gpu_block import TYPES, block, inputs  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu


def check(back, kept, bad, dtype):
    """bad: [rows][groups], those that come back as NaN."""
    width = kept.codes.shape[1]
    bad = bad.repeat_interleave(R.GROUP, dim=1)[:, :width]
    assert torch.equal(torch.isnan(kept.scales).repeat_interleave(R.GROUP, dim=1)[:, :width], bad)
    assert torch.equal(torch.isnan(back), bad)
    most = torch.finfo(dtype).max
    assert torch.equal(back[~bad], R.kept(kept).clamp(-most, most).to(dtype)[~bad])


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("n", [1, 8, 12, 20, 40, 64, 70, 300])
@pytest.mark.parametrize("hidden,inner", [(64, 96), (40, 67)])
def test_rows_that_are_not_finite(block, hidden, inner, n, dtype):  # noqa: F811
    groups = -(-inner // R.GROUP)
    for value in (math.nan, math.inf, -math.inf):
        x, wg, wu, wd, _ = inputs(n, hidden, inner, dtype)
        x[n // 2, 3] = value
        with block.DeftBlock(("ffn", "restore"), dtype, n, hidden, inner) as b:
            _, saved = b.ffn(x, wg, wu, wd, save="packed")
            back = [b.restore(saved.gate), b.restore(saved.up)]
            torch.cuda.synchronize()
        bad = torch.zeros((n, groups), dtype=torch.bool, device="cuda")
        bad[n // 2] = True   # (no weight is 0: every sum of this row is infinite or NaN)
        assert (wg != 0).all() and (wu != 0).all()
        for got, kept in zip(back, saved):
            check(got, kept, bad, dtype)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("n", [1, 8, 12, 20, 40, 64, 70, 300])
def test_groups_that_are_not_finite(block, n, dtype):  # noqa: F811
    """Of the gate alone, one whole group and the last one, which is shorter."""
    hidden, inner = 64, 99
    x, wg, wu, wd, _ = inputs(n, hidden, inner, dtype)
    wg[40], wg[97, 5] = math.nan, math.inf
    with block.DeftBlock(("ffn", "restore"), dtype, n, hidden, inner) as b:
        _, saved = b.ffn(x, wg, wu, wd, save="packed")
        gate, up = b.restore(saved.gate), b.restore(saved.up)
        torch.cuda.synchronize()
    assert (x != 0).all()
    bad = torch.zeros((n, 4), dtype=torch.bool, device="cuda")
    check(up, saved.up, bad, dtype)
    bad[:, 1] = bad[:, 3] = True
    check(gate, saved.gate, bad, dtype)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("n", [5, 70])
def test_as_the_checkpoint_of_x(block, n, dtype):  # noqa: F811
    """A projection's checkpoint read as the next call's x: its rows of NaN are rows of NaN in the gradients."""
    width = 96
    x, wg, wu, wd, gy = inputs(n, width, width, dtype)
    x[n // 2, 3] = math.inf
    with block.DeftBlock(("ffn", "ffn_grad"), dtype, n, width, width) as b:
        _, saved = b.ffn(x, wg, wu, wd, save="packed")
        gx, gg, gu, gd = b.ffn_grad(gy, saved.up, wg, wu, wd)
        torch.cuda.synchronize()
    others = torch.arange(n, device="cuda") != n // 2
    assert torch.isnan(gx[n // 2]).all() and torch.isfinite(gx[others]).all()
    for g in (gg, gu, gd):
        assert torch.isnan(g).all()
