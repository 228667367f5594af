"""What lies between the feed-forward block's products and passes the type's largest number is infinite, whatever the number of rows:
with weights of one sign, so is what it adds to, and never NaN."""
import math

import pytest
import torch

from tests.test_gpu_block import block, gen  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu

ROWS = [1, 8, 9, 12, 16, 17, 20, 32, 33, 64, 65, 90]   # either side of where the kernels change


def signs(g, n):
    s = torch.randn(n, generator=g, device="cuda").sign()
    s[:2] = torch.tensor([1.0, -1.0])
    return s


def overflowing(n, hidden, inner):
    """16-bit floats, where row n // 2 has one hidden activation of 600 * 200 (the largest number is 65504), whose derivatives by both
    projections are 1000 * 200 and 1000 * 600 times grad_y's largest, 1; the others are far within the range."""
    g = gen(n + hidden)
    r = lambda *shape: torch.randn(shape, generator=g, device="cuda")  # noqa: E731
    row, j = n // 2, inner // 2
    s, t = signs(g, hidden), signs(g, hidden)
    x, gy = r(n, hidden) * 2.0 ** -9, r(n, hidden).clamp(-4, 4) * 2.0 ** -7
    wg, wu, wd = r(inner, hidden) / 8, r(inner, hidden) / 8, r(hidden, inner) / 8
    x[row], gy[row] = s / 32, t
    wg[j], wu[j], wd[:, j] = s * (600 * 32 / hidden), s * (200 * 32 / hidden), t * (1000 / hidden)
    return row, j, s, t, [v.half() for v in (x, wg, wu, wd, gy)]


@pytest.mark.parametrize("n", ROWS)
@pytest.mark.parametrize("hidden,inner", [(64, 96), (65, 97), (128, 192)])
@pytest.mark.parametrize("save", [None, "full", "packed"])
def test_hidden_activations_and_derivatives_of_16_bit_floats(block, n, hidden, inner, save):  # noqa: F811
    row, j, s, t, (x, wg, wu, wd, gy) = overflowing(n, hidden, inner)
    with block.DeftBlock(("ffn", "ffn_grad"), torch.float16, n, hidden, inner) as b:
        y = b.ffn(x, wg, wu, wd, save=save)
        y, saved = y if save else (y, None)
        gx, gg, gu, gd = b.ffn_grad(gy, x, wg, wu, wd, saved=saved)
        torch.cuda.synchronize()
    rows, columns = torch.arange(n, device="cuda") != row, torch.arange(inner, device="cuda") != j
    inf = torch.tensor(math.inf, dtype=torch.float16, device="cuda")
    assert torch.equal(y[row], t * inf) and torch.isfinite(y[rows]).all()
    assert torch.equal(gx[row], s * inf) and torch.isfinite(gx[rows]).all()
    assert torch.equal(gg[j], s * inf) and torch.isfinite(gg[columns]).all()
    assert torch.equal(gu[j], s * inf) and torch.isfinite(gu[columns]).all()
    assert torch.equal(gd[:, j], t * inf) and torch.isfinite(gd[:, columns]).all()


@pytest.mark.parametrize("n", ROWS)
@pytest.mark.parametrize("hidden,inner", [(64, 96), (65, 97), (128, 192)])
def test_the_largest_hidden_activation_that_is_finite(block, n, hidden, inner):  # noqa: F811
    """65512, which is rounded to 65504 (and, of few rows, 8 more)."""
    x, wg, wu, wd = (torch.zeros(shape, device="cuda") for shape in ((n, hidden), (inner, hidden), (inner, hidden), (hidden, inner)))
    x[n // 2, 0] = x[n // 2, 1] = 1.0
    wg[5, 0], wu[5, 0], wu[5, 1] = 128.0, 512.0, -0.1875   # (128 * 511.8125, and silu takes nothing of 128)
    wd[:, 5] = 2.0 ** -4
    with block.DeftBlock(("ffn",), torch.float16, n, hidden, inner) as b:
        y = b.ffn(x.half(), wg.half(), wu.half(), wd.half())
        torch.cuda.synchronize()
    # 65512 / 16 = 4094.5, a step of 2 there; 65504 / 16 = 4094
    assert (y[n // 2] == 4094.0).all() and (y.double().sum(dim=1) != 0).sum() == 1


@pytest.mark.parametrize("n", ROWS)
@pytest.mark.parametrize("hidden,inner", [(64, 96), (65, 97), (128, 192)])
def test_hidden_activations_of_bfloat16(block, n, hidden, inner):  # noqa: F811
    """2^128 (1 - 2^-10), a number of 32 bits that is rounded to infinity: so is y, with weights of 1."""
    g = gen(n)
    t = signs(g, hidden)
    x, wg, wu, wd = (torch.zeros(shape, device="cuda") for shape in ((n, hidden), (inner, hidden), (inner, hidden), (hidden, inner)))
    x[n // 2, 0] = x[n // 2, 1] = 1.0
    wg[5, 0], wu[5, 0], wu[5, 1] = 2.0 ** 64, 2.0 ** 64, -2.0 ** 54
    wd[:, 5] = t
    with block.DeftBlock(("ffn",), torch.bfloat16, n, hidden, inner) as b:
        y = b.ffn(x.bfloat16(), wg.bfloat16(), wu.bfloat16(), wd.bfloat16())
        torch.cuda.synchronize()
    assert torch.equal(y[n // 2], t.bfloat16() * math.inf)
    assert (y[torch.arange(n, device="cuda") != n // 2] == 0).all()
