"""The head's gradient by the positions' factors (row_grad): zeros among small ones, and factors that are not finite.
Definitions and bounds as in test_gpu_ends.py."""
import math

import pytest

from tests.test_gpu_ends import ALL, handle, head_definition, head_inputs, torch, within  # noqa: F401 (torch is a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ALL)
@pytest.mark.parametrize("size", [1.0, 100.0])
@pytest.mark.parametrize("top", [1e-5, 1.0 / 8192, 0.3])
@pytest.mark.parametrize("rows", [40, 300])
def test_factors_of_zero(torch, dtype, size, top, rows):  # noqa: F811
    """Positions with a label and a factor of zero (a loss mask) add nothing, however small the other factors and however
    large their own hidden states."""
    vocab, hidden = 700, 96
    h, w, labels, _ = head_inputs(torch, rows, rows, vocab, hidden, 0, 0, 0.1, dtype)
    h *= size
    w /= size
    h[0] = 60000.0
    labels[0] = 3
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    row_grad = top * (0.25 + 0.75 * torch.rand(rows, generator=g, device="cuda"))
    row_grad[::9] = 0.0
    valid, _, _, gh, gw = head_definition(torch, h, w, labels, 1.0, row_grad, dtype)
    with handle(torch, ("head_loss", "head_grad"), dtype, rows, vocab, hidden) as e:
        lse = e.head_loss(h, w, labels)[1]
        got_gh, got_gw = e.head_grad(h, w, labels, lse, row_grad)
        within(got_gh, gh[0], gh[1] + (top * 2.0 ** -36 * w.double().abs().sum(0) if dtype == "f16" else 0.0), "grad_hidden")
        assert bool((got_gh[::9] == 0).all())
        floor = 2.0 ** -22 * float(row_grad.sum()) * max(1.0, size * 2.0 ** -9) if dtype == "f16" else 0.0   # (hidden states are scaled by 2^-3 at the least)
        within(got_gw, gw[0], gw[1] + floor, "grad_weight")
        nothing = e.head_grad(h, w, labels, lse, torch.zeros_like(row_grad))
        assert all(bool((x == 0).all()) for x in nothing)


@pytest.mark.parametrize("dtype", ALL)
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("others", [1e-4, 64.0])
def test_factors_that_are_not_finite(torch, dtype, value, others):  # noqa: F811
    """They show in their own row of the hidden states' gradient and in all of the weights', and nowhere else."""
    rows, vocab, hidden = 90, 400, 64
    h, w, labels, _ = head_inputs(torch, 8, rows, vocab, hidden, 0, 0, 0.0, dtype)
    row_grad = torch.full((rows,), others, device="cuda")
    row_grad[7], row_grad[20] = value, 0.0
    with handle(torch, ("head_loss", "head_grad"), dtype, rows, vocab, hidden) as e:
        gh, gw = e.head_grad(h, w, labels, e.head_loss(h, w, labels)[1], row_grad)
    assert not bool(gh[7].isfinite().any()) and not bool(gw.isfinite().any())
    assert bool(gh[:7].isfinite().all()) and bool(gh[8:].isfinite().all()) and bool((gh[20] == 0).all())
