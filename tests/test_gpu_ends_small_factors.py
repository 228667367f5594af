"""A row of the weights' gradient that depends on a position of a small factor (row_grad) alone.  Definitions and bounds as in
test_gpu_ends.py; beside them what deft_ends.h allows in 16-bit floats: a position whose factor is 2^-r of the largest
adds with an error of its own factor times 2^(t - 25) for each of its hidden states' elements and 2^(s - 38) for each of its
derivative's, where s = r - 4 from 0 to 12 and t = r - s."""
import pytest

from tests.test_gpu_ends import ALL, TINY, handle, head_definition, head_inputs, torch, within  # noqa: F401 (torch is a fixture)

pytestmark = pytest.mark.gpu


def shares(r):
    s = min(max(r - 4, 0), 12)
    return r - s, s


@pytest.mark.parametrize("dtype", ALL)
@pytest.mark.parametrize("r", [3, 6, 12, 20, 26])
@pytest.mark.parametrize("rows", [50, 200])
def test_a_row_of_one_small_factor(torch, dtype, r, rows):  # noqa: F811
    """A label that occurs at one position alone, whose factor is 2^-r of the others', while no other position gives that
    row of the vocabulary any probability: its gradient is that position's."""
    vocab, hidden, top, own = 900, 128, 1024.0, 899
    h, w, labels, _ = head_inputs(torch, r + rows, rows, vocab, hidden, 0, 0, 0.0, dtype)
    labels[labels == own] = 5
    labels[0] = own
    h[:, 0], h[0, 0], w[:, 0] = 1.0, 0.0, 0.0
    w[own] *= 0.1
    w[own, 0] = -60.0
    h[0, 1:9] = torch.tensor([1.01, 0.0137, -0.33, 2.5, -0.051, 0.77, 3.1, -1.0], device="cuda").to(h.dtype)
    row_grad = torch.full((rows,), top, device="cuda")
    row_grad[0] = top * 2.0 ** -r
    t, s = shares(r)
    _, _, _, gh, gw = head_definition(torch, h, w, labels, 1.0, row_grad, dtype)
    with handle(torch, ("head_loss", "head_grad"), dtype, rows, vocab, hidden) as e:
        got_gh, got_gw = e.head_grad(h, w, labels, e.head_loss(h, w, labels)[1], row_grad)
    factor = float(row_grad[0])
    in_w, in_h = (factor * (2.0 ** (t - 25) + 2.0 ** (s - 38) * h[0].double().abs()), 2.0 ** (s - 38) * w.double().abs().sum(0)) \
        if dtype == "f16" else (0.0, 0.0)
    within(got_gw[own], gw[0][own], gw[1][own] + in_w, "the row's gradient")
    within(got_gh, gh[0], gh[1] + row_grad[:, None].double() * in_h, "grad_hidden")
    off = (got_gw[own].double() - gw[0][own]).norm() / gw[0][own].norm()
    # half a unit of the elements' rounding, and of subnormal results where the factor makes them so
    assert float(off) <= {"f32": 2e-6, "f16": 2.0 ** -10, "bf16": 2.0 ** -7}[dtype] + TINY[dtype] / factor / 2
