"""The hidden states' gradient in tiles of 256 x 256 that are not cut into parts, which the largest calls run: of one piece of the
vocabulary, and added to over several.  Definitions and bounds as in test_gpu_ends.py."""
import pytest

from tests.test_gpu_ends import ALL, handle, head_definition, head_inputs, torch, within  # noqa: F401 (torch is a fixture)

pytestmark = pytest.mark.gpu

WIDE = [  # rows, limit of rows, vocab, hidden (what they run is worked out in test_ends_plans.py)
    (4090, 4090, 1100, 4001),
    (4096, 4096, 600, 4096),
    (4090, 1 << 17, 2100, 4001),   # several pieces
]


@pytest.mark.parametrize("dtype", ALL)
@pytest.mark.parametrize("rows,most,vocab,hidden", WIDE)
def test_wide_tiles(torch, dtype, rows, most, vocab, hidden):  # noqa: F811
    h, w, labels, row_grad = head_inputs(torch, rows + most, rows, vocab, hidden, 0, 0, 0.05, dtype)
    valid, loss, lse, gh, gw = head_definition(torch, h, w, labels, 1.0, row_grad, dtype)
    with handle(torch, ("head_loss", "head_grad"), dtype, most, vocab, hidden) as e:
        got_loss, got_lse = e.head_loss(h, w, labels)
        within(got_loss, *loss, "loss")
        within(got_lse, *lse, "lse")
        got = e.head_grad(h, w, labels, got_lse, row_grad)
        within(got[0], *gh, "grad_hidden")
        within(got[1], *gw, "grad_weight")
        # The bounds add up every error at its largest; in the norm, where they meet by chance, there is the
        # output's rounding (its largest relative size / sqrt(3), a half more for the derivative's; in 32 bits the sums')
        half = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}
        at_most = 1.5 * half[dtype] / 3 ** 0.5 if dtype != "f32" else 6e-6
        assert float((got[0].double() - gh[0]).norm() / gh[0].norm()) <= at_most
        again = e.head_grad(h, w, labels, got_lse, row_grad, need_weight=False)
        assert torch.equal(again[0], got[0])
