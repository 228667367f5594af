"""Distillation from teachers whose kept entries are NaN, on both of its kernels: rows that stay in registers (up to 65536
32-bit or 131072 16-bit logits) and longer ones.  Definitions and bounds as in test_gpu_ends.py."""
import math

import pytest

from tests.test_gpu_ends import ALL, distill_definition, generator, handle, torch, within  # noqa: F401 (torch is a fixture)

pytestmark = pytest.mark.gpu

SIZES = [100, 8003, 12345, 30001, 50257, 100003, 140001]   # (every width of workgroup, by 32- or by 16-bit logits)


@pytest.mark.parametrize("dtype", ALL)
@pytest.mark.parametrize("vocab", SIZES)
def test_teachers_that_are_not_numbers(torch, dtype, vocab):  # noqa: F811
    """A NaN among the kept entries makes the row's loss and its whole gradient's part at them NaN, and is no fault of the
    row's indices, whatever the vocabulary; a NaN that is not kept is nothing."""
    nan, inf = math.nan, math.inf
    value = torch.tensor([[nan, nan], [nan, -inf], [-inf, nan], [nan, 0.0], [-inf, -inf], [-inf, 1.0], [0.5, nan]], device="cuda")
    rows = len(value)
    index = torch.tensor([[5, 90]], dtype=torch.int32, device="cuda").repeat(rows, 1)
    index[6, 1] = -1
    z = torch.randn((rows, vocab), generator=generator(torch, 3), device="cuda").to(
        getattr(torch, {"f32": "float32", "f16": "float16", "bf16": "bfloat16"}[dtype]))
    row_grad = torch.ones(rows, device="cuda")
    with handle(torch, "distill", dtype, rows, vocab, 0, 2) as e:
        status = torch.full((rows,), -9, dtype=torch.int32, device="cuda")
        loss, grad = e.distill_grad(z, index, value, row_grad, 1.0, status=status)
        alone = e.distill(z, index, value, 1.0)
    assert status.tolist() == [0, 0, 0, 0, 1, 0, 0]
    for x in (loss, alone):
        assert x.isnan().tolist() == [True, True, True, True, False, False, False]
        assert float(x[4]) == 0.0
    assert bool(grad[:4, 5].isnan().all()) and bool(grad[:4, 90].isnan().all())
    assert bool((grad[4] == 0).all()) and bool(grad[5:].isfinite().all())
    _, want, want_grad = distill_definition(torch, z[5:], index[5:], torch.where(index[5:] < 0, 0.0, value[5:]), 1.0, row_grad[5:], dtype)
    within(loss[5:], *want, "loss")
    within(grad[5:], *want_grad, "grad_logits")
