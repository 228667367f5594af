"""Distillation at the limits of its types: logits of the type's lowest and largest value, which are finite and have a
softmax like any others.  The sizes run both of its kernels: rows that stay in registers (up to 65536 32-bit or 131072
16-bit logits) and longer ones.  Definitions and bounds as in test_gpu_ends.py."""
import pytest

from tests.test_gpu_ends import ALL, distill_definition, generator, handle, torch, within  # noqa: F401 (torch is a fixture)

pytestmark = pytest.mark.gpu

SIZES = [100, 8003, 12345, 30001, 50257, 100003, 140001]   # (every width of workgroup, by 32- or by 16-bit logits)


@pytest.mark.parametrize("dtype", ALL)
@pytest.mark.parametrize("vocab", SIZES)
@pytest.mark.parametrize("t", [0.5, 1.0, 3.0])
def test_lowest_and_largest_values(torch, dtype, vocab, t):  # noqa: F811
    rows, k = 8, 4
    g = generator(torch, vocab)
    z = torch.randn((rows, vocab), generator=g, device="cuda").to(getattr(torch, {"f32": "float32", "f16": "float16", "bf16": "bfloat16"}[dtype]))
    low, high = torch.finfo(z.dtype).min, torch.finfo(z.dtype).max
    index = torch.tensor([5, 60, 7, 90], dtype=torch.int32, device="cuda").repeat(rows, 1)
    value = torch.randn((rows, k), generator=g, device="cuda")
    lowest, largest = (torch.finfo(torch.float32).min, torch.finfo(torch.float32).max)
    z[0] = low                                              # a row that is masked as a whole: all alike
    z[1] = low                                              # all but one masked
    z[1, 5] = 2.0
    index[1, 1:] = -1
    z[2, 7] = high                                          # one that stands above all others
    index[2] = torch.tensor([7, -1, -1, -1])
    z[3] = high
    value[4] = lowest                                       # the teacher's entries are all alike
    value[5, 1] = lowest                                    # one of them masked
    value[6] = torch.tensor([0.0, 1.0, largest, -2.0])      # one above all others
    z[7, vocab // 2 + 50:] = low                            # a vocabulary of which a part is masked
    index[7] = torch.tensor([5, 3, 7, 90])
    row_grad = torch.rand(rows, generator=g, device="cuda") + 0.5
    _, loss, grad = distill_definition(torch, z, index, value, t, row_grad, dtype)
    with handle(torch, "distill", dtype, rows, vocab, 0, k) as e:
        status = torch.full((rows,), -9, dtype=torch.int32, device="cuda")
        alone = e.distill(z, index, value, t, status=status)
        assert status.tolist() == [0] * rows
        within(alone, *loss, "loss")
        got, got_grad = e.distill_grad(z, index, value, row_grad, t)
        within(got, *loss, "loss with gradient")
        within(got_grad, *grad, "grad_logits")


@pytest.mark.parametrize("dtype", ALL)
@pytest.mark.parametrize("vocab", SIZES)
def test_masked_label_costs_its_logit(torch, dtype, vocab):  # noqa: F811
    """The teacher keeps an entry that the student masks by the type's lowest value: a finite loss, that value's share of it."""
    t = 2.0
    z = torch.zeros((1, vocab), device="cuda").to(getattr(torch, {"f32": "float32", "f16": "float16", "bf16": "bfloat16"}[dtype]))
    z[0, 9] = torch.finfo(z.dtype).min
    index = torch.tensor([[9, 4]], dtype=torch.int32, device="cuda")
    value = torch.tensor([[-6.0, 0.0]], device="cuda")
    _, loss, _ = distill_definition(torch, z, index, value, t, torch.ones(1, device="cuda"), dtype)
    with handle(torch, "distill", dtype, 1, vocab, 0, 2) as e:
        within(e.distill(z, index, value, t), *loss, "loss")
