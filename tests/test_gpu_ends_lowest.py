"""The head where every logit is the type's lowest value, or next to it: finite, with a softmax like any others.  The last tile
of the vocabulary holds few rows, so that some wavefronts have none."""
import pytest

from tests.test_gpu_ends import handle, torch  # noqa: F401 (torch is a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,hidden", [("bf16", 64), ("f32", 64), ("f32", 5), ("bf16", 5)])
@pytest.mark.parametrize("rows", [1, 40, 90])
@pytest.mark.parametrize("vocab", [1, 3, 257, 300, 1000])
def test_all_logits_lowest(torch, dtype, hidden, rows, vocab):  # noqa: F811
    t = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    low = torch.finfo(t).min
    w = torch.zeros((vocab, hidden), dtype=t, device="cuda")
    w[:, 0] = low
    h = torch.zeros((rows, hidden), dtype=t, device="cuda")
    h[:, 0] = 1.0
    h[-1] = 0.0                                             # a row of logits of zero beside them
    labels = torch.zeros(rows, dtype=torch.int32, device="cuda")
    with handle(torch, ("head_loss", "head_grad"), dtype, rows, vocab, hidden) as e:
        loss, lse = e.head_loss(h, w, labels)
    # lse = low + log(vocab), which is low in 32 bits; the loss is that less the label's logit
    assert bool((lse[:-1] == low).all()) and bool((loss[:-1] == 0).all()), (lse[:3], loss[:3])
    want = torch.log(torch.tensor(float(vocab)))
    assert abs(float(lse[-1]) - float(want)) < 1e-4 and abs(float(loss[-1]) - float(want)) < 1e-4
