"""The binding refuses what is no tensor, or a tensor without rows, with ValueError, whichever argument it is.  No GPU needed."""
import pytest


@pytest.mark.parametrize("name,count", [("embed", 2), ("embed_grad", 2), ("head_loss", 3), ("head_grad", 5), ("distill", 3), ("distill_grad", 4)])
@pytest.mark.parametrize("what", ["number", "list", "scalar"])
def test_no_tensors(name, count, what):
    import torch
    from paper_2503_16815_amd import ends
    e = object.__new__(ends.DeftEnds)
    e._h, e.dtype, e.device, e._index = None, torch.float32, torch.device("cpu"), -1
    thing = {"number": 3, "list": [[1.0]], "scalar": torch.tensor(1.0)}[what]
    with pytest.raises(ValueError):
        getattr(e, name)(*[thing] * count)
