"""A call is refused a stream of another device than the handle's.  No GPU needed: the stream's device is all that is looked at."""
import types

import pytest


@pytest.mark.parametrize("name", ["embed", "embed_grad", "head_loss", "head_grad", "distill", "distill_grad"])
def test_streams_of_other_devices(name):
    import torch
    from paper_2503_16815_amd import ends
    e = object.__new__(ends.DeftEnds)
    e._h, e.dtype, e.device, e._index = None, torch.float32, torch.device("cuda", 0), 0
    with pytest.raises(ValueError, match="stream"):
        getattr(e, name)(stream=types.SimpleNamespace(device_index=1))
