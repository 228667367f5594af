"""Checkpoints of as many rows and columns as a handle may have: more workgroups than one launch takes."""
import pytest
import torch

from tests import block_reference as R
from tests.test_gpu_block import block, gen  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu


def test_more_workgroups_than_a_launch_has(block):  # noqa: F811
    n, width, dtype = 1 << 20, 1 << 15, torch.bfloat16
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 112 << 30:
        pytest.skip("98 GiB of rows and their checkpoint do not fit")
    g = gen(7)
    at = [0, 1, n // 2, n - 2, n - 1]   # (the last row is the second launch's)
    some = torch.randn((len(at), width), generator=g, device="cuda").to(dtype)
    x = torch.zeros((n, width), dtype=dtype, device="cuda")
    for i, k in enumerate(at):
        x[k] = some[i]
    kept = block.Checkpoint(torch.full((n, width), 7, dtype=torch.int8, device="cuda"), torch.full((n, width // R.GROUP), 7.0, dtype=dtype, device="cuda"))
    with block.DeftBlock(("checkpoint", "restore"), dtype, n, 16, width) as b:
        b.checkpoint(x, out=kept)
        codes, scales = R.checkpoint(some)
        for i, k in enumerate(at):
            assert torch.equal(kept.codes[k], codes[i]) and torch.equal(kept.scales[k].double(), scales[i])
        x.fill_(3.0)
        b.restore(kept, out=x)
        torch.cuda.synchronize()
    for i, k in enumerate(at):
        assert torch.equal(x[k], R.kept(block.Checkpoint(codes[i:i + 1], scales[i:i + 1]))[0].to(dtype))
        x[k] = 0.0
        kept.codes[k] = 0
    for first in range(0, n, n // 16):   # (all others are zeros)
        rows = slice(first, first + n // 16)
        assert not kept.codes[rows].view(torch.int64).any() and not x[rows].view(torch.int64).any()
    # (-0.0 is none: the words are compared)
    scales = kept.scales.clone()
    scales[at] = 2.0 ** -126
    assert (scales == 2.0 ** -126).all()
    del x, kept, scales, rows
    torch.cuda.empty_cache()
