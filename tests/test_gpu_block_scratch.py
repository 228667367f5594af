"""Handles that hold scratch memory for few rows alone give what handles with room for everything give, whatever is called within their
limits, and two of them at once."""
import pytest
import torch

from tests.test_gpu_block import TYPES, block, inputs  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows,hidden,inner", [(16, 1100, 2100), (32, 1024, 2048), (64, 1024, 4096), (1, 1600, 6400)])
def test_calls_within_the_limits(block, rows, hidden, inner, dtype):  # noqa: F811
    few = rows <= 16 or dtype == torch.float32 or (rows <= 32 and hidden * inner <= 1 << 21)
    with block.DeftBlock("ffn", dtype, rows, hidden, inner) as b, block.DeftBlock(("ffn", "ffn_grad"), dtype, 300, hidden, inner) as large, \
            block.DeftBlock("ffn", dtype, rows, hidden, inner) as other:
        held = b.info().scratch_bytes   # (two arrays of 64 rows of h; or the matrices as operands, among much else)
        assert held < 129 * (inner + 8) * torch.finfo(dtype).bits // 8 if few else held > 3 * hidden * inner * 2
        for n in sorted({1, 8, 9, 16, 17, 32, 33, 64}):
            if n > rows:
                continue
            for h, i, pad in ((hidden, inner, 0), (hidden, inner, 3), (64, inner, 0), (65, 97, 0), (1, 1, 0)):
                x, wg, wu, wd, _ = inputs(n, h, i, dtype, seed=n, pad=pad)
                x2 = inputs(n, h, i, dtype, seed=n + 100, pad=pad)[0]
                want = [large.ffn(v, wg, wu, wd, save="packed") for v in (x, x2)]
                got = [g.ffn(v, wg, wu, wd, save="packed") for g, v in ((b, x), (other, x2))]
                torch.cuda.synchronize()
                for (y, saved), (y2, saved2) in zip(want, got):
                    assert torch.equal(y, y2), (n, h, i, pad)
                    for c, c2 in zip(saved, saved2):
                        assert torch.equal(c.codes, c2.codes) and torch.equal(c.scales, c2.scales)
