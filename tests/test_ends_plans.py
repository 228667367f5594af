"""Which shape of tiles each product of the head runs at the sizes that the GPU tests give it, worked out on the host by the
library's own cost model: so that every shape of the gradients' products has a test, and keeps it when the model changes.
No GPU needed."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2503_16815_amd", "csrc")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
UNITS = 256   # compute units of an MI355X
SHAPES = ["256x256", "192x256", "160x256", "256x128", "128x128", "256x64"]

PROGRAM = r"""
#include "ends_shapes.h"
#include "ends_head.hip"
#include <cstdio>
#include <cstdlib>
namespace deft {   // (the plan alone is asked for)
#define NO_KERNELS(NAME)                                                                                            \
    hipError_t head_prepare_##NAME() { return hipSuccess; }                                                         \
    hipError_t head_loss_##NAME(const HeadPlan &, const deft_head_loss_t &, void *, int, hipStream_t) { return hipSuccess; } \
    hipError_t head_grad_##NAME(const HeadPlan &, const deft_head_grad_t &, void *, int, hipStream_t) { return hipSuccess; }
NO_KERNELS(bf16)
NO_KERNELS(f16)
NO_KERNELS(f32)
}
using namespace deft;
int main(int argc, char **argv)   // dtype, limit of rows, rows, vocabulary, hidden, units; a line per piece
{
    if (argc != 7) return 1;
    const int dtype = atoi(argv[1]), most = atoi(argv[2]), rows = atoi(argv[3]), vocab = atoi(argv[4]), hidden = atoi(argv[5]), units = atoi(argv[6]);
    HeadPlan p;
    head_plan(dtype, most, vocab, hidden, true, units, &p);
    const int64_t products = p.planes == 3 ? 6 : 1;
    const int splits = splits_of(hidden, rows, up(p.piece < vocab ? p.piece : vocab, kStep) / kStep * products, units);
    for (int first = 0; first < vocab; first += p.piece) {
        const int here = vocab - first < p.piece ? vocab - first : p.piece;
        printf("%d %d %d %d\n", shape_of(here, rows, up(hidden, kStep) / kStep * products, 1, units),
               shape_of(hidden, here, up(rows, kStep) / kStep * products, 1, units),
               shape_of(hidden, rows, up(here, kStep) / kStep * products, splits, units), splits);
    }
    return 0;
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    if not os.path.exists(HIPCC):
        pytest.skip("hipcc not available")
    at = tmp_path_factory.mktemp("plan")
    source, program = at / "plan.cpp", at / "plan"
    source.write_text(PROGRAM)
    subprocess.run([HIPCC, "-x", "hip", "--offload-arch=gfx950", "--offload-host-only", "-std=c++17", "-w", "-I", CSRC, "-o", str(program), str(source)],
                   check=True, capture_output=True)

    def ask(dtype, most, rows, vocab, hidden):
        """[(derivative, weights' gradient, hidden states' gradient, parts of the last)] of each piece of the vocabulary"""
        number = {"f32": 0, "f16": 1, "bf16": 2}[dtype]
        out = subprocess.run([str(program), *(str(x) for x in (number, most, rows, vocab, hidden, UNITS))], check=True, capture_output=True, text=True).stdout
        return [(*(SHAPES[int(x)] for x in line.split()[:3]), int(line.split()[3])) for line in out.splitlines()]
    return ask


def test_every_shape_of_the_gradients_products_is_tested(plan):
    from tests.test_gpu_ends import HEAD
    from tests.test_gpu_ends_shapes import SIZES
    from tests.test_gpu_ends_wide import WIDE
    sizes = [(r, r, v, h) for r, v, h, *_ in HEAD] + [(r, r, v, h) for r, v, h in SIZES] + list(WIDE)
    for dtype in ("bf16", "f16", "f32"):
        pieces = [x for rows, most, vocab, hidden in sizes for x in plan(dtype, most, rows, vocab, hidden)]
        for product in range(3):
            assert {x[product] for x in pieces} == set(SHAPES), (dtype, product)


def test_the_wide_tiles_of_the_hidden_states_gradient(plan):
    """The shape of the largest calls: in one part, and added to over several pieces of the vocabulary."""
    from tests.test_gpu_ends_wide import WIDE
    for dtype in ("bf16", "f16", "f32"):
        got = [plan(dtype, most, rows, vocab, hidden) for rows, most, vocab, hidden in WIDE]
        assert all(x[2:] == ("256x256", 1) for pieces in got for x in pieces), (dtype, got)
        assert max(len(pieces) for pieces in got) > 1, (dtype, got)
    assert all(x[2:] == ("256x256", 1) for rows, vocab, hidden in ((8192, 50257, 1600), (8192, 131072, 4096))
               for x in plan("bf16", rows, rows, vocab, hidden))
