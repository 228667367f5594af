"""Which shape of tiles, and how many parts of a sum, each product of the feed-forward block takes at the sizes that the GPU tests
give it, worked out on the host by the library's own cost model: so that every shape of every product, whole and in parts, has a
test, and keeps it when the model changes.  No GPU needed."""
import os
import subprocess

import pytest

from tests import test_gpu_block as G

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2503_16815_amd", "csrc")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
UNITS = 256   # compute units of an MI355X
SHAPES = ["256x256", "192x256", "160x256", "256x128", "128x128", "256x64", "128x64"]
PRODUCTS = ["gate", "out", "by_h", "down", "projections", "input"]

PROGRAM = r"""
#include "block_ffn.h"
#include <cstdio>
#include <cstdlib>
using namespace deft;
template <typename F, int E> void tell(int64_t m, int64_t n, int64_t k, int arrays, bool split, int units)
{
    constexpr unsigned kWithout = E == kGate || E == kGateGrad ? kNoAct : kNoOther;
    const int64_t steps = up(k, kStep) / kStep * (split ? 6 : 1) * (E == kInput ? 2 : 1) * arrays;
    const int parts = F::parts_of(m, n, steps, units, kWithout);
    printf("%d %d ", shape_of(m, n, steps, parts, units, kWithout, F::kAlone), parts);
}
template <typename F> void all(int64_t n, int64_t hidden, int64_t inner, bool split, int units)
{
    const int arrays = F::panels(FfnScratch(FfnPlan{}, nullptr), (int)n, (int)inner, 0).arrays;
    tell<F, kGate>(up(inner, 16) * 2, n, hidden, 1, split, units);
    tell<F, kOut>(hidden, n, inner, arrays, split, units);
    tell<F, kGateGrad>(inner, n, hidden, 1, split, units);
    tell<F, kOuter>(inner, hidden, n, arrays, split, units);
    tell<F, kOuter>(hidden, 2 * up(inner, 256), n, arrays, split, units);
    tell<F, kInput>(hidden, n, inner, arrays, split, units);
    printf("\n");
}
int main(int argc, char **argv)   // whether in 32 bits, units; rows, hidden, inner ...
{
    const bool split = atoi(argv[1]) != 0;
    for (int i = 3; i + 2 < argc; i += 3) {
        const int n = atoi(argv[i]), hidden = atoi(argv[i + 1]), inner = atoi(argv[i + 2]);
        if (split) all<Ffn<float, bf16, 3>>(n, hidden, inner, true, atoi(argv[2]));
        else all<Ffn<bf16, bf16, 1>>(n, hidden, inner, false, atoi(argv[2]));
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
    subprocess.run([HIPCC, "-x", "hip", "--offload-arch=gfx950", "--offload-host-only", "-std=c++17", "-w", "-I", CSRC, "-c", "-o", str(at / "plan.o"),
                    str(source)], check=True, capture_output=True)
    subprocess.run([HIPCC, "-o", str(program), str(at / "plan.o"), "-Wl,--unresolved-symbols=ignore-all"], check=True, capture_output=True)

    def ask(split, sizes):
        """{product: [(shape, parts) of each size]}"""
        out = subprocess.run([str(program), str(int(split)), str(UNITS), *[str(v) for s in sizes for v in s]], check=True, capture_output=True, text=True)
        lines = [[int(v) for v in line.split()] for line in out.stdout.splitlines()]
        assert len(lines) == len(sizes)
        return {p: [(SHAPES[line[2 * i]], line[2 * i + 1]) for line in lines] for i, p in enumerate(PRODUCTS)}
    return ask


@pytest.mark.parametrize("split", [False, True], ids=["16-bit", "32-bit"])
def test_every_shape_of_every_product_has_a_test(plan, split):
    found = plan(split, G.SIZES + G.SHAPES)
    found["outer"] = found.pop("down") + found.pop("projections")   # (the same kernels)
    missing = {}
    for p, plans in found.items():
        shapes = {"256x256", "256x128", "128x128", "256x64", "128x64"} | (set() if p in ("gate", "by_h") else {"192x256"})
        got = {s for s, _ in plans}
        assert got <= shapes, p
        if shapes - got:
            missing[p] = shapes - got
        assert any(parts > 1 for _, parts in plans) and any(parts == 1 for _, parts in plans), p
    assert not missing, missing
