"""What scratch memory a handle of the feed-forward block holds, worked out on the host by the library's own plan: a handle whose calls
all go to the kernels for few rows holds only what these use, and every such call stays within it; others hold what they did.  No GPU needed."""
import itertools
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2503_16815_amd", "csrc")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
F32, F16, BF16 = range(3)

PROGRAM = r"""
#include "block_ffn.hip"
#include <cstdio>
#include <cstdlib>
using namespace deft;
int main(int argc, char **argv)   // dtype, rows, hidden, inner, grad ...
{
    for (int i = 1; i + 4 < argc; i += 5) {
        FfnPlan p{};
        const int64_t size = atoll(argv[i + 2]) * atoll(argv[i + 3]);
        const bool f32 = atoi(argv[i]) == DEFT_F32;
        ffn_plan(atoi(argv[i]), atoi(argv[i + 1]), atoi(argv[i + 2]), atoi(argv[i + 3]), atoi(argv[i + 4]) != 0, 256, &p);
        printf("%lld %lld %d %d\n", (long long)p.scratch_bytes, (long long)p.h, few_rows(f32, size, true), few_rows(f32, size, false));
    }
    return 0;
}
"""

ROWS = [1, 8, 9, 16, 17, 32, 33, 64, 65, 1000]
MATRICES = [(1, 1), (64, 96), (768, 2048), (1024, 2048), (1024, 2049), (1600, 6400), (2051, 3061), (2051, 3079), (4096, 12288), (16384, 65536)]


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    if not os.path.exists(HIPCC):
        pytest.skip("hipcc not available")
    at = tmp_path_factory.mktemp("scratch")
    source, program = at / "scratch.cpp", at / "scratch"
    source.write_text(PROGRAM)
    subprocess.run([HIPCC, "-x", "hip", "--offload-arch=gfx950", "--offload-host-only", "-std=c++17", "-w", "-I", CSRC, "-c", "-o", str(at / "scratch.o"),
                    str(source)], check=True, capture_output=True)
    subprocess.run([HIPCC, "-o", str(program), str(at / "scratch.o"), "-Wl,--unresolved-symbols=ignore-all"], check=True, capture_output=True)
    cases = [(t, n, h, i, g) for t, n, (h, i), g in itertools.product((F32, F16, BF16), ROWS, MATRICES, (0, 1))]
    out = subprocess.run([str(program), *[str(v) for c in cases for v in c]], check=True, capture_output=True, text=True).stdout.splitlines()
    assert len(out) == len(cases)
    return {c: [int(v) for v in line.split()] for c, line in zip(cases, out)}


def up(x, to):
    return -(-x // to) * to


def test_handles_for_few_rows_hold_what_these_use(plans):
    for (dtype, n, hidden, inner, grad), (held, h, _, _) in plans.items():
        element = 4 if dtype == F32 else 2
        fewest = 64 if dtype == F32 else 32 if hidden * inner <= 1 << 21 else 16
        used = 2 * 64 * up(inner, 8) * element   # two arrays of 64 rows of hidden activations
        if not grad and n <= fewest:
            assert h == 0 and used <= held < used + 256
        else:   # (the matrices as operands, of three 16-bit arrays in 32 bits)
            assert held >= used + 3 * hidden * inner * (6 if dtype == F32 else 2)


def test_no_call_of_a_smaller_matrix_leaves_the_kernels_for_few(plans):
    """A handle's limits bound its calls: of any matrices within them, read in place or not, the rows that go to these kernels are no
    fewer than of the limits' own, read in place."""
    few = {(t, h, i): v[2:] for (t, _, h, i, _), v in plans.items()}
    for (t, h, i), (whole, _) in few.items():
        for (t2, h2, i2), both in few.items():
            if t2 == t and h2 <= h and i2 <= i:
                assert min(both) >= whole
