"""How the checkpoints' rows are cut into launches, whose threads have to be fewer than 2^32, worked out on the host by the library's
own code: the launches have all rows once, in their order, and each is within the limit, at the corners of what a call may have.  No GPU needed."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2503_16815_amd", "csrc")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

PROGRAM = r"""
#include "block.h"
#include <cstdio>
#include <cstdlib>
using namespace deft;
int main(int argc, char **argv)   // rows, columns ...: "first rows workgroups" of each launch
{
    for (int i = 1; i + 1 < argc; i += 2) {
        const hipError_t e = by_launches(atoll(argv[i]), atoll(argv[i + 1]), [](int64_t first, const RowPieces &by) {
            printf("%lld %d %u ", (long long)first, by.rows, by.blocks());
            return hipSuccess;
        });
        printf("%d\n", (int)e);
    }
    int calls = 0;   // a launch that fails is the last one
    const hipError_t e = by_launches(1 << 20, 65536, [&](int64_t, const RowPieces &) { ++calls; return hipErrorInvalidValue; });
    printf("%d %d\n", calls, e == hipErrorInvalidValue);
    return 0;
}
"""

ROWS = [1, 2, 255, 256, 257, 1003, 2 ** 19, 2 ** 19 + 1, 2 ** 20 - 1, 2 ** 20]
COLUMNS = [32, 64, 1600, 2016, 2048, 2080, 4096, 16384, 30720, 30752, 32768, 32800, 65504, 65536]


@pytest.fixture(scope="module")
def launches(tmp_path_factory):
    if not os.path.exists(HIPCC):
        pytest.skip("hipcc not available")
    at = tmp_path_factory.mktemp("launches")
    source, program = at / "launches.cpp", at / "launches"
    source.write_text(PROGRAM)
    subprocess.run([HIPCC, "-x", "hip", "--offload-arch=gfx950", "--offload-host-only", "-std=c++17", "-w", "-I", CSRC, "-o", str(program), str(source)],
                   check=True, capture_output=True)
    sizes = [(n, w) for n in ROWS for w in COLUMNS]
    out = subprocess.run([str(program), *[str(v) for s in sizes for v in s]], check=True, capture_output=True, text=True).stdout.splitlines()
    assert len(out) == len(sizes) + 1
    return {s: [int(v) for v in line.split()] for s, line in zip(sizes, out)}, [int(v) for v in out[-1].split()]


def test_every_row_is_in_one_launch_within_the_limit(launches):
    for (n, width), said in launches[0].items():
        assert said.pop() == 0
        each = [said[i:i + 3] for i in range(0, len(said), 3)]
        at = 0
        for first, rows, blocks in each:
            assert first == at and rows > 0
            assert blocks * 256 < 2 ** 32, (n, width)
            assert blocks * 256 * 8 >= rows * width   # (eight elements a thread)
            at += rows
        assert at == n
        assert len(each) == 1 or n * -(-width // 2048) >= 2 ** 24, (n, width)


def test_a_launch_that_fails_is_the_last(launches):
    assert launches[1] == [1, 1]
