"""Host-side check of the generated gfx950 code of the feed-forward block's products, as test_ends_isa.py has it for the head's:
wait states between what the compiler writes and the loads and matrix instructions that are written as inline asm, and no
registers of the main loop in memory.

No GPU needed."""
import os
import re
import subprocess
import tempfile

import pytest

from tests import test_ends_isa as isa


@pytest.mark.skipif(not os.path.exists(isa.HIPCC), reason="hipcc not available")
@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
def test_loads_and_products_written_as_asm(kind):
    with tempfile.TemporaryDirectory() as tmp:
        out = os.path.join(tmp, "out.s")
        subprocess.run([isa.HIPCC, "--offload-arch=gfx950", "-O3", "-std=c++17", "-fno-gpu-rdc", "-Xclang", "-target-feature",
                        "-Xclang", "-packed-fp32-ops", "-w", "--cuda-device-only", "-S", "-o", out,
                        os.path.join(isa.CSRC, f"block_ffn_{kind}.hip")], check=True, capture_output=True)
        text = open(out).read()
    assert not re.search(r"^\s+v_pk_(add|mul|fma)_f32", text, re.M)
    found = list(isa.kernels(text))
    assert len(found) == 5 * 2 + 6 * 3   # five shapes of tiles before the activation, six for each of the three other products
    for name, code, at in found:
        loads = [i for i, c in enumerate(code) if c.startswith("buffer_load_dwordx4") and c.endswith("lds")]
        assert loads, name
        for i in loads:
            reads, states = isa.registers(code[i]), 0
            for c in reversed(code[max(0, i - 8):i]):
                if states >= 5:
                    break
                op, _, rest = c.partition(" ")
                assert not (op.startswith("v_") and isa.registers(rest.split(",")[0]) & reads), (name, c, code[i])
                states += isa.waited(c)
        products = [i for i, c in enumerate(code) if c.startswith("v_mfma")]
        assert len(products) >= 16, name
        assert not early_reads(code, at), (name, [code[i] for i in early_reads(code, at)])
        assert not any(c.startswith("scratch_") for c in code[products[0]:products[-1]]), name


def reads_sums(c):
    """Whether an instruction reads accumulation registers: moves, and stores that take them as they are."""
    return c.startswith("v_accvgpr_read") or (re.match(r"(ds_write|global_store|scratch_store)", c) and re.search(r"\ba\[?\d", c))


def early_reads(code, at):
    """Reads of accumulation registers that some path reaches less than 18 wait states behind a matrix instruction."""
    seen, bad, work = {}, set(), [(0, 99)]
    while work:
        i, since = work.pop()
        while i < len(code) and since < seen.get(i, 100):
            seen[i] = since
            c = code[i]
            if reads_sums(c) and since < 18:
                bad.add(i)
            since = 0 if c.startswith("v_mfma") else min(99, since + isa.waited(c))
            if c.startswith("s_endpgm"):
                break
            m = isa.BRANCH.match(c)
            if m:
                work.append((at[m.group(2)], since))
                if not m.group(1):
                    break
            i += 1
    return sorted(bad)
