"""Host-side check of the generated gfx950 code of the head's products, which write their loads to LDS and
their matrix instructions as inline asm, so that the compiler's own hazard checks do not see them:

* a vector instruction that writes a scalar register (a lane read back, a spill) is followed by at least five wait
  states before a buffer load reads that register;
* on every path from a matrix instruction to a read of an accumulation register there are enough wait states.

No GPU needed."""
import os
import re
import subprocess
import tempfile

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2503_16815_amd", "csrc")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


LABEL = re.compile(r"^([.\w$]+):")
BRANCH = re.compile(r"^s_(c?)branch\w*\s+([.\w$]+)")


def kernels(text):
    """(name, instructions, label -> place) of every product kernel."""
    for m in re.finditer(r"^(\S*product_kernel\S*):[^\n]*\n(.*?)^\.Lfunc_end", text, re.M | re.S):
        code, at = [], {}
        for line in m.group(2).splitlines():
            c = line.split(";", 1)[0].strip()
            label = LABEL.match(c)
            if label:
                at[label.group(1)] = len(code)
            elif c and not c.startswith("."):
                code.append(c)
        yield m.group(1), code, at


def waited(c):
    """Wait states that an instruction takes, at least."""
    return 1 + (int(c.split()[1], 0) if c.startswith("s_nop") else 0)


def early_reads(code, at):
    """Reads of accumulation registers that some path reaches less than 18 wait states behind a matrix instruction."""
    seen, bad, work = {}, set(), [(0, 99)]
    while work:
        i, since = work.pop()
        while i < len(code) and since < seen.get(i, 100):
            seen[i] = since
            c = code[i]
            if c.startswith("v_accvgpr_read") and since < 18:
                bad.add(i)
            since = 0 if c.startswith("v_mfma") else min(99, since + waited(c))
            if c.startswith("s_endpgm"):
                break
            m = BRANCH.match(c)
            if m:
                work.append((at[m.group(2)], since))
                if not m.group(1):
                    break
            i += 1
    return sorted(bad)


def registers(operands):
    found = set()
    for a, b in re.findall(r"\bs\[(\d+):(\d+)\]", operands):
        found |= set(range(int(a), int(b) + 1))
    return found | {int(a) for a in re.findall(r"\bs(\d+)\b", operands)}


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not available")
@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
def test_loads_and_products_written_as_asm(kind):
    with tempfile.TemporaryDirectory() as tmp:
        out = os.path.join(tmp, "out.s")
        subprocess.run([HIPCC, "--offload-arch=gfx950", "-O3", "-std=c++17", "-fno-gpu-rdc", "-Xclang", "-target-feature",
                        "-Xclang", "-packed-fp32-ops", "-w", "--cuda-device-only", "-S", "-o", out,
                        os.path.join(CSRC, f"ends_head_{kind}.hip")], check=True, capture_output=True)
        found = list(kernels(open(out).read()))
    assert len(found) == (23 if kind == "f32" else 24)   # four epilogues, six shapes of tiles (few logits in 32 bits apart)
    for name, code, at in found:
        loads = [i for i, c in enumerate(code) if c.startswith("buffer_load_dwordx4") and c.endswith("lds")]
        assert loads, name
        for i in loads:
            reads, states = registers(code[i]), 0
            for c in reversed(code[max(0, i - 8):i]):
                if states >= 5:
                    break
                op, _, rest = c.partition(" ")
                assert not (op.startswith("v_") and registers(rest.split(",")[0]) & reads), (name, c, code[i])
                states += waited(c)
        assert sum(c.startswith("v_mfma") for c in code) >= 32, name
        assert not early_reads(code, at), name
