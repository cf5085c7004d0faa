"""The feed-forward kernels as the compiler lays them out (host code, no GPU): the
library's own source and flags, compiled to assembly.

* A direct load to LDS that takes its base or its LDS address from scalar registers
  which a vector instruction wrote comes at least five wait states after it.  The
  loads are inline assembly: the compiler places no waits for what it does not see.
* No spilled register is touched beside matrix instructions: its access would drain
  the loads in flight."""
import os
import re
import subprocess

import pytest

from paper_2607_02043_amd import build

WAIT_STATES = 5


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """name -> instructions and labels"""
    if not os.path.exists(build.HIPCC):
        pytest.skip("hipcc not available")
    out = str(tmp_path_factory.mktemp("asm") / "ffn_kernels.s")
    flags = [f for f in build.FLAGS if f != "-fPIC"]
    subprocess.run([build.HIPCC, *flags, "-fPIC", "--offload-device-only", "-S", os.path.join(build.CSRC, "ffn_kernels.hip"), "-o", out],
                   check=True, capture_output=True)
    text = open(out).read()
    found = {}
    for m in re.finditer(r"^(_ZN3ffn\S*_kernel\S*):", text, re.M):
        body = text[m.end():text.index(".Lfunc_end", m.end())]
        lines = [line.split(";")[0].strip() for line in body.splitlines()]
        found[m.group(1)] = [x for x in lines if x and (x.endswith(":") or not x.startswith("."))]
    return found


def _registers(name):
    m = re.match(r"s\[(\d+):(\d+)\]$", name)
    return {f"s{i}" for i in range(int(m.group(1)), int(m.group(2)) + 1)} if m else {name}


def short_waits(lines):
    """(writer, load) of every load to LDS whose scalar operand a vector instruction wrote too shortly before."""
    code = [x for x in lines if not x.endswith(":")]
    bad = []
    for i, load in enumerate(code):
        if not load.startswith("global_load_lds"):
            continue
        need = {"m0"}
        for operand in re.findall(r"s\[\d+:\d+\]", load):
            need |= _registers(operand)
        waited = 0
        for before in reversed(code[max(0, i - 3 * WAIT_STATES):i]):
            if waited >= WAIT_STATES:
                break
            m = re.match(r"v_\w+ (m0|s\d+|s\[\d+:\d+\]),", before)
            if m and _registers(m.group(1)) & need:
                bad.append((before, load))
                break
            nop = re.match(r"s_nop (\d+)", before)
            waited += int(nop.group(1)) + 1 if nop else 1
    return bad


def test_the_scan_sees_a_short_wait():
    load = "global_load_lds_dwordx4 v2, s[6:7]"
    assert short_waits(["v_readfirstlane_b32 s7, v1", "s_nop 0", load])
    assert short_waits(["v_readfirstlane_b32 m0, v1", "s_nop 3", load])
    assert not short_waits(["v_readfirstlane_b32 s7, v1", "s_nop 4", load])
    assert not short_waits(["v_readfirstlane_b32 s8, v1", load])


def test_scalar_operands_of_loads_to_lds(kernels):
    assert sum(any("global_load_lds" in x for x in lines) for lines in kernels.values()) >= 9
    bad = {name: short_waits(lines)[:2] for name, lines in kernels.items() if short_waits(lines)}
    assert not bad, bad


def test_no_spills_beside_products(kernels):
    bad = []
    for name, lines in kernels.items():
        block = []
        for x in [*lines, "end:"]:
            if x.endswith(":"):
                if any("v_mfma" in y for y in block) and any(y.startswith("scratch_") for y in block):
                    bad.append(name)
                block = []
            else:
                block.append(x)
    assert not bad, bad
