"""Distances that the compiler keeps between instructions, but not in front of or inside asm: kept by hand in the gradients of
the experts' products, and counted here in what it makes of them."""
import re
import subprocess

import pytest

from paper_2605_10670_amd import build


@pytest.fixture(scope="module")
def lines(tmp_path_factory):
    out = tmp_path_factory.mktemp("asm") / "product_grad.s"
    flags = [f for f in build.FLAGS if f not in ("-shared", "-fPIC")]
    subprocess.run([build.HIPCC, *flags, "-w", "-S", "--cuda-device-only", "-o", str(out), build.HERE + "/csrc/product_grad.hip"], check=True)
    return [s for s in (line.split(";")[0].strip() for line in out.read_text().splitlines()) if s]


def waits(line):
    """How many instructions this one counts for."""
    m = re.match(r"s_nop (\d+)$", line)
    return int(m[1]) + 1 if m else 1


def test_loads_into_lds_wait_for_their_address(lines):
    found = 0
    for i, line in enumerate(lines):
        if line.startswith("global_load_lds_dwordx4"):
            found += 1
            assert lines[i - 1] == "s_nop 4" and lines[i - 2].startswith("s_mov_b32 m0,"), lines[i - 3:i + 1]
    assert found > 0


def test_values_of_other_lanes_are_there(lines):
    """Two instructions at least between a vector instruction and one that reads other lanes' results of it."""
    found = 0
    for i, line in enumerate(lines):
        m = re.match(r"v_cndmask_b32_dpp v\d+, (v\d+), ", line)
        if not m:
            continue
        found += 1
        distance, j = 0, i - 1
        while distance < 2:
            to = re.match(r"v_\w+ (v\d+|v\[(\d+):(\d+)\]),", lines[j])
            if to:
                written = {to[1]} if to[2] is None else {f"v{n}" for n in range(int(to[2]), int(to[3]) + 1)}
                assert m[1] not in written, lines[j:i + 1]
            assert not lines[j].endswith(":"), lines[j:i + 1]
            distance += waits(lines[j])
            j -= 1
    assert found > 0


def test_matrix_instructions_are_done(lines):
    """Nineteen instructions at least between a matrix instruction (of 16 passes at most) and asm that reads its result: on the way from any
    of them to the first turn of a result there is the wait for that."""
    found, waited = 0, 0
    for line in lines:
        if line.startswith("v_mfma"):
            waited = 0
        elif line == "s_nop 15":
            waited += 16
        elif line.startswith("v_cndmask_b32_dpp"):
            found += 1
            assert waited >= 19
    assert found > 0
