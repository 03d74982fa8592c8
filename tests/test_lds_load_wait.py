"""A load to LDS written in inline assembly keeps its distance from the vector instructions that set its descriptor.

The hardware does not check a memory instruction's scalar registers against a vector instruction that is still writing them
(v_readfirstlane, v_readlane, a comparison): five wait states have to lie between, or the load may use the old base or size.
For its own memory instructions the compiler puts them there; inside inline assembly it does not look."""
import os
import re
import subprocess

import pytest

from paper_2607_06202_amd import _build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
WAIT_STATES = 5


def scalar_registers(operand: str) -> set:
    m = re.fullmatch(r"s\[(\d+):(\d+)\]", operand) or re.fullmatch(r"s(\d+)()", operand)
    return set(range(int(m[1]), int(m[2] or m[1]) + 1)) if m else set()


def instructions(assembly: str):
    """Mnemonic and operands of each instruction, wait states counted as the instruction issues."""
    for line in assembly.split("\n"):
        text = line.split(";")[0].strip()
        if text and not text.startswith(".") and not text.endswith(":"):
            op, *operands = text.replace(",", " ").split()
            yield op, operands


def distances(assembly: str):
    """For each load to LDS, the wait states since a vector instruction last wrote one of its scalar registers."""
    written, clock = {}, 0
    for op, operands in instructions(assembly):
        if op.startswith("buffer_load") and "lds" in operands:
            used = set().union(*map(scalar_registers, operands))
            yield min((clock - written[r] for r in used if r in written), default=clock)
        clock += int(operands[0], 0) + 1 if op == "s_nop" else 1
        if op.startswith("v_") and operands:
            for r in scalar_registers(operands[0]):
                written[r] = clock
        elif op.startswith("s_") and operands:
            for r in scalar_registers(operands[0]):
                written.pop(r, None)


@pytest.fixture(scope="module")
def assembly(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("lds") / "probe.s")
    subprocess.check_call([_build.HIPCC, *_build.FLAGS, "-I", os.path.join(ROOT, "paper_2607_06202_amd", "csrc"),
                           "--cuda-device-only", "-S", os.path.join(ROOT, "tests", "host", "lds_load_probe.hip"), "-o", out],
                          stderr=subprocess.DEVNULL)
    with open(out) as f:
        return f.read()


def test_descriptor_set_right_before_the_load(assembly):
    found = list(distances(assembly))
    assert len(found) == 2, found  # both loads, and a vector write to their descriptors in sight
    assert min(found) >= WAIT_STATES, found
    assert "v_readfirstlane" in assembly
