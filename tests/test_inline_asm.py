"""Rules that the device sources' inline assembly keeps, read from the sources: the compiler looks for hazards of its own instructions
only, so an asm block states every register that it writes and holds every distance that its first instructions may need."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_08910_amd", "csrc")


def blocks():
    """(file, instructions, clobbers) of each asm statement that has instructions."""
    out = []
    for f in sorted(glob.glob(os.path.join(CSRC, "*.h*"))):
        src = open(f).read()
        for m in re.finditer(r'\basm(?:\s+volatile)?\s*\(((?:[^()"]|"(?:[^"\\]|\\.)*"|\((?:[^()]|\([^()]*\))*\))*)\)\s*;', src):
            body = m.group(1)
            head = re.match(r'\s*((?:"(?:[^"\\]|\\.)*"\s*)*)', body).group(1)
            text = "".join(re.findall(r'"((?:[^"\\]|\\.)*)"', head)).replace("\\n", "\n").replace("\\t", " ")
            parts = re.split(r":(?![^(]*\))", re.sub(r'"(?:[^"\\]|\\.)*"', lambda s: s.group(0).replace(":", " "), body[len(head):]))
            lines = [x.strip() for x in text.split("\n") if x.strip()]
            if lines:
                out.append((os.path.basename(f), lines, parts[3] if len(parts) > 3 else ""))
    return out


def test_blocks_are_found():
    assert sum("lds" in b[1][-1].split() for b in blocks()) == 2  # the loads into LDS, 16 and 4 bytes a lane


@pytest.mark.parametrize("block", blocks(), ids=lambda b: f"{b[0]}:{b[1][-1].split()[0]}")
def test_written_scalar_registers_are_clobbers(block):
    _, lines, clobbers = block
    for line in lines:
        op, *args = line.replace(",", " ").split()
        if op.startswith("s_") and args and re.fullmatch(r"m0|vcc|exec|s\d+|s\[\d+:\d+\]", args[0]):
            assert f'"{args[0]}"' in clobbers, (line, clobbers)


@pytest.mark.parametrize("block", blocks(), ids=lambda b: f"{b[0]}:{b[1][-1].split()[0]}")
def test_wait_states_ahead_of_buffer_loads(block):
    """A buffer access may follow a vector instruction that wrote one of its scalar registers (v_readfirstlane) after five wait states, and
    an access of LDS by M0 a write of M0 after one."""
    waits, since_m0 = 0, None
    for line in block[1]:
        op, *args = line.replace(",", " ").split()
        if op.startswith("buffer_"):
            assert waits >= 5, (line, waits)
            assert "lds" not in args or (since_m0 is not None and since_m0 >= 1), line
        n = int(args[0]) + 1 if op == "s_nop" else 1
        waits += n
        since_m0 = 0 if args and args[0] == "m0" else None if since_m0 is None else since_m0 + n
