"""Rules that the compiler cannot keep inside inline assembly, read from the sources: what a block writes is named or put back, and a scalar
address that a vector instruction may have written is not used within five wait states (CDNA: "VALU writes SGPR, VMEM reads that SGPR")."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2406_11430_amd", "csrc")


def blocks():
    """(file, instructions, clobbers) of every block with instructions in it."""
    for path in sorted(glob.glob(os.path.join(CSRC, "*"))):
        if not path.endswith((".hip", ".hpp", ".cpp")):
            continue
        with open(path) as f:
            text = f.read()
        for m in re.finditer(r'\basm\s+volatile\s*\(((?:[^()"]|"(?:[^"\\]|\\.)*"|\([^()]*\))*)\)\s*;', text):
            # split at the colons that stand outside of texts and brackets
            parts, rest = [], re.sub(r"//.*", "", m.group(1))
            piece = ""
            for token in re.findall(r'"(?:[^"\\]|\\.)*"|\([^()]*\)|.', rest, re.S):
                if token == ":":
                    parts.append(piece)
                    piece = ""
                else:
                    piece += token
            parts.append(piece)
            code = "".join(re.findall(r'"((?:[^"\\]|\\.)*)"', parts[0]))
            lines = [x.strip() for x in re.split(r"\\n|;", code.replace("\\t", " ")) if x.strip()]
            if lines:
                yield os.path.basename(path), lines, re.findall(r'"([^"]*)"', parts[3]) if len(parts) > 3 else []


BLOCKS = list(blocks())


def test_blocks_are_found():
    assert sum("global_load_lds" in " ".join(lines) for _, lines, _ in BLOCKS) == 2


@pytest.mark.parametrize("name,lines,clobbers", BLOCKS)
def test_scalar_registers_written_are_named_or_put_back(name, lines, clobbers):
    for line in lines:
        m = re.match(r"s_\w+\s+(m0|vcc|scc|s\d+|s\[\d+:\d+\])\b", line)
        if m and m.group(1) not in clobbers:
            register = m.group(1)
            kept = re.fullmatch(r"s_mov_b32 (%%\d), %s" % register, lines[0])
            assert kept and lines[-1] == "s_mov_b32 %s, %s" % (register, kept.group(1)), (name, line)
            assert not any(re.match(r"\w+ %s\b" % re.escape(kept.group(1)), x) for x in lines[1:]), (name, lines)


@pytest.mark.parametrize("name,lines,clobbers", BLOCKS)
def test_distance_to_scalar_addresses(name, lines, clobbers):
    """A memory instruction with an operand of the surrounding code: five wait states from the beginning of the block."""
    states = 0
    for line in lines:
        if re.match(r"(global|buffer|flat|scratch)_", line) and "%" in line:
            assert states >= 5, (name, lines)
        m = re.match(r"s_nop\s+(\d+)", line)
        states += int(m.group(1)) + 1 if m else 1
