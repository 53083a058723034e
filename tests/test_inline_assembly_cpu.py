"""What inline assembly in the kernels does to registers that it names itself is declared, so that the compiler keeps nothing in them across it."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2601_16986_amd", "csrc")
REGISTERS = re.compile(r"\b(m0|vcc|exec|flat_scratch|s\d+|v\d+|s\[\d+:\d+\]|v\[\d+:\d+\])\b")


def statements():
    for path in sorted(glob.glob(os.path.join(CSRC, "*.h")) + glob.glob(os.path.join(CSRC, "*.hip"))):
        with open(path) as f:
            text = f.read()
        for m in re.finditer(r'\basm(?:\s+volatile)?\s*\(((?:[^()"]|"(?:\\.|[^"\\])*"|\((?:[^()"]|"[^"]*")*\))*)\)\s*;', text):
            yield os.path.basename(path), text.count("\n", 0, m.start()) + 1, m.group(1)


def test_registers_named_in_assembly_are_clobbered():
    found = list(statements())
    assert sum("global_load_lds" in body for _, _, body in found) == 2, "the loads into LDS, which say where to by m0"
    for name, line, body in found:
        parts = re.split(r':(?=(?:[^"]*"[^"]*")*[^"]*$)', body)
        named, declared = set(REGISTERS.findall(parts[0])), set(re.findall(r'"(\w+)"', parts[3])) if len(parts) > 3 else set()
        assert named <= declared, f"{name}:{line} writes {named - declared} without saying so"
