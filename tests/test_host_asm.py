"""CPU-only checks of the instructions that the kernels write by hand: the compiler takes them as they stand and puts no waits between them."""

import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2508_15806_amd", "csrc")


def blocks():
    """(file, instructions) of every asm statement."""
    for path in sorted(glob.glob(os.path.join(CSRC, "*"))):
        if not path.endswith((".hip", ".h")):
            continue
        for text in re.findall(r"\basm\s*(?:volatile)?\s*\(((?:\s*\"(?:[^\"\\]|\\.)*\")+)", open(path).read()):
            code = "".join(re.findall(r"\"((?:[^\"\\]|\\.)*)\"", text))
            yield os.path.basename(path), [x.strip() for x in re.split(r"\\n|;", code.replace("\\t", " ")) if x.strip()]


def states(code):
    """Wait states that instructions take: one each, s_nop n: n + 1."""
    return sum(int(x.split()[1]) + 1 if x.startswith("s_nop") else 1 for x in code)


def test_loads_wait_for_their_scalar_operands():
    """A load into LDS needs one wait state behind a scalar write of m0, and a load from memory five behind a vector instruction's write of its scalar address (v_readfirstlane), which
    may stand right before the statement."""
    seen = 0
    for name, code in blocks():
        for i, x in enumerate(code):
            if not re.match(r"(global|buffer|flat|scratch)_", x):
                continue
            seen += 1
            assert states(code[:i]) >= 5, (name, code)
            written = [j for j in range(i) if re.match(r"s_\w+ m0\b", code[j])]
            if "lds" in x:
                assert written and states(code[written[-1] + 1:i]) >= 1, (name, code)
    assert seen >= 2
