"""What the prompt kernel's source has to keep, and no run on one kind of hardware shows."""
import os
import re

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_a_warpgroup_moves_its_registers_with_one_instruction():
    """setmaxnreg is an aligned instruction: all warps of a warpgroup execute the same one, so it stands once for the
    softmax warpgroups and once for the third, ahead of that one's roles."""
    with open(os.path.join(ROOT, "paper_2609_37062_b200", "csrc", "prompt.cuh")) as f:
        lines = f.read().split("\n")
    at = [i for i, line in enumerate(lines) if "setmaxnreg." in line.split("//")[0]]
    assert len(at) == 2
    dec, inc = at
    assert "setmaxnreg.dec" in lines[dec] and "setmaxnreg.inc" in lines[inc]
    for i in at:                                              # a statement, not the body of a lambda or a macro
        assert re.match(r"\s*asm volatile\(", lines[i]), lines[i]

    def branch_of(i):
        """The line that opens the block in which line i stands."""
        indent = len(lines[i]) - len(lines[i].lstrip())
        return next(line.strip() for line in reversed(lines[:i]) if line.strip() and not line.startswith("#")
                    and len(line) - len(line.lstrip()) < indent)
    assert branch_of(dec) == "if (role >= kPromptSoftmaxWarps) {"
    assert branch_of(inc) == "} else {"
