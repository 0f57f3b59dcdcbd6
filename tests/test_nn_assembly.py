"""Assembly written in the kernels' sources: the compiler sees neither what a line of it
writes besides its operands nor how long it has to wait, so every statement says the one
and does the other."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2010_13972_amd", "csrc")


def statements():
    """(file, its text, everything after the text) of each asm statement with instructions."""
    for path in sorted(glob.glob(os.path.join(CSRC, "*"))):
        text = open(path).read()
        for m in re.finditer(r"\basm\s+volatile\s*\(((?:\s*\"[^\"]*\")+)([^;]*)\);", text):
            code = "".join(re.findall(r'"([^"]*)"', m.group(1)))
            if code.strip():
                yield os.path.basename(path), code.replace("\\n", "\n").replace("\\t", " "), m.group(2)


def test_m0_is_declared():
    seen = 0
    for name, code, rest in statements():
        if re.search(r"^\s*s_\w+ m0\b", code, re.M):
            seen += 1
            assert '"m0"' in rest.rsplit(":", 1)[1], (name, code)
    assert seen


def test_scalars_of_a_load_have_settled():
    """A memory instruction reads scalar registers that a vector instruction may have written
    just before: 5 wait states, an instruction or a step of s_nop each.  m0 needs one."""
    seen = 0
    for name, code, _ in statements():
        lines = [l.strip() for l in code.split("\n") if l.strip()]
        for i, line in enumerate(lines):
            if not re.match(r"(buffer|global|flat|scratch)_", line):
                continue
            seen += 1
            waits = 0
            for before in reversed(lines[:i]):
                nop = re.match(r"s_nop (\d+)", before)
                waits += int(nop.group(1)) + 1 if nop else 1
                if re.match(r"s_\w+ m0\b", before):
                    assert waits >= 2, (name, code)
            assert waits >= 5, (name, code)
    assert seen
