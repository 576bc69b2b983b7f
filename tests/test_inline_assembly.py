"""Registers that inline assembly writes by name are named to the compiler, which may keep something of its own there."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2504_04673_amd", "csrc")
FIXED = re.compile(r"\bm0\b|\bvcc(?:_lo|_hi)?\b|\bexec(?:_lo|_hi)?\b|\bs\d+\b|\bs\[\d+:\d+\]")


def statements(text):
    """Each asm statement, up to its closing parenthesis."""
    for m in re.finditer(r"\basm\s*(?:volatile\s*)?\(", text):
        depth, i, quoted = 1, m.end(), False
        while depth:
            c = text[i]
            if quoted:
                quoted = c != '"' or text[i - 1] == "\\"
            elif c == '"':
                quoted = True
            else:
                depth += (c == "(") - (c == ")")
            i += 1
        yield text[m.end():i - 1]


def written(statement):
    """Fixed registers that its instructions name first, where a destination stands."""
    code = "".join(re.findall(r'"((?:[^"\\]|\\.)*)"', statement.split(":")[0]))
    for line in re.split(r"\\n|;", code):
        words = line.replace("\\t", " ").split(None, 1)
        if len(words) == 2 and not words[0].startswith(("s_waitcnt", "s_nop", "s_barrier")):
            first = words[1].split(",")[0].strip()
            if FIXED.fullmatch(first):
                yield first


def test_registers_that_assembly_writes_are_named():
    found = 0
    for path in sorted(glob.glob(os.path.join(CSRC, "*"))):
        for s in statements(open(path).read()):
            for register in written(s):
                found += 1
                assert f'"{register}"' in s.rsplit(":", 1)[-1], f"{os.path.basename(path)}: {s}"
    assert found
