"""No asm statement of the kernels writes a special register behind the compiler's back, and those that read m0 (loads to LDS) have it as
an operand, so that the compiler writes it."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2605_08565_amd", "csrc")
WRITES = re.compile(r"(?:^|\n)\s*[sv]_\w+\s+(m0|vcc|exec|scc)\b")       # the first operand is the destination


def statements():
    for path in sorted(glob.glob(os.path.join(CSRC, "*.h*"))):
        with open(path) as f:
            text = f.read()
        for at in re.finditer(r"\basm\s+(?:volatile\s*)?\(", text):
            depth, i, quoted = 1, at.end(), False
            while depth:
                c = text[i]
                if c == '"' and text[i - 1] != "\\":
                    quoted = not quoted
                depth += 0 if quoted else (c == "(") - (c == ")")
                i += 1
            yield os.path.basename(path), text[at.end():i - 1]


def test_special_registers_are_operands():
    loads = 0
    for path, body in statements():
        template = "".join(re.findall(r'"([^"]*)"', re.match(r'\s*((?:"[^"]*"\s*)+)', body).group(1))).replace("\\n", "\n").replace("\\t", "\t")
        assert not WRITES.findall(template), (path, body)
        if re.search(r"\blds\b", template):
            loads += 1
            assert '"{m0}"(' in body, (path, body)
    assert loads >= 1
