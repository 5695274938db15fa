"""Inline assembly names what it changes: a register that it writes and does not name may be one that the compiler holds a
value in."""
import os
import re

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2408_04323_amd", "csrc")


def _statements():
    for name in sorted(f for f in os.listdir(CSRC) if f.endswith((".h", ".hip", ".cpp"))):
        text = open(os.path.join(CSRC, name)).read()
        for m in re.finditer(r"\basm\b(?:\s+volatile)?\s*\(((?:[^()\"]|\"(?:[^\"\\]|\\.)*\"|\([^()]*\))*)\)", text):
            yield name, m.group(1)


def test_assembly_names_the_registers_that_it_writes():
    found = 0
    for name, body in _statements():
        code = "".join(re.findall(r'"((?:[^"\\]|\\.)*)"', body.split("::")[0].split(" :")[0]))
        for line in code.replace("\\n", "\n").replace("\\t", " ").split("\n"):
            m = re.match(r"\s*[sv]_\w+\s+(m0|vcc|scc|exec|[sv]\d+|[sv]\[\d+:\d+\])\s*,", line)
            if m:
                found += 1
                assert f'"{m.group(1)}"' in body.rsplit(":", 1)[-1], (name, line)
    assert found  # the pattern still sees the statements
