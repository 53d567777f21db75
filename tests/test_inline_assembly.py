"""Inline assembly declares the registers that it writes by name: the compiler may keep a value of its own there."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2405_12591_amd", "csrc")
# first operand of scalar and vector instructions; stores, waits and their like have none
_WRITTEN = re.compile(r"^\s*(?:s|v|ds|global|buffer)_\w+\s+(m0|vcc|exec|scc|[sv]\d+|[sv]\[\d+:\d+\])\b")


def _statements(text):
    for m in re.finditer(r"\basm\s*(?:volatile)?\s*\(", text):
        depth, at, quoted = 1, m.end(), False
        while depth:
            c = text[at]
            if c == '"' and text[at - 1] != "\\":
                quoted = not quoted
            elif not quoted:
                depth += (c == "(") - (c == ")")
            at += 1
        yield text[m.end():at - 1]


def test_written_registers_are_declared():
    seen = 0
    for path in sorted(glob.glob(os.path.join(CSRC, "*.h")) + glob.glob(os.path.join(CSRC, "*.hip"))):
        with open(path) as f:
            text = f.read()
        for s in _statements(text):
            code = re.match(r'\s*((?:"(?:[^"\\]|\\.)*"\s*)+)', s)
            if not code:
                continue
            lines = "".join(re.findall(r'"((?:[^"\\]|\\.)*)"', code.group(1))).replace("\\t", " ").split("\\n")
            clobbers = re.findall(r'"(\w+)"', s.rsplit(":", 1)[1]) if ":" in s else []
            for line in lines:
                m = _WRITTEN.match(line)
                if m:
                    seen += 1
                    assert m.group(1) in clobbers, "%s: %s writes %s without saying so" % (os.path.basename(path), line.strip(), m.group(1))
    assert seen >= 3
