"""Inline assembly of the kernels names every register that it writes by name."""
import glob
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCES = sorted(glob.glob(os.path.join(ROOT, "paper_2606_14782_amd", "csrc", "*")))

WRITES = re.compile(r"^\s*[a-z]\w*\s+(m0|vcc|exec|[sv]\d+|[sv]\[\d+:\d+\])\s*,")


def _statements(text):
    """Parts of every asm statement (code, outputs, inputs, clobbers): split at colons
    outside of strings and brackets."""
    for m in re.finditer(r"\basm\b\s*(?:volatile\b)?\s*\(", re.sub(r"//[^\n]*", "", text)):
        rest = re.sub(r"//[^\n]*", "", text)[m.end():]
        parts, depth, at, quoted, i = [], 0, 0, False, 0
        while depth >= 0:
            c = rest[i]
            if c == '"' and (i == 0 or rest[i - 1] != "\\"):
                quoted = not quoted
            elif not quoted:
                depth += (c in "([") - (c in ")]")
                if c == ":" and depth == 0 or depth < 0:
                    parts.append(rest[at:i])
                    at = i + 1
            i += 1
        yield parts


def _strings(part):
    return re.findall(r'"((?:[^"\\]|\\.)*)"', part)


def _undeclared(text):
    """Instructions that write a register which their statement does not name as written."""
    found = []
    for parts in _statements(text):
        clobbers = _strings(parts[3]) if len(parts) > 3 else []
        for line in "".join(_strings(parts[0])).replace("\\t", " ").split("\\n"):
            m = WRITES.match(line)
            if m and m.group(1) not in clobbers:
                found.append((line.strip(), m.group(1)))
    return found


def test_the_search_finds_what_it_is_for():
    bad = r'asm volatile("s_mov_b32 m0, %0\n\ts_nop 0" :: "s"(f(a, (b))), "v"(at[i]) : "memory");'
    assert _undeclared(bad) == [("s_mov_b32 m0, %0", "m0")]
    assert _undeclared(bad.replace('"memory"', '"m0", "memory"')) == []
    assert _undeclared('asm volatile("" : "+v"(x));') == []
    assert _undeclared(r'asm("s_nop 0\n\tv_mov_b32 v7, %0" : : "v"(x ? a : b));') == [("v_mov_b32 v7, %0", "v7")]


@pytest.mark.parametrize("path", SOURCES, ids=os.path.basename)
def test_registers_written_by_name_are_declared(path):
    assert _undeclared(open(path).read()) == []
