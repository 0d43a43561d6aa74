"""Inline assembly names every register that it writes by name, so that the compiler keeps nothing there (no GPU needed)."""
import glob
import os
import re

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _statements(text):
    """The asm statements of a source, from the keyword to the parenthesis that closes them."""
    for m in re.finditer(r"\basm\b(?:\s+volatile)?\s*\(", text):
        depth, quoted, i = 1, False, m.end()
        while depth:
            c = text[i]
            if c == '"' and text[i - 1] != "\\":
                quoted = not quoted
            depth += 0 if quoted else (c == "(") - (c == ")")
            i += 1
        yield text[m.end():i - 1]


def _written(code):
    """Registers that instructions of `code` have as their first operand, by name."""
    return {w for line in re.split(r"\\n|;", code) for w in re.findall(r"^(?:\\t|\s)*[sv]_\w+\s+(m0|vcc|scc|exec|[sva]\d+)\b", line)}


def _clobbers(statement):
    code = "".join(re.findall(r'"((?:[^"\\]|\\.)*)"', re.split(r':(?=(?:[^"]*"[^"]*")*[^"]*$)', statement)[0]))
    parts = re.split(r':(?=(?:[^"]*"[^"]*")*[^"]*$)', statement.replace("::", ": :"))
    return code, set(re.findall(r'"(\w+)"', parts[3])) if len(parts) > 3 else set()


def test_the_reading_of_statements():
    code, clobbers = _clobbers('"s_mov_b32 m0, %0\\n\\ts_nop 0" ::"s"(to) : "memory", "m0"')
    assert _written(code) == {"m0"} and clobbers == {"memory", "m0"}
    code, clobbers = _clobbers('"v_mov_b32 %0, %1" : "=v"(high) : "i"(f(x))')
    assert not _written(code) and not clobbers


def test_registers_written_by_name_are_clobbers():
    seen = 0
    for path in sorted(glob.glob(os.path.join(ROOT, "paper_2305_06942_amd", "csrc", "*"))):
        with open(path) as f:
            for statement in _statements(f.read()):
                code, clobbers = _clobbers(statement)
                seen += 1
                assert _written(code) <= clobbers, f"{os.path.basename(path)}: {statement}"
    assert seen > 5
