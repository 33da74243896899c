"""Inline assembly of the kernels: what it changes is named to the compiler."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1910_00178_amd", "csrc")


def asm_statements():
    for path in sorted(glob.glob(os.path.join(CSRC, "*.h")) + glob.glob(os.path.join(CSRC, "*.hip"))):
        text = re.sub(r"//[^\n]*", "", open(path).read())
        for m in re.finditer(r"\basm\b\s*(?:volatile)?\s*\(", text):
            depth, quoted, at = 1, False, m.end()
            while depth:
                c = text[at]
                if c == '"' and text[at - 1] != "\\":
                    quoted = not quoted
                depth += 0 if quoted else (c == "(") - (c == ")")
                at += 1
            yield os.path.basename(path), text[m.end():at - 1]


def test_registers_written_by_name_are_clobbers():
    """An instruction that writes M0 (or another register by its name) says so: else the compiler may keep a value of its own there."""
    seen = 0
    for path, statement in asm_statements():
        strings = re.findall(r'"((?:[^"\\]|\\.)*)"', statement)
        code = strings[0].replace("\\n", "\n").replace("\\t", " ")
        for line in re.split(r"[\n;]", code):
            words = re.findall(r"[\w%\[\]:]+", line)
            if len(words) > 1 and re.fullmatch(r"m0|vcc(_lo|_hi)?|exec(_lo|_hi)?|scc|[sv]\d+", words[1]) and not words[0].startswith(("s_cmp", "s_setreg")):
                seen += 1
                assert words[1] in strings[1:], f"{path}: {line.strip()} without the clobber {words[1]}"
    assert seen >= 1
