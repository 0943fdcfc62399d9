"""Registers that inline assembly names by itself, and not through an operand, are in its list of what it overwrites:
the compiler would otherwise keep values of its own there.  Read from the sources, without a GPU."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2110_09132_amd", "csrc")
NAMED = re.compile(r"\b(m0|vcc|exec|[sv]\d+|[sv]\[\d+:\d+\])\b")


def statements(text):
    """(the instructions, what stands behind the third colon) of every asm statement."""
    for m in re.finditer(r"\basm\s+volatile\s*\(", text):
        depth, at, quoted = 1, m.end(), False
        while depth:
            c = text[at]
            if c == '"' and text[at - 1] != "\\":
                quoted = not quoted
            elif not quoted:
                depth += (c == "(") - (c == ")")
            at += 1
        body = text[m.end():at - 1]
        parts, strings = [""], re.split(r'("(?:[^"\\]|\\.)*")', body)
        for s in strings:
            if s.startswith('"'):
                parts[-1] += s
            else:
                first, *more = s.split(":")
                parts[-1] += first
                parts += more
        yield parts[0], parts[3] if len(parts) > 3 else ""


def written(instructions):
    """Registers in the first place of an instruction that has a destination there."""
    for line in re.sub(r'"\s*"', "", instructions).strip().strip('"').split("\\n"):
        words = line.replace("\\t", " ").split(None, 1)
        if len(words) == 2 and not words[0].startswith(("s_waitcnt", "s_nop", "s_sleep", "global_store", "buffer_store")):
            yield from NAMED.findall(words[1].split(",")[0])


def test_written_registers_are_listed():
    seen = 0
    for path in sorted(glob.glob(os.path.join(CSRC, "*.h*"))):
        with open(path) as f:
            for instructions, clobbers in statements(f.read()):
                seen += 1
                for register in written(instructions):
                    assert f'"{register}"' in clobbers, f"{os.path.basename(path)}: {instructions.strip()}"
    assert seen >= 5
