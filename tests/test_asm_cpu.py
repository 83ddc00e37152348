"""Inline assembly in the kernels leaves fixed registers as the compiler expects them: it names those that it writes as
clobbered, and keeps m0, which the compiler takes for reserved and does not heed there (read from the sources: no GPU needed)."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2605_18825_amd", "csrc")
SOURCES = sorted(glob.glob(os.path.join(CSRC, "*.h")) + glob.glob(os.path.join(CSRC, "*.hip")))
# registers that an instruction writes as its first operand, without an operand of the statement standing for them
WRITTEN = re.compile(r"^[a-z_0-9]+ +(m0|vcc|vcc_lo|vcc_hi|exec|scc)\s*,")


def statements(text):
    """(instructions, clobbers) of every asm statement."""
    text = re.sub(r"//[^\n]*", "", text)
    for m in re.finditer(r"\basm\s+(?:volatile\s*)?\((.*?)\)\s*;", text, re.S):
        strings = [(s.start(), s.group(1)) for s in re.finditer(r'"((?:[^"\\]|\\.)*)"', m.group(1))]
        bare = re.sub(r'"(?:[^"\\]|\\.)*"', lambda s: "_" * len(s.group(0)), m.group(1))
        colons = [i for i, ch in enumerate(bare) if ch == ":"]
        end = colons[0] if colons else len(bare)
        last = colons[2] if len(colons) > 2 else len(bare)
        template = "".join(s for at, s in strings if at < end).replace("\\n", "\n").replace("\\t", " ")
        yield [line.strip() for line in template.split("\n") if line.strip()], {s for at, s in strings if at > last}


def wrong(instructions, clobbers):
    """The registers that a statement writes unasked."""
    bad = {m.group(1) for m in map(WRITTEN.match, instructions) if m and m.group(1) not in clobbers}
    if any(WRITTEN.match(i) and WRITTEN.match(i).group(1) == "m0" for i in instructions):
        kept = re.fullmatch(r"s_mov_b32 (%\d), m0", instructions[0])
        bad -= {"m0"}
        if not kept or instructions[-1] != "s_mov_b32 m0, " + kept.group(1):
            bad |= {"m0"}
    return bad


def test_the_reader():
    one, = statements('asm volatile("s_mov_b32 m0, %0\\n\\t" "x %1" : : "s"(at), "v"(from) : "m0", "memory");')
    assert one == (["s_mov_b32 m0, %0", "x %1"], {"m0", "memory"}) and wrong(*one) == {"m0"}
    one, = statements('asm volatile("s_mov_b32 %0, m0\\n\\ts_mov_b32 m0, %1\\n\\tx %2\\n\\ts_mov_b32 m0, %0" : "=&s"(h) : "s"(a) : "memory");')
    assert not wrong(*one)
    one, = statements('asm volatile("v_cmp_eq_u32 vcc, %0, 0" : : "v"(a));')
    assert wrong(*one) == {"vcc"}
    assert list(statements('asm volatile("");')) == [([], set())]


@pytest.mark.parametrize("path", SOURCES, ids=os.path.basename)
def test_fixed_registers_are_kept_or_named(path):
    with open(path) as f:
        for one in statements(f.read()):
            assert not wrong(*one), one
