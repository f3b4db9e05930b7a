"""Inline assembly of the kernels, without a GPU: what the compiler has to know about it."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2603_14303_amd", "csrc")


def blocks():
    """(file, assembly text, constraints) of every asm statement."""
    for name in sorted(os.listdir(CSRC)):
        with open(os.path.join(CSRC, name)) as f:
            source = f.read()
        for m in re.finditer(r'asm volatile\(\s*((?:"(?:[^"\\]|\\.)*"\s*)+)(.*?)\);', source, re.S):
            yield name, "".join(re.findall(r'"((?:[^"\\]|\\.)*)"', m.group(1))).replace("\\n", "\n").replace("\\t", ""), m.group(2)


def test_m0_is_the_compilers():
    """It has uses of m0 of its own: it is an operand, so that the compiler writes it and knows what it holds."""
    found = 0
    for name, text, constraints in blocks():
        lines = [x.strip() for x in text.split("\n")]
        assert not any(re.match(r"\S+\s+m0\b", x) for x in lines), (name, text)
        if any(x.endswith(" lds") for x in lines):
            found += 1
            assert '"{m0}"' in constraints, (name, text)
    assert found


def test_a_loads_descriptor_is_settled():
    """A vector instruction (v_readfirstlane) that writes a scalar register needs five wait states before a memory instruction reads it.  The compiler does not look into the text: it waits by itself."""
    found = 0
    for name, text, _ in blocks():
        lines = [x.strip() for x in text.split("\n")]
        for i, line in enumerate(lines):
            if line.startswith("buffer_"):
                found += 1
                states = sum(int(x.split()[1]) + 1 if x.startswith("s_nop") else 1 for x in lines[:i])
                assert states >= 5, (name, text)
    assert found
