"""Every inline instruction that reads, writes or orders shared or global memory that C++ code writes too tells the compiler so:
without a "memory" clobber a plain store may be moved past it.  Streaming loads of constant data (ld.global.nc) need none."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2302_07475_b200", "csrc")
TOUCHES = re.compile(r"\b(ld\.|st\.|red\.|atom\.|multimem\.|cp\.async|mbarrier\.|fence\.|bar\.|barrier\.|tcgen05\.(mma|commit|alloc|fence|wait))")


def statements(text):
    for m in re.finditer(r"\basm\b(\s+volatile)?\s*\(", text):
        depth, at, quoted = 1, m.end(), False
        while depth:
            c = text[at]
            if c == '"' and text[at - 1] != "\\":
                quoted = not quoted
            elif not quoted:
                depth += (c == "(") - (c == ")")
            at += 1
        yield text.count("\n", 0, m.start()) + 1, text[m.start():at]


def lacking(text):
    found = []
    for line, statement in statements(text):
        code = "".join(re.findall(r'"((?:[^"\\]|\\.)*)"', statement)).replace("\\n", " ").replace("\\t", " ")
        if TOUCHES.search(re.sub(r"\b(ld\.global\.nc|tcgen05\.ld)\S*", "", code)) and '"memory"' not in statement:
            found.append(line)
    return found


def test_the_rule_itself():
    assert lacking('asm volatile("ld.shared.f32 %0, [%1];" : "=f"(x) : "r"(p));') == [1]
    assert not lacking('asm volatile("ld.shared.f32 %0, [%1];" : "=f"(x) : "r"(p) : "memory");')
    assert not lacking('asm("mov.u32 %0, %%lanemask_lt;" : "=r"(m));\nasm volatile("ld.global.nc.v2.u32 {%0,%1}, [%2];" : "=r"(a), "=r"(b) : "l"(p));')


@pytest.mark.parametrize("path", sorted(glob.glob(os.path.join(CSRC, "*.cu*")) + glob.glob(os.path.join(CSRC, "*.inl"))), ids=os.path.basename)
def test_inline_memory_instructions_are_ordered(path):
    with open(path) as f:
        assert lacking(f.read()) == []
