"""Reads in inline assembly of the decoding kernels: the compiler takes an asm's results as written when it ends, so a
read's wait stands in the same asm; loads that go straight to LDS have no results."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2404_02445_amd", "csrc")


def asm_blocks(text):
    """(template, operands) of every asm statement."""
    for m in re.finditer(r"\basm\s+volatile\s*\(", text):
        depth, i, quoted = 1, m.end(), False
        while depth:
            c = text[i]
            if quoted:
                i += c == "\\"
                quoted = c != '"'
            elif c == '"':
                quoted = True
            else:
                depth += (c == "(") - (c == ")")
            i += 1
        body = text[m.end():i - 1]
        template = re.match(r'\s*((?:"(?:[^"\\]|\\.)*"\s*)+)', body)
        yield "".join(re.findall(r'"((?:[^"\\]|\\.)*)"', template[1])).replace("\\n", "\n").replace("\\t", ""), body[template.end():]


def faults(text):
    found = []
    for template, operands in asm_blocks(text):
        lines = [x.strip() for x in template.split("\n") if x.strip()]
        results = operands.split(":")[1] if operands.startswith(":") else ""
        waiting = False
        for x in lines:
            if re.match(r"(ds_read|ds_load)", x):
                waiting = True
            elif re.match(r"(buffer|global|flat|scratch|s_buffer|s)_load", x):
                waiting = waiting or not re.search(r"\blds\b|_lds_", x)
                if not waiting and "=" in results:
                    found.append(template)
            elif x.startswith("s_waitcnt") and re.search(r"(lgkm|vm)cnt\(0\)", x):
                waiting = False
        if waiting:
            found.append(template)
    return found


def test_the_check_sees_what_it_is_for():
    assert faults('asm volatile("ds_read_b128 %0, %1" : "=v"(v) : "v"(a));')
    assert faults('asm volatile("s_waitcnt lgkmcnt(0)\\n\\tds_read_b32 %0, %1" : "=v"(v) : "v"(a));')
    assert faults('asm volatile("global_load_dword %0, %1, off" : "=v"(v) : "v"(a));')
    assert not faults('asm volatile("ds_read_b32 %0, %1\\n\\t" "s_waitcnt lgkmcnt(0)" : "=v"(v) : "v"(a) : "memory");')
    assert not faults('asm volatile("s_mov_b32 m0, %0\\n\\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(d), "v"(o), "s"(r) : "memory");')
    assert not faults('asm volatile("" : "+v"(v)); asm volatile("s_waitcnt vmcnt(0)" ::: "memory");')


@pytest.mark.parametrize("name", ["attention.hip", "rotary.hip"])
def test_no_read_outlives_its_asm(name):
    with open(os.path.join(CSRC, name)) as f:
        text = f.read()
    assert faults(text) == []
