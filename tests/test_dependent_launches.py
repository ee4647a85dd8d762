"""Kernels that may begin before the launch ahead of them has ended (programmatic dependent launches) do not read
as read-only data what that launch writes: such loads need not wait where the kernel does."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_21653_gb300", "csrc")
READ_ONLY = re.compile(r"__ldg\(|ld\.global\.nc")
# the weights, and x of the first product, whose launch begins after all before it
ALLOWED = {"ffn_rows.cu": ['asm volatile("ld.global.nc.L1::no_allocate.v4.u32', "return kGlu ? __ldg(q) : __ldcg(q);"]}


def test_no_read_only_loads_of_an_earlier_launch():
    found = 0
    for name in sorted(os.listdir(CSRC)):
        with open(os.path.join(CSRC, name)) as f:
            text = f.read()
        if "ProgrammaticStreamSerialization" not in text:
            continue
        found += 1
        for line in text.splitlines():
            if READ_ONLY.search(line):
                assert any(a in line for a in ALLOWED.get(name, [])), (name, line.strip())
    assert found >= 2
