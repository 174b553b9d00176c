"""Waits that hand-written assembly has to bring itself: the compiler puts them between its own instructions, but not
inside an asm statement."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2606_10520_amd", "csrc")
SOURCES = sorted(glob.glob(os.path.join(CSRC, "*.h*")))


def asm_statements(text):
    """The instructions of every asm statement of a source."""
    for m in re.finditer(r"\basm\b(?:\s+volatile)?\s*\(((?:\s*\"(?:[^\"\\]|\\.)*\")+)", text):
        joined = "".join(re.findall(r"\"((?:[^\"\\]|\\.)*)\"", m.group(1)))
        yield [i.strip() for i in re.split(r"(?:\\n|\\t|;)+", joined) if i.strip()]


def states(instruction):
    """Wait states that an instruction takes: s_nop n takes n + 1."""
    m = re.match(r"s_nop\s+(\d+)", instruction)
    return int(m.group(1)) + 1 if m else 1


def missing_waits(text):
    """Loads that go to LDS by M0 with no wait state after the write of M0, or less than five after the statement's
    start (before it a vector instruction may have written the scalar registers that they read)."""
    bad = []
    for block in asm_statements(text):
        since_m0, since_start = None, 0
        for i in block:
            if re.match(r"(buffer|global|scratch)_load", i) and re.search(r"\blds\b|_lds_", i):
                if since_m0 is None or since_m0 < 1 or since_start < 5:
                    bad.append(i)
            if since_m0 is not None:
                since_m0 += states(i)
            since_start += states(i)
            if re.match(r"s_\w+\s+m0\b", i):
                since_m0 = 0
    return bad


def test_the_scan_sees_missing_waits():
    def source(s):
        return 'asm volatile("%s" ::"s"(to));' % s
    load = "buffer_load_dwordx4 %1, %2, 0 offen lds"
    assert missing_waits(source("s_mov_b32 m0, %0\\n\\t" + load)) == [load]
    assert missing_waits(source("s_mov_b32 m0, %0\\n\\ts_nop 0\\n\\t" + load)) == [load]  # too near the start
    assert missing_waits(source("s_mov_b32 m0, %0\\n\\ts_nop 3\\n\\t" + load)) == []
    assert missing_waits(source("s_nop 3\\n\\ts_mov_b32 m0, %0\\n\\t" + load)) == [load]


@pytest.mark.parametrize("path", SOURCES, ids=os.path.basename)
def test_loads_to_lds_wait_for_their_address(path):
    with open(path) as f:
        assert missing_waits(f.read()) == []


def test_there_are_such_loads():
    with open(os.path.join(CSRC, "attn_prompt.hip")) as f:
        assert sum(i.endswith(" lds") for block in asm_statements(f.read()) for i in block) == 6
