"""Where the attention kernels fill a place of an LDS ring again without a barrier, a wave by itself,
the source orders its LDS reads of that place before the DMAs: a wait for them stands directly ahead
of the DMAs.  A build without it may still happen to wait, so this reads the source."""
import os
import re

from paper_2606_18394_amd import build

WAIT = r'asm volatile\("s_waitcnt lgkmcnt\(0\)" ::: "memory"\);'


def source(name):
    with open(os.path.join(build.CSRC, name)) as f:
        return re.sub(r"//[^\n]*", "", f.read())


def test_8_bit_ring():
    body = source("tv_attention_fp8.hip")
    refill = re.search(r"auto refill = \[&\]\(\) \{(.*?)\n  \};", body, re.S).group(1)
    assert re.match(rf"\s*if \(kAlone\) {WAIT}", refill)
    # units are issued there and, into an empty ring, by the prologue
    assert len(re.findall(r"issue_unit\((?!int)", body)) == 2 and "issue_unit(issued)" in refill


def test_16_bit_ring():
    body = source("tv_attention.hip")
    step = re.search(r"auto ring_step = \[&\]\(int i\) \{(.*?)\n  \};", body, re.S).group(1)
    shared, alone = re.split(r"\} else \{", step)
    assert "__syncthreads();" in shared.partition("issue_tile")[0]
    assert re.match(rf"\s*{WAIT}", alone) and "issue_tile" in alone
