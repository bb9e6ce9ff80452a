"""Alignment of the kernels' dynamic shared memory, read from the sources.  No GPU is needed."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_23264_b200", "csrc")


def declarations():
    """File, line, declaration and the lines behind it, of every array that its kernel stores to."""
    for path in sorted(glob.glob(os.path.join(CSRC, "*.cu*"))):
        text = open(path).read().split("\n")
        for at, line in enumerate(text):
            found = re.search(r"extern\s+__shared__.*?(\w+)\[\]", line)
            if found and len(re.findall(rf"\b{found[1]}\b", "\n".join(text))) > 1:
                yield os.path.basename(path), at, line.strip(), text[at + 1:at + 6]


DECLARED = list(declarations())


@pytest.mark.parametrize("name,at,line,after", DECLARED, ids=[f"{d[0]}:{d[1] + 1}" for d in DECLARED])
def test_dynamic_shared_memory_begins_on_16_bytes(name, at, line, after):
    """Vectors are stored in all of it.  The declared type's alignment is all that is promised, whatever static arrays happen to lie
    in front: a 16-byte type, an alignment of its own, or an address rounded up by the kernel."""
    aligned = re.search(r"__align__\((\d+)\)", line)
    vector = re.search(r"__shared__\s+(float4|uint4|int4|double2)\b", line)
    rounded = any(re.search(r"1024u - \(\w+ & 1023u\)", text) for text in after)
    assert (aligned and int(aligned[1]) >= 16) or vector or rounded, line
