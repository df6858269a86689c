"""The logits' statistics run with 8 waves per SIMD: at most 64 vector registers in
each of their kernels (no GPU needed: the counts in the library's own code objects).
With the registers that their tails ask for where they are left to, a tail makes
the loss of a 4-bit head 2.7% slower."""

import re

from conftest import ensure_library


def _registers(name):
    """vgpr_count of every kernel of the library whose name has `name`, from the code objects' metadata."""
    ensure_library()
    from paper_2609_04526_amd import sq
    with open(sq.LIB_PATH, "rb") as f:
        data = f.read()
    found = {}
    for m in re.finditer(rb"\.symbol.{1,3}?(_Z\w*" + name + rb"\w*)\.kd(.{0,400}?)\.vgpr_count(\xcc.|[\x00-\x7f])", data, re.S):
        found[m.group(1)] = m.group(3)[-1]
    return found


def test_waves_of_the_logits_statistics():
    counts = _registers(b"ce_part_kernel")
    assert len(counts) == 3
    assert max(counts.values()) <= 64, counts
