"""The tile products of the loss that the library holds are those that a call can
reach (no GPU needed: the kernels' names as the library registers them).

Logits that pass through memory (mode 3) are formed where twice the tiles do not
exceed the compute units, in as many splits as go into them: so never in more
workgroups than compute units, for which 64-token tiles have three stages, and
never of more tokens, since few tiles cost the least with 64."""

import re

from conftest import ensure_library

STATS, GRAD, DX, LOGITS = range(4)


def test_every_tile_product_is_reachable():
    ensure_library()
    from paper_2609_04526_amd import sq
    with open(sq.LIB_PATH, "rb") as f:
        names = set(re.findall(rb"ce_kernelILi(\d)ELi(\d+)ELi(\d+)ELi\dELi\dELi(\d)ELb(\d)E", f.read()))
    have = {(int(m), int(bm), int(bn), int(st), int(c)) for m, bm, bn, st, c in names}
    want = {(LOGITS, 256, 64, 3, 0)} | {(m, 256, bn, st, 0) for m in (STATS, GRAD) for bn, st in ((64, 2), (64, 3), (128, 3), (256, 2))}
    want |= {(m, 256, bn, 3, 1) for m in (STATS, GRAD) for bn in (64, 128, 256)}
    want |= {(DX, 64, 256, 3, 0), (DX, 128, 256, 3, 0), (DX, 256, 256, 2, 0)}
    want |= {(DX, bm, 256, 2, 1) for bm in (64, 128, 256)}
    assert have == want
