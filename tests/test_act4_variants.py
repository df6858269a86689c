"""The products of two 4-bit operands that the library holds are those that a call
can reach (no GPU needed: the kernels' names as the library registers them).

The few rows' kernel takes 16, 32 or 64 outputs by 16 rows to a workgroup, by what
leaves a workgroup for every compute unit; more than 16 rows only of one layer of up
to 4096 outputs, whose 64-output groups are fewer than those a wider one needs, so
only with 16 outputs."""

import re

from conftest import ensure_library


def _names():
    ensure_library()
    from paper_2609_04526_amd import sq
    with open(sq.LIB_PATH, "rb") as f:
        return f.read()


def test_every_kernel_of_few_rows_is_reachable():
    have = {tuple(map(int, m)) for m in re.findall(rb"act4_thin_kernelILi(\d)ELi(\d)ELb(\d)ELb(\d)E", _names())}
    want = {(rm, nt, words, bf16) for rm, nt in ((1, 1), (2, 1), (4, 1), (1, 2), (1, 4)) for words in (0, 1) for bf16 in (0, 1)}
    assert have == want


def test_every_tile_is_reachable():
    names = _names()
    tiles = {tuple(map(int, m)) for m in re.findall(rb"act4_tile_kernelILi(\d+)ELi(\d+)ELi\dELi\dELi(\d)ELb(\d)E", names)}
    assert tiles == {(bm, bt, st, b) for bm, bt, st in ((128, 64, 6), (128, 128, 4), (256, 64, 3), (256, 128, 3), (256, 256, 2)) for b in (0, 1)}
    tables = {tuple(map(int, m)) for m in re.findall(rb"act4_experts_kernelILi(\d+)ELb(\d)E", names)}
    assert tables == {(bt, b) for bt in (64, 128, 256) for b in (0, 1)}
