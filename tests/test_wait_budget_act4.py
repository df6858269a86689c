"""Host-side replay of the 4-bit tiles' pipeline (csrc/sq_act4.hip): the counted waits
over a wave's copies, the ring of code buffers and the sets of scales, for every
tile that is launched.  Barrier s publishes stage s; checked for each:

  (a) every copy of stage s and the scales of its pair have completed under the wait
      before barrier s (a wait for n completes all but the n youngest);
  (b) the buffer that a copy fills holds no stage, and the set no pair, that is read
      behind the barrier that precedes the copy (reads of stage s begin behind barrier s
      and have ended at barrier s + 1);
  (c) the counts fit the counter of the wait instruction."""

import os
import re

import pytest

from conftest import ROOT

SOURCE = os.path.join(ROOT, "paper_2609_04526_amd", "csrc", "sq_act4.hip")


def text():
    with open(SOURCE) as f:
        return f.read()


def launched():
    """(BM, BT, STAGES) of every tile that the dispatch names."""
    return sorted({(int(m), int(t), int(s)) for m, t, s in re.findall(r"tile_go<(\d+), (\d+), \d+, \d+, (\d+)>\(", text())})


def replay(BM, BT, ST, steps, slack=0):
    dma = BM // 64 + BT // 64
    lead, sets = (1 if ST == 3 else ST // 2), (2 if ST <= 3 else 4)
    ahead, first = (ST - 2) * dma, dma // 2
    queue, buffers, held = [], {}, {}

    def codes(stage, lo, hi, barrier):
        old = buffers.get(stage % ST, stage)
        assert old in (stage, stage - ST) and (old == stage or old + 1 <= barrier), (stage, old, barrier)     # (b)
        buffers[stage % ST] = stage
        queue.extend(("codes", stage, n) for n in range(lo, hi))

    def scales(pair, barrier):
        old = held.get(pair % sets)
        assert old is None or 2 * old + 2 <= barrier, (pair, old, barrier)                                    # (b)
        held[pair % sets] = pair
        queue.append(("scales", pair, 0))

    def publish(stage, keep):
        assert keep <= 63                                                                                     # (c)
        done = queue[:len(queue) - keep - slack]
        assert [v for v in done if v[:2] == ("codes", stage)] == [("codes", stage, n) for n in range(dma)]    # (a)
        assert ("scales", stage // 2, 0) in done
        assert buffers[stage % ST] == stage and held[stage // 2 % sets] == stage // 2

    scales(0, -1)
    for s in range(ST - 1):
        codes(s, 0, dma, -1)
        if s % 2 == 1 and s // 2 + 1 < lead:
            scales(s // 2 + 1, -1)
    codes(ST - 1, 0, first, -1)
    publish(0, ahead + first + lead - 1)
    for kt in range(steps):
        codes(kt + ST - 1, first, dma, kt)
        if kt % 2 == 0:
            scales(kt // 2 + lead, kt)
        publish(kt + 1, ahead + lead - kt % 2)
        codes(kt + ST, 0, first, kt + 1)


@pytest.mark.parametrize("tile", launched(), ids=str)
def test_ring_and_sets(tile):
    BM, BT, ST = tile
    replay(BM, BT, ST, 40)
    sets = 2 if ST <= 3 else 4
    assert ST * (BM + BT) * 128 + sets * (BM + BT) * 16 <= 160 * 1024


@pytest.mark.parametrize("tile", launched(), ids=str)
def test_one_copy_more_in_flight_would_show(tile):
    with pytest.raises(AssertionError):
        replay(*tile, 40, slack=1)


def test_model_follows_the_kernel_source():
    """The copies, waits and barriers that the replay assumes, in their order."""
    src = text()
    body = src[src.index("void act4_tile("):src.index("// 32 x 32 result")]
    for line in ("kAhead = (STAGES - 2) * kDma;", "kLead = STAGES == 3 ? 1 : STAGES / 2, kSets = STAGES <= 3 ? 2 : 4;",
                 "kFirst = kDma / 2, kSecond = kDma - kFirst;", "kInstA = BM / 64, kInstB = BT / 64, kDma = kInstA + kInstB;"):
        assert line in body
    seq = re.findall(r"dma_scales\([^;]*\);|dma_all\(S, [^;]*\);|dma_first\([^;]*\);|wait_vm_lgkm0<[^;]*>\(\)|s_barrier\(\)|dma\(SP?\{?\}?, kt \+ [^,]*,", body[body.index("auto step ="):])
    assert seq == ["dma(SP{}, kt + STAGES - 1,", "dma_scales((kt >> 1) + kLead);", "wait_vm_lgkm0<kAhead + kLead - v>()", "s_barrier()",
                   "dma(S, kt + STAGES,", "dma_scales(0);", "dma_all(S, decltype(S)::value);", "dma_scales(decltype(S)::value / 2 + 1);",
                   "dma_first(std::integral_constant<int, STAGES - 1>{}, STAGES - 1);", "wait_vm_lgkm0<kAhead + kFirst + kLead - 1>()",
                   "s_barrier()", "wait_vm_lgkm0<0>()"]
    assert "decltype(S)::value % 2 == 1 && decltype(S)::value / 2 + 1 < kLead" in body
    assert "kk == 0 && v == 0 && decltype(N)::value == kProducts - 1) dma_scales" in body
