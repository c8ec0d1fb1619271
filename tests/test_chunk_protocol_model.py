"""Randomised model of how the chunk-attention kernel's cp.async loaders hand over a tile and its key mask
(csrc/pad_chunk_tc.cu, bf16 pages of four tokens).

Four loader warps each write a word of a tile's key mask with an ordinary store, start their rows' copies and arrive
on the K barrier; the S issuer waits for it and starts S, whose completion lets the softmax warps read the mask.  A
cp.async arrival comes when the thread's copies are done and orders nothing else that the thread wrote: in the model an
ordinary store is visible to others only after an ordinary (releasing) arrival of its warp that the reader's wait has
seen.  The barrier's count and the arrivals are those of the source.  Checked under random interleavings: every mask
word read is published and its tile's, no slot of the ring of masks is written while a tile that is still read has
it, no K or V stage is refilled while read, and nothing deadlocks.
"""
import os
import random
import re

import pytest

SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_02963_gb300", "csrc",
                      "pad_chunk_tc.cu")


def source_facts():
    """The K barrier's count without TMA and 8-bit tiles, the slots for masks, and whether a loader warp arrives
    on it by an ordinary arrival after its mask word."""
    text = open(SOURCE).read()
    expr = re.search(r"mbar_init\(&bars->kfull\[s\], (.*?)\);", text).group(1)
    count = int(re.sub(r"\w+ \? \d+ : ", "", expr))
    loop = text[text.index("} else if (!wide) {"):text.index("} else if constexpr (FP8) {")]
    loop = loop[:loop.index("vt = ")]  # K's part
    releases = bool(re.search(r"note\(t\);.*if \(lane == 0\) mbar_arrive\(&bars->kfull\[ks\]\);.*mbar_arrive_copies", loop, re.S))
    return count, int(re.search(r"kMasks = (\d+);", text).group(1)), releases


class Bar:
    def __init__(s, count):
        s.count, s.pending, s.done = count, 0, 0
        s.seen, s.published = set(), set()  # stores released by the arrivals of this phase; by completed phases

    def arrive(s, n=1, stores=()):
        s.pending += n
        s.seen |= set(stores)
        assert s.pending <= s.count, "an arrival of the next phase before this one is complete"
        if s.pending == s.count:
            s.pending, s.done = 0, s.done + 1
            s.published |= s.seen

    def ready(s, parity):
        return (s.done % 2) != parity


def run(n, seed, split, stages, count, masks, releases):
    rnd = random.Random(seed)
    ks, vs = stages
    kfull, kfree = [Bar(count) for _ in range(ks)], [Bar(1) for _ in range(ks)]
    vfull, vfree = [Bar(128) for _ in range(vs)], [Bar(1) for _ in range(vs)]
    sfull, pdone, pvdone = [Bar(1), Bar(1)], [Bar(4), Bar(4)], [Bar(1), Bar(1)]
    mask = [[None] * 4 for _ in range(masks)]
    kst, vst = [[None] * 4 for _ in range(ks)], [[None] * 4 for _ in range(vs)]
    visible = {0: set(), 1: set()}       # mask stores that the softmax of a slot may rely on
    k_published = set()
    reading = {}                         # tile -> softmax warps that have not read its mask yet
    inflight, now = [], [0]

    def later(fn, of=None):
        """of: an issuer, whose operations complete in order (a commit covers all of its MMAs so far)."""
        at = max([now[0]] + [op[0] for op in inflight if of is not None and op[2] == of]) + rnd.randint(1, 30)
        inflight.append((at, fn, of))

    def slots(t):
        return [t & 1] if split else [0, 1]

    def nth(t):
        return t >> 1 if split else t

    def readers(t):
        return {(g, w) for g in slots(t) for w in range(4)}

    def loader(w):
        for t in range(n):
            s, u = t % ks, t // ks
            if u > 0:
                yield kfree[s], (u - 1) & 1
            assert not reading.get(t - masks), f"mask of tile {t} written over that of {t - masks}, still read"
            mask[t % masks][w] = t
            kst[s][w] = None

            def landed(t=t, s=s):
                kst[s][w] = t
                kfull[s].arrive(32)
            if releases:
                kfull[s].arrive(1, {(t, w)})
            later(landed)
            s, u = t % vs, t // vs
            if u > 0:
                yield vfree[s], (u - 1) & 1
            vst[s][w] = None

            def v_landed(t=t, s=s):
                vst[s][w] = t
                vfull[s].arrive(32)
            later(v_landed)
            yield None

    def s_issuer():
        for t in range(n):
            s = t % ks
            yield kfull[s], (t // ks) & 1
            k_published.update(kfull[s].published)
            for g in slots(t):
                if nth(t) > 0:
                    yield pvdone[g], (nth(t) - 1) & 1
                assert kst[s] == [t] * 4, f"S({t}) reads a K stage that does not hold it"
                reading.setdefault(t, set()).update((g, w) for w in range(4))

                def done(t=t, s=s, g=g, seen=frozenset(k_published)):
                    assert kst[s] == [t] * 4, f"K stage of tile {t} refilled under S"
                    visible[g].update(seen)
                    sfull[g].arrive()
                    if split or g == 1:
                        kfree[s].arrive()
                later(done, "S")
                yield None

    def pv_issuer():
        for t in range(n):
            s = t % vs
            yield vfull[s], (t // vs) & 1
            for g in slots(t):
                yield pdone[g], nth(t) & 1
                assert vst[s] == [t] * 4, f"P.V({t}) reads a V stage that does not hold it"

                def done(t=t, s=s, g=g):
                    assert vst[s] == [t] * 4, f"V stage of tile {t} refilled under P.V"
                    pvdone[g].arrive()
                    if split or g == 1:
                        vfree[s].arrive()
                later(done, "PV")
                yield None

    def softmax(g, w):
        for t in range(g if split else 0, n, 2 if split else 1):
            yield sfull[g], nth(t) & 1
            for _ in range(rnd.choice([0, 3, 60])):
                yield None
            assert mask[t % masks] == [t] * 4, f"mask of tile {t} read as that of {mask[t % masks]}"
            assert all((t, u) in visible[g] for u in range(4)), f"mask of tile {t} read before it is published"
            reading[t].discard((g, w))
            pdone[g].arrive()

    actors = [loader(w) for w in range(4)] + [s_issuer(), pv_issuer()] + [softmax(g, w) for g in range(2) for w in range(4)]
    waiting, alive = [None] * len(actors), [True] * len(actors)
    while any(alive):
        now[0] += 1
        assert now[0] < 200000, "no progress"
        for op in [op for op in inflight if op[0] <= now[0]]:
            inflight.remove(op)
            op[1]()
        order, progressed = list(range(len(actors))), False
        rnd.shuffle(order)
        for i in order:
            if not alive[i] or (waiting[i] is not None and not waiting[i][0].ready(waiting[i][1])):
                continue
            waiting[i] = None
            if rnd.random() < 0.5:
                progressed = True
                continue
            try:
                waiting[i] = next(actors[i])
            except StopIteration:
                alive[i] = False
            progressed = True
        assert progressed or inflight or not any(alive), "deadlock"


FORMS = [(split, stages) for split in (False, True) for stages in ((3, 2), (4, 4))]


@pytest.mark.parametrize("split,stages", FORMS)
def test_a_tiles_mask_is_published_with_its_keys(split, stages):
    count, masks, releases = source_facts()
    for n in range(1, 14):
        for seed in range(12):
            run(n, 131 * seed + n, split, stages, count, masks, releases)


def fails(**kw):
    a = dict(count=132, masks=8, releases=True) | kw
    bad = 0
    for split, stages in FORMS:
        for n in range(1, 14):
            for seed in range(4):
                try:
                    run(n, 17 * seed + n, split, stages, **a)
                except AssertionError:
                    bad += 1
    return bad


def test_the_model_detects_planted_mistakes():
    assert fails() == 0
    assert fails(count=128, releases=False) > 0  # the copies' arrivals alone
    assert fails(count=128) > 0                  # an arrival more than the barrier counts
    assert fails(releases=False) > 0             # one less
    assert fails(masks=2) > 0
