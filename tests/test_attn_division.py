"""The division of an attention call's work among its workgroups, and the arrival counters with which the parts of a shared item are
joined: restated in whole numbers, with the constants, and where an arrival is counted, read from the source.  Every step of every item is
taken once, parts have places of their own, and a counter belongs to one item.  Needs no GPU."""
import collections
import os
import random
import re

import pytest

from paper_2410_11305_amd import build

SOURCE = re.sub(r"//.*", "", open(os.path.join(build.HERE, "csrc", "attn_kv4.hpp")).read())
WAVES = 4


def constant(name, NB, F):
    """A static constant of an instance's shape."""
    text = re.search(r"static constexpr int %s = ([^;]*);" % name, SOURCE).group(1)
    text = re.sub(r"NB == 1 \? (\d+) : NB == 2 \? (\d+) : (\d+)", r"{1: \1, 2: \2}.get(NB, \3)", text)
    text = re.sub(r"F > 1 \? (\d+) : (\d+)", r"(\1 if F > 1 else \2)", text).replace("/", "//")
    return eval(text, {}, dict(NB=NB, F=F, **{n: constant(n, NB, F) for n in ("tiles", "step") if n in text and n != name}))


def instance(rows):
    return (1, 4) if rows <= 4 else (1, 2) if rows <= 8 else (1, 1) if rows <= 16 else (2, 1) if rows <= 32 else (4, 1)


def counted(n, stage):
    """Whether a workgroup of a set of n takes part in an arrival in this stage: what stands in front of last_arrival in the loop over the stages."""
    loop = SOURCE[SOURCE.index("for (int stage"):]
    loop = loop[:loop.index("last_arrival(")]
    skip = re.search(r"if \(([^;{}]*)\) continue;", loop)
    return not (skip and eval(skip.group(1).replace("&&", "and"), {}, dict(n=n, stage=stage)))


def span(pos, T, G, block, rows, step, window, sinks, end_of_cache):
    lo, hi = pos + block * rows // G, pos + (min(T * G, (block + 1) * rows) - 1) // G
    end = min(hi + 1, end_of_cache)
    first = max(lo - window + 1, 0) // step if window else 0
    sink_steps = max(min(-(-min(sinks, end) // step), first), 0) if window else 0
    return max(sink_steps + max(-(-end // step) - first, 0), 1)


def check(T, Hq, Hkv, positions, window=0, sinks=0, end_of_cache=1 << 30):
    """Walks the division of one call; returns the number of parts of the item with the most."""
    G = Hq // Hkv
    NB, F = instance(T * G)
    step, OVER, whole, least, grid, rows = (constant(n, NB, F) for n in ("step", "over", "whole", "least", "workgroups", "rows"))
    blocks = -(-T * G // rows)
    starts, steps, at = [], [], 0                              # of the items, in their order
    for pos in positions:
        for block in range(blocks):
            n = span(pos, T, G, block, rows, step, window, sinks, end_of_cache)
            for _ in range(Hkv):
                starts.append(at)
                steps.append(n)
                at += OVER + n
    total, items = at, len(starts)
    groups = min(grid, max(items, (total - items * OVER) // least))
    share, more = divmod(total, groups)
    start_of = lambda w: w * share + min(w, more)

    def group_of(x):
        wide = more * (share + 1)
        return x // (share + 1) if x < wide else more + (x - wide) // share

    def places():                                              # (item, step) where each workgroup begins
        item = 0
        for w in range(groups + 1):
            x = start_of(w)
            while item < items and starts[item] + OVER + steps[item] <= x:
                item += 1
            if item == items:
                yield items, 0
            else:
                into = x - starts[item]
                yield item, 0 if OVER + steps[item] <= whole + OVER or into < OVER else (into - OVER) & ~(WAVES - 1)

    place = list(places())
    taken, slots = collections.defaultdict(list), {}
    for w in range(groups):
        (item, begin), (last, last_step), first_run = place[w], place[w + 1], True
        while item < last or (item == last and begin < last_step):
            stop = last_step if item == last else steps[item]
            taken[item].append((begin, stop, w))
            if begin > 0 or stop < steps[item]:
                slot = 2 * w + (0 if first_run else 1)
                assert slot not in slots and slot < 2 * grid
                slots[slot] = item
            item, begin, first_run = item + 1, 0, False
    owner, most = {}, 0
    for item in range(items):
        runs = taken[item]
        assert runs[0][0] == 0 and runs[-1][1] == steps[item] and all(a[1] == b[0] for a, b in zip(runs, runs[1:])), item
        if len(runs) == 1:
            continue
        # the workgroups that the kernel takes for the item's, and the places where it looks for their parts
        w0, w1 = group_of(starts[item] + OVER + WAVES - 1), group_of(starts[item] + OVER + steps[item] - 1)
        assert [r[2] for r in runs] == list(range(w0, w1 + 1))
        parts = w1 - w0 + 1
        most = max(most, parts)
        assert all(slots[(2 * w0 + (start_of(w0) < starts[item])) if w == w0 else 2 * w] == item for w in range(w0, w1 + 1))
        counters = [w0]
        if parts > 16:
            for first in range(w0, w1 + 1, 8):
                if counted(min(8, w1 + 1 - first), 0):
                    counters.append(grid + first)
        for c in counters:
            assert c < 2 * grid and owner.setdefault(c, item) == item, (c, item, owner[c])
    return most


def test_the_constants_are_found():
    assert [constant(n, 1, 4) for n in ("tiles", "step", "over", "whole", "least", "workgroups", "rows")] == [4, 64, 16, 16, 8, 512, 4]
    assert [constant(n, 4, 1) for n in ("tiles", "step", "over", "whole", "least", "workgroups", "rows")] == [2, 32, 16, 32, 40, 512, 64]
    assert "OVER = Form::over" in SOURCE and "counter = Form::workgroups + first;" in SOURCE and "uint32_t first = w0, stride = 1, n = parts, counter = w0;" in SOURCE
    assert "int stage = parts > 16 ? 0 : 1; shared && stage < 2;" in SOURCE and "first = w0 + ((me - w0) & ~7u);" in SOURCE
    assert counted(2, 0) and counted(8, 0) and counted(17, 1)


@pytest.mark.parametrize("T,Hq,Hkv", [(1, 8, 1), (1, 32, 32), (4, 32, 32), (1, 64, 8), (4, 64, 8), (8, 8, 1), (16, 32, 16), (2, 40, 8), (1, 7, 1), (3, 5, 5)])
def test_one_sequence_of_any_length(T, Hq, Hkv):
    most = [check(T, Hq, Hkv, [n - T]) for n in list(range(T, 3000, 173)) + list(range(3000, 131072, 1409)) + [20531, 40000, 60000, 100000, 130880, 131008, 131071]]
    assert max(most) > 16


def test_ragged_batches_and_windows():
    rng = random.Random(1)
    most = []
    for _ in range(600):
        Hkv, G, T = rng.choice((1, 2, 4, 8, 32)), rng.choice((1, 2, 7, 8)), rng.choice((1, 1, 2, 4, 9, 40, 300))
        longest = rng.choice((300, 5000, 40000, 130000))
        window = rng.choice((0, 0, 100, 4096, 30000))
        pos = [rng.randint(-T, longest - 1) for _ in range(rng.choice((1, 2, 2, 3, 7, 40)))]
        most.append(check(T, Hkv * G, Hkv, pos, window, rng.choice((0, 4, 5000)) if window else 0, rng.choice((1 << 30, longest // 2 + 16))))
    assert max(most) > 64


# calls in which an item's last set is one workgroup, with which the next item's first set begins: (T, Hq, Hkv, tokens)
NEIGHBOURS = [(1, 32, 32, 20507), (36, 2, 2, 21409), (8, 16, 2, 21122), (33, 3, 3, 20917)]


@pytest.mark.parametrize("T,Hq,Hkv,n", NEIGHBOURS)
def test_the_check_sees_a_counter_of_two_items(monkeypatch, T, Hq, Hkv, n):
    check(T, Hq, Hkv, [n - T])
    monkeypatch.setitem(globals(), "counted", lambda n, stage: True)
    with pytest.raises(AssertionError):
        check(T, Hq, Hkv, [n - T])
