"""The division of the shared tokens' launch of qspec_attn_kv4_shared, and where the second launch looks for the sums of an item: restated in whole numbers, with the
constants read from the source.  Every step of every group's item is taken once, no part is empty, parts have places of their own, and the directory that an item's first workgroup
writes leads to all of them.  (Nothing counts arrivals here: the second launch reads what the directory says.)  Needs no GPU."""
import collections
import random
import re

import pytest

from tests.test_attn_division import SOURCE, WAVES, constant, instance

ROUNDS = int(re.search(r"constexpr int kAttnRounds = (\d+);", SOURCE).group(1))
GRID = constant("workgroups", 1, 1)                            # (one launch serves all instances)


def least_of(NB, F):
    """What a workgroup gets on average at least, in steps."""
    text = re.search(r"constexpr int LEAST = ([^;]*);", SOURCE).group(1)
    text = re.fullmatch(r"MODE == kAttnWhole \|\| F > 1 \? Form::least : \(NB == 4 \? (\d+) : (\d+)\) / STEP", text)
    return constant("least", NB, F) if F > 1 else int(text.group(1 if NB == 4 else 2)) // constant("step", NB, F)


def steps_of(shared, step, least_shared, end_of_cache):
    n = min(max(shared, 0), end_of_cache)
    n = 0 if n < least_shared else n
    return max(int((n - 1 + step) / step), 1)                  # (towards zero)


def check(rows, Hkv, shared, least_shared=0, end_of_cache=1 << 30, least=None):
    """Walks one launch over groups of so many rows (heads of a key/value head counted); returns the number of parts of the item with the most, and
    of workgroups."""
    NB, F = instance(rows)
    step, OVER, whole, block = (constant(n, NB, F) for n in ("step", "over", "whole", "rows"))
    least = least or least_of(NB, F)
    starts, steps, at = [], [], 0
    for n in shared:
        for _ in range(-(-rows // block)):
            for _ in range(Hkv):
                starts.append(at)
                steps.append(steps_of(n, step, least_shared, end_of_cache))
                at += OVER + steps[-1]
    items = len(starts)
    groups = min(GRID, max(items, (at - items * OVER) // least))
    share, more = divmod(at, groups)
    assert share >= 1
    start_of = lambda w: w * share + min(w, more)

    def group_of(x):
        wide = more * (share + 1)
        return x // (share + 1) if x < wide else more + (x - wide) // share

    place, item = [], 0
    for w in range(groups + 1):
        x = start_of(w)
        while item < items and starts[item] + OVER + steps[item] <= x:
            item += 1
        into = x - starts[item] if item < items else 0
        place.append((item, 0 if item == items or OVER + steps[item] <= whole + OVER or into < OVER else (into - OVER) & ~(WAVES - 1)))
    taken, directory, places = collections.defaultdict(list), {}, {}
    for w in range(groups):
        (item, begin), (last, last_step), first_run = place[w], place[w + 1], True
        while item < last or (item == last and begin < last_step):
            stop = last_step if item == last else steps[item]
            assert begin < stop
            taken[item].append((begin, stop))
            shared_out = begin > 0 or stop < steps[item]
            slot = 2 * w + (0 if first_run else 1)
            if shared_out:
                assert slot not in places and slot < 2 * GRID
                places[slot] = item, len(taken[item]) - 1
            if begin == 0:
                w0, w1 = group_of(starts[item] + OVER + WAVES - 1), group_of(starts[item] + OVER + steps[item] - 1)
                directory[item] = (slot, w1 - w0 + 1) if shared_out else (0, 1)
            item, begin, first_run = item + 1, 0, False
    most = 0
    for item in range(items):
        runs = taken[item]
        assert runs[0][0] == 0 and runs[-1][1] == steps[item] and all(a[1] == b[0] for a, b in zip(runs, runs[1:])), item
        first, parts = directory[item]
        assert parts == len(runs), item
        if parts > 1:
            for i in range(parts):
                assert places[first if i == 0 else (first & ~1) + 2 * i] == (item, i)
        most = max(most, parts)
    return most, groups


def test_the_formulas_are_found():
    assert "if (begin == 0 && tid == 0) p.first_items[(size_t)entry * Hkv + head] = shared ? int2{(int)(2 * me + (first_run ? 0 : 1)), (int)(w1 - w0 + 1)} : int2{0, 1};" in SOURCE
    assert "place = i == 0 ? item_of.x : (item_of.x & ~1) + 2 * i;" in SOURCE
    assert "w0 = group_of(item + OVER + WAVES - 1);" in SOURCE and "w1 = group_of(item + OVER + span.steps - 1);" in SOURCE
    assert "s.lo = s.hi = w.at - 1;" in SOURCE and "s.steps = max((s.hi + STEP) / STEP, 1);" in SOURCE
    assert "max((uint32_t)(entries * Hkv), (total - (uint32_t)(entries * Hkv) * OVER) / LEAST)" in SOURCE
    assert "return AttnWhere{n < p.least_shared ? 0 : n, 0, false};" in SOURCE
    for NB, F in ((1, 4), (1, 2), (1, 1), (2, 1), (4, 1)):
        assert least_of(NB, F) >= 2 * WAVES and constant("workgroups", NB, F) == GRID


@pytest.mark.parametrize("rows", [1, 4, 5, 8, 16, 17, 32, 33, 64, 65, 130, 1024])
@pytest.mark.parametrize("Hkv", [1, 2, 8, 32])
def test_one_group_of_any_length(rows, Hkv):
    most = [check(rows, Hkv, [n]) for n in list(range(0, 3000, 61)) + list(range(3000, 131072, 2819)) + [1 << 20, (1 << 30) - 1, 1 << 30]]
    items = -(-rows // constant("rows", *instance(rows))) * Hkv
    assert max(groups for _, groups in most) == GRID
    assert max(parts for parts, _ in most) > 4 if items <= GRID // 8 else items <= GRID        # (an item to each workgroup has nothing to divide)


def test_groups_of_mixed_lengths():
    rng = random.Random(2)
    most = []
    for _ in range(500):
        longest = rng.choice((70, 900, 9000, 130000))
        shared = [rng.choice((rng.randint(-3, longest), rng.randint(0, 70))) for _ in range(rng.choice((1, 2, 3, 7, 16, 64, 300)))]
        most.append(check(rng.choice((1, 3, 8, 16, 20, 32, 64, 200)), rng.choice((1, 2, 5, 8)), shared, rng.choice((0, 0, 1, 64, 400, longest // 2 + 1)),
                          rng.choice((1 << 30, 16 * (longest // 32 + 1)))))
    assert max(parts for parts, _ in most) > 16


def test_items_by_the_rounds():
    """As many items as the workgroups take whole in up to eight rounds, and more: where they are not dealt out whole they divide like others."""
    for groups in (GRID, GRID + 1, 2 * GRID, ROUNDS * GRID, ROUNDS * GRID + 1):
        check(3, 1, [n * 37 % 5000 for n in range(groups)])


def test_the_check_sees_shares_that_round_down_to_nothing():
    """A share of fewer steps than a round of wavefronts leaves a workgroup without a part where readers look for one."""
    with pytest.raises(AssertionError):
        for n in range(1100, 40000, 32):
            check(16, 1, [n], least=2)
