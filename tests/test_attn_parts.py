"""Parts of items that a launch of attention with a workgroup to each has (shared beginnings, chosen pages): how many the host asks for, against the arrival
counters and the places for their sums.  The rules are compiled from their source.  Needs no GPU."""
import ctypes
import os
import random
import re
import shutil
import subprocess

import pytest

from paper_2410_11305_amd import binding as B
from paper_2410_11305_amd import build
from tests.test_attn_division import SOURCE, constant

PLANS = [(1, 4), (1, 2), (1, 1), (2, 1), (4, 1)]
ROWS = {p: constant("rows", *p) for p in PLANS}
TICKETS = int(re.search(r"constexpr size_t kAttnTicketBytes = (\d+);", SOURCE).group(1))
COUNTERS = TICKETS // 4
PLACES = 2 * constant("workgroups", 1, 1)


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    compiler = shutil.which("g++")
    if compiler is None:
        pytest.skip("no host compiler")
    source = open(os.path.join(build.HERE, "csrc", "qspec_api.hip")).read()
    text = source[source.index("constexpr int attn_part_sets("):source.index("// A call's workspace: what the second launch")]
    folder = tmp_path_factory.mktemp("parts")
    code, library = str(folder / "parts.cpp"), str(folder / "parts.so")
    open(code, "w").write("struct AttnPlan { int nb, f; };\ntemplate <int NB, int F> struct AttnForm { static constexpr int places = %d; };\nconstexpr int kAttnCounters = %d;\n"
                          % (PLACES, COUNTERS) + text + """
extern "C" long long most(int nb, int f) { return attn_most_parts({nb, f}); }
extern "C" int own(long long items, long long tokens, int nb, int f) { const AttnParts p = own_parts(items, tokens, {nb, f}); return p.fill << 8 | p.split; }
extern "C" int listed(long long items, int steps) { const AttnParts p = list_parts(items, steps); return p.fill << 8 | p.split; }
""")
    subprocess.run([compiler, "-std=c++17", "-shared", "-fPIC", "-o", library, code], check=True, capture_output=True)
    L = ctypes.CDLL(library)
    L.most.restype, L.most.argtypes = ctypes.c_longlong, [ctypes.c_int] * 2
    L.own.argtypes, L.listed.argtypes = [ctypes.c_longlong, ctypes.c_longlong, ctypes.c_int, ctypes.c_int], [ctypes.c_longlong, ctypes.c_int]
    return L


def numbers(seed, top):
    rng = random.Random(seed)
    edges = [x for k in range(25) for x in ((1 << k) - 1, 1 << k, (1 << k) + 1)]
    return sorted({x for x in edges + [int(2 ** rng.uniform(0, 25)) for _ in range(200)] if 1 <= x <= top})


def test_the_kernel_counts_and_places_by_these():
    """An item's counter and its parts' places, as the kernel has them: below items << split."""
    assert "if constexpr (FIXED) counter = item << p.split;" in SOURCE
    assert "MODE == kAttnPages ? me - part_of_item + w : FIXED ? w * items + item" in SOURCE
    assert "write_part(FIXED ? me : 2 * me + (first_run ? 0 : 1), r, ref, total_l, v);" in SOURCE
    assert "static constexpr int places = 2 * workgroups;" in SOURCE and all(2 * constant("workgroups", *p) == PLACES for p in PLANS)


@pytest.mark.parametrize("plan", PLANS)
def test_parts_have_counters_and_places(rules, plan):
    most = rules.most(*plan)
    assert most <= COUNTERS and most % PLACES == 0
    split_at_all = 0
    for items in numbers(1, 1 << 24):
        for tokens in [16, 4096, 4097, 8192, 8193, 16384, 40000, 131072, 1 << 20, 1 << 30]:
            fill, split = divmod(rules.own(items, tokens, *plan), 256)
            assert 0 <= fill <= split <= 4
            if split:
                split_at_all += 1
                assert items << split <= most, (items, tokens)
            assert fill == 0 or items << fill <= 256
    assert split_at_all > 100


def test_parts_of_lists_have_counters_and_places(rules):
    for items in numbers(2, 1 << 24):
        for steps in numbers(3, 1 << 20):
            fill, split = divmod(rules.listed(items, steps), 256)
            assert fill == split <= 4 and (split == 0 or (items << split <= min(PLACES, COUNTERS) and steps >> split >= 4))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G", [1, 2, 4, 7, 8, 16, 33])
@pytest.mark.parametrize("T", [1, 2, 3, 5, 40])
def test_workspaces_hold_them(rules, D, G, T):
    """Sizes as the library says them: the counters, the parts of both launches, their directory, sums of all rows."""
    instance = lambda rows: (1, 4) if rows <= 4 else (1, 2) if rows <= 8 else (1, 1) if rows <= 16 else (2, 1) if rows <= 32 else (4, 1)
    part = (D + 4) * 4
    assert B.attn_kv4_blocks_workspace_bytes(5, T, 3 * G, 3, D) >= TICKETS + PLACES * ROWS[instance(G)] * part
    for groups, per in ((1, 1), (1, 8), (3, 5), (16, 2)):
        own, first, Hkv, Bn = instance(T * G), instance(per * T * G), 3, groups * per
        items = groups * -(-per * T * G // ROWS[first]) * Hkv
        least = TICKETS + rules.most(*own) * ROWS[own] * part + PLACES * ROWS[first] * part + items * 8 + Bn * T * Hkv * G * part
        assert B.attn_kv4_shared_workspace_bytes(Bn, T, Hkv * G, Hkv, D, groups) >= least
