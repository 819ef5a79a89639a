"""Host-side checks of attention behind shared beginnings, the bounds of pages, the choice of pages and attention over them that need no
GPU: sizes, refusals before anything is launched, and pins of the oracle."""
import math
import os
import re

import numpy as np
import pytest

from oracle import kv4_pages_oracle as pg
from paper_2410_11305_amd import binding as B
from paper_2410_11305_amd import build

A = 4096          # any 16-byte aligned non-null address: rejected before use


def share(**k):
    a = dict(q=A, cache=A, pos=A, table=A, shared=A, B=6, T=3, Hq=8, Hkv=2, D=128, groups=2, page=64, each=4, pages=30, scale=0.1, out=A, ws=A, nws=1 << 30)
    a.update(k)
    return B.lib().qspec_attn_kv4_shared(*a.values(), None)


def bound(**k):
    a = dict(cache=A, pos=A, table=A, B=2, T=3, Hkv=2, D=128, page=64, each=4, pages=9, bounds=A)
    a.update(k)
    return B.lib().qspec_kv4_bounds(*a.values(), None)


def read(**k):
    a = dict(cache=A, pos=A, table=A, B=2, T=3, Hkv=2, D=128, page=64, each=4, pages=9, upper=A, lower=A)
    a.update(k)
    return B.lib().qspec_kv4_bounds_read(*a.values(), None)


def select(**k):
    a = dict(q=A, cache=A, pos=A, table=A, B=2, T=3, Hq=8, Hkv=2, D=128, page=64, each=4, pages=9, first=1, last=1, count=3, out=A, ws=A, nws=1 << 30)
    a.update(k)
    return B.lib().qspec_kv4_select(*a.values(), None)


def attend(**k):
    a = dict(q=A, cache=A, pos=A, table=A, list=A, B=2, T=3, Hq=8, Hkv=2, D=128, count=3, page=64, each=4, pages=9, scale=0.1, out=A, ws=A, nws=1 << 30)
    a.update(k)
    return B.lib().qspec_attn_kv4_blocks(*a.values(), None)


def test_sizes():
    assert B.kv4_bounds_bytes(8, 128) == 8 * 256 + 32 and B.kv4_bounds_bytes(1, 64) == 128 + 16 and B.kv4_bounds_bytes(5, 64) == 5 * 128 + 32
    assert B.kv4_bounds_bytes(0, 128) == B.kv4_bounds_bytes(8, 96) == 0
    joint = 8 * 2 * 16 * 132 * 4
    assert B.attn_kv4_shared_workspace_bytes(8, 2, 16, 2, 128, 2) > 16384 + joint
    for bad in ((8, 2, 16, 2, 128, 0), (8, 2, 16, 2, 128, 3), (8, 2, 16, 3, 128, 2), (8, 2, 16, 2, 96, 2), (8, 1 << 18, 1, 1, 64, 1)):
        assert B.attn_kv4_shared_workspace_bytes(*bad) == 0
    assert B.kv4_select_workspace_bytes(2, 3, 8, 2, 65) == 2 * 3 * 2 * 128 * 4
    assert B.kv4_select_workspace_bytes(2, 3, 8, 3, 65) == B.kv4_select_workspace_bytes(2, 3, 8, 2, (1 << 24) + 1) == 0
    assert B.attn_kv4_blocks_workspace_bytes(2, 300, 8, 2, 128) == B.attn_kv4_workspace_bytes(2, 1, 8, 2, 128)
    assert B.attn_kv4_blocks_workspace_bytes(2, 3, 8, 2, 80) == 0


@pytest.mark.parametrize("call", [share, bound, read, select, attend])
def test_cache_shapes_are_refused(call):
    for bad in (dict(B=0), dict(T=0), dict(D=96), dict(page=24), dict(page=8), dict(each=0), dict(pages=0), dict(Hkv=0),
                dict(table=None, pages=7), dict(page=1 << 15, each=1 << 16), dict(T=(1 << 20) + 1, B=2, D=64)):
        assert call(**bad) == B.ERR_SHAPE, bad
    if call is not share:
        assert call(page=32) == B.ERR_SHAPE                   # a block is a page of 64 tokens at least
    assert call(cache=A + 8) == B.ERR_ALIGN and call(pos=A + 2) == B.ERR_ALIGN and call(table=A + 2) == B.ERR_ALIGN
    assert call(cache=None) == B.ERR_NULL and call(pos=None) == B.ERR_NULL


@pytest.mark.parametrize("call", [share, attend])
def test_attention_refusals(call):
    for bad in (dict(Hq=9), dict(Hq=0), dict(Hq=1), dict(Hq=512), dict(scale=0.0), dict(scale=-1.0), dict(scale=math.nan), dict(scale=1e11), dict(B=1 << 14, T=1 << 14)):
        assert call(**bad) == B.ERR_SHAPE, bad
    assert call(q=None) == call(out=None) == call(ws=None) == B.ERR_NULL
    assert call(q=A + 2) == call(out=A + 8) == call(ws=A + 4) == B.ERR_ALIGN


def test_shared_refusals():
    assert share(shared=None) == B.ERR_NULL and share(shared=A + 2) == B.ERR_ALIGN
    for bad in (dict(groups=0), dict(groups=-1), dict(groups=4), dict(groups=7), dict(B=4, T=1 << 19, groups=1, Hq=1, Hkv=1, D=64)):
        assert share(**bad) == B.ERR_SHAPE, bad
    size = B.attn_kv4_shared_workspace_bytes(6, 3, 8, 2, 128, 2)
    assert share(nws=size - 1) == B.ERR_WORKSPACE
    # more work than is counted in 32 bits
    assert share(B=1024, T=4, Hq=64, Hkv=64, D=64, groups=1024, each=1 << 14) == B.ERR_SHAPE
    assert share(B=1024, T=4, Hq=64, Hkv=64, D=64, groups=1, each=1 << 14) == B.ERR_SHAPE


def test_bounds_refusals():
    assert bound(bounds=None) == read(upper=None) == read(lower=None) == B.ERR_NULL
    assert bound(bounds=A + 8) == read(upper=A + 4) == read(lower=A + 8) == B.ERR_ALIGN
    assert bound(B=1 << 22, T=70) == read(B=1 << 22, T=70) == bound(Hkv=65536, D=64) == B.ERR_SHAPE
    assert read(B=1 << 14, T=1 << 10, Hkv=16) == B.ERR_SHAPE              # 17 pages of 8 KB a sequence


def test_choice_refusals():
    for bad in (dict(Hq=9), dict(Hq=0), dict(Hq=512), dict(count=0), dict(first=-1), dict(last=-1), dict(first=2, last=2), dict(first=2 ** 31 - 1, last=2 ** 31 - 1),
                dict(count=1 << 28), dict(B=1 << 14, T=1 << 14)):
        assert select(**bad) == B.ERR_SHAPE, bad
    assert select(q=None) == select(out=None) == select(ws=None) == B.ERR_NULL
    assert select(q=A + 8) == select(out=A + 2) == select(ws=A + 8) == B.ERR_ALIGN
    assert select(nws=B.kv4_select_workspace_bytes(2, 3, 8, 2, 4) - 1) == B.ERR_WORKSPACE


def test_blocks_refusals():
    assert attend(list=None) == B.ERR_NULL and attend(list=A + 2) == B.ERR_ALIGN
    assert attend(count=0) == attend(count=1 << 28) == B.ERR_SHAPE
    assert attend(nws=B.attn_kv4_blocks_workspace_bytes(2, 3, 8, 2, 128) - 1) == B.ERR_WORKSPACE
    assert attend(B=1024, T=4, Hq=64, Hkv=64, D=64, count=1000, page=1024, each=1 << 14) == B.ERR_SHAPE         # more work than is counted in 32 bits


def test_binding_refuses_tensors_that_do_not_fit():
    import torch
    cache, pos = torch.zeros((4, B.kv4_page_bytes(2, 64, 64)), dtype=torch.uint8), torch.zeros(2, dtype=torch.int32)
    bounds, q = torch.zeros((4, B.kv4_bounds_bytes(2, 64)), dtype=torch.uint8), torch.zeros((2, 1, 4, 64), dtype=torch.float16)
    calls = [lambda: B.attn_kv4_shared(q, cache, pos, pos, 2, 64), lambda: B.kv4_bounds(cache, pos, 1, bounds, 2, 64, 64), lambda: B.kv4_bounds_read(bounds, pos, 1, 2, 64, 64),
             lambda: B.kv4_select(q, bounds, pos, 2, 64, 2), lambda: B.attn_kv4_blocks(q, cache, pos, pos, 2, 64)]
    for call in calls:
        with pytest.raises(ValueError, match="GPU"):
            call()
    with pytest.raises(B.QSpecError):
        B.alloc_kv4_bounds(4, 2, 96)
    with pytest.raises(B.QSpecError):
        B.kv4_select(q, bounds, torch.zeros(0, dtype=torch.int32), 2, 64, 2)
    with pytest.raises(B.QSpecError):
        B.kv4_bounds_read(bounds, pos, 1, 2, 80, 64)


# ------------------------------------------------------------------ parts of an item
def test_parts_of_an_item_take_every_step_once():
    """A workgroup's share of an item as the kernel has it, with the formulas read from the source: parts follow each other, cover all steps, and are as many as are
    waited for."""
    source = re.sub(r"//.*", "", open(os.path.join(build.HERE, "csrc", "attn_kv4.hpp")).read())
    block = source[source.index("if constexpr (FIXED) {\n      const int rounds"):]
    whole, *longs = map(int, re.search(r"constexpr int WHOLE = (\d+), LONG = F > 1 \? (\d+) : (\d+);", source).groups())

    def formula(text):
        e = re.search(text, block).group(1).replace("/", "//").replace("span.steps", "steps").replace("p.split", "split").replace("p.fill", "fill")
        e = re.sub(r"(.*?) \? (.*?) : (.*?) \? (.*?) : (.*)", r"((\2) if \1 else (\4) if \3 else (\5))", e)
        return compile(e, "formula", "eval")

    rounds_of, even_of, least_of, each_of, parts_of = (formula(t) for t in (r"const int rounds = ([^,;]*),", r"even = ([^,;]*),", r"least = ([^,;]*);", r"const int each = ([^;]*);", r"item_parts = ([^;]*);"))
    assert "begin = (int)part_of_item * each * WAVES;" in block and "if (begin >= span.steps) return;" in block and "stop = min(span.steps, begin + each * WAVES);" in block
    for WAVES, long_ in [(w, n) for w in (1, 4, 8) for n in longs]:
        for fill in range(5):
            for split in range(fill, 5):
                for steps in list(range(1, 300)) + [1000, 1023, 1024, 1025, 65536]:
                    names = dict(WAVES=WAVES, WHOLE=whole, LONG=long_, fill=fill, split=split, steps=steps, max=max)
                    for name, code in (("rounds", rounds_of), ("even", even_of), ("least", least_of), ("each", each_of)):
                        names[name] = eval(code, {}, names)
                    parts, at = eval(parts_of, {}, names), 0
                    for part in range(1 << split):
                        begin = part * names["each"] * WAVES
                        if begin >= steps:
                            assert part >= parts
                            continue
                        assert begin == at and part < parts
                        at = min(steps, begin + names["each"] * WAVES)
                    assert at == steps and 1 <= parts <= 1 << split


# ------------------------------------------------------------------ pins of the oracle
def test_grids():
    assert [pg.grid_of(x) for x in (0.0, 127.0, 127.5, 63.5, 63.0, 1.0, 254.0)] == [1.0, 1.0, 2.0, 0.5, 0.5, 2.0 ** -6, 2.0]
    assert pg.grid_of(2.0 ** -24) == 2.0 ** -30 and pg.grid_of(65504.0) == 1024.0


def test_bounds_hold_every_key():
    rng = np.random.default_rng(1)
    codes, step, low = rng.integers(0, 16, (40, 64)), rng.uniform(0.1, 0.5, 40).astype(np.float16), rng.uniform(-4, 1, 40).astype(np.float16)
    upper, lower, grid = pg.bounds(codes, step, low)
    keys = codes * step.astype(float)[:, None] + low.astype(float)[:, None]
    assert (upper * float(grid) >= keys.max(0) * (1 - 2.0 ** -24)).all() and (upper * float(grid) < keys.max(0) + grid * 1.001).all()
    assert (lower * float(grid) <= keys.min(0) * (1 - 2.0 ** -24) + 2.0 ** -20).all() and 64 <= max(abs(upper.astype(int)).max(), abs(lower.astype(int)).max()) <= 127
    # and the score of a page is no smaller than any token's, but for the rounding of the query
    q = rng.standard_normal((2, 64)).astype(np.float16)
    c = pg.query_codes(q)
    s = pg.scores(q, upper[None], lower[None], np.array([grid]), np.array([True]))
    assert s[0] >= (c @ keys.T).max() * (1 - 1e-6)


def test_choices_by_hand():
    s = np.array([1.0, 5.0, 3.0, 5.0, 0.0, 2.0])
    assert pg.choose(s, 0, 0, 1).tolist() == [1] and pg.choose(s, 0, 0, 2).tolist() == [1, 3] and pg.choose(s, 1, 1, 3).tolist() == [0, 1, 5]
    assert pg.choose(s, 0, 0, 8).tolist() == [0, 1, 2, 3, 4, 5, -1, -1] and pg.choose(np.zeros(0), 0, 0, 2).tolist() == [-1, -1]
    assert pg.choose(np.array([0.0, -np.inf, 1.0, np.inf]), 0, 0, 3).tolist() == [0, 2, 3]
    assert pg.listed([3, 3, 2, 5, 9], 9, 8) == [3, 5] and pg.listed([-1, 0, 1], 2, 8) == [0] and pg.listed([0, 1, 2], 1, 8) == [0]
