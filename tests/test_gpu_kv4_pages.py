"""Bounds of pages, the choice of pages by them, and attention over chosen pages, against the oracle.  Bounds and choices are whole numbers and
have to be equal.  How far the attention may be off: as in tests/test_gpu_attn_kv4.py, over the tokens that the row's list leaves."""
import numpy as np
import pytest

from oracle import kv4_oracle as kv
from oracle import kv4_pages_oracle as pg
from tests.test_gpu_attn_kv4 import Cache, dev, queries, shuffled

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2410_11305_amd import binding as B
    assert torch.cuda.is_available()
    B.lib()
    return torch, B


# ------------------------------------------------------------------ bounds
def oracle_bounds(c, table, pos, T, upper, lower, grid):
    """Updates the codes [pages, Hkv, D] and grids [pages, Hkv] as a call does."""
    for b in range(len(pos)):
        last = min(int(pos[b]) + T, table.shape[1] * c.P) - 1
        first = max(int(pos[b]), 0)
        for number in range(first // c.P, last // c.P + 1 if last >= first else 0):
            page, n = int(table[b, number]), min(last + 1 - number * c.P, c.P)
            if 0 <= page < c.n_pages:
                for h in range(c.Hkv):
                    upper[page, h], lower[page, h], grid[page, h] = pg.bounds(c.k[page, h, :n], c.ks[page, h, :n], c.kl[page, h, :n])


def empty_bounds(c):
    return np.zeros((c.n_pages, c.Hkv, c.D), np.int8), np.zeros((c.n_pages, c.Hkv, c.D), np.int8), np.zeros((c.n_pages, c.Hkv), np.float32)


def check_bounds(env, c, table, pos, T, no_table=False):
    torch, B = env
    state = empty_bounds(c)
    state[0][:] = 77
    bounds = dev(torch, pg.bounds_bytes(*state))
    tab = None if no_table else dev(torch, table.astype(np.int32))
    at = dev(torch, np.asarray(pos, np.int32))
    B.kv4_bounds(dev(torch, c.bytes()), at, T, bounds, c.Hkv, c.D, c.P, tab)
    oracle_bounds(c, table, pos, T, *state)
    assert (bounds.cpu().numpy() == pg.bounds_bytes(*state)).all()
    # and their values back
    touched = (T - 1) // c.P + 2
    upper, lower = B.kv4_bounds_read(bounds, at, T, c.Hkv, c.D, c.P, tab)
    want = np.zeros((2, len(pos), touched, c.Hkv, c.D), np.float32)
    for b in range(len(pos)):
        first, last = max(int(pos[b]), 0), min(int(pos[b]) + T, table.shape[1] * c.P) - 1
        for i in range(touched):
            number = first // c.P + i
            if number * c.P <= last and 0 <= table[b, number] < c.n_pages:
                for w in range(2):
                    want[w, b, i] = state[w][table[b, number]].astype(np.float32) * state[2][table[b, number]][:, None]
    assert np.array_equal(upper.cpu().numpy(), want[0], equal_nan=True) and np.array_equal(lower.cpu().numpy(), want[1], equal_nan=True)
    return bounds


@pytest.mark.parametrize("Bn,T,Hkv,D,P,n", [(1, 1, 1, 64, 64, 1), (3, 1, 2, 128, 64, 200), (2, 64, 5, 64, 64, 300), (1, 65, 3, 128, 64, 200), (2, 130, 1, 128, 128, 500), (4, 5, 8, 64, 256, 700),
                                           (1, 700, 2, 128, 64, 700), (40, 1, 32, 128, 64, 128)])
def test_bounds(env, Bn, T, Hkv, D, P, n):
    rng = np.random.default_rng(T + n)
    pos = np.r_[n - T, rng.integers(-1, n - T + 1, Bn - 1)]
    each = -(-n // P)
    check_bounds(env, Cache(n + D, Bn * each + 1, Hkv, D, P), shuffled(T, Bn, each, Bn * each + 1), pos, T)


def test_bounds_at_the_ends(env):
    """Idle sequences, positions in front of and past the cache, pages that are not there, pages in order."""
    P, each, T = 64, 4, 70
    pos = np.array([-70, -69, 0, 186, 187, 255, 256, 2 ** 31 - 1, -(2 ** 31), 100])
    c = Cache(3, 42, 2, 64, P)
    table = shuffled(4, 10, each, 42).astype(np.int64)
    table[2, 1], table[3, 2], table[9, 1] = -1, 42, 2 ** 31 - 1
    check_bounds(env, c, table, pos, T)
    check_bounds(env, c, np.arange(40).reshape(10, 4), pos, T, no_table=True)


@pytest.mark.parametrize("D", [64, 128])
def test_bounds_of_every_size(env, D):
    """Zeros, subnormals, fp16's largest, values next to the grid's borders, NaN rows, and what stands behind the last token."""
    P = 64
    c = Cache(5, 12, 2, D, P)
    c.ks[0], c.kl[0] = 0, 0
    c.ks[1], c.kl[1] = 2.0 ** -24, 0
    c.ks[2], c.kl[2] = 65504.0, -65504.0
    c.ks[3], c.kl[3] = 0, 127.0                                # exactly 127 of the grid
    c.ks[4], c.kl[4] = 0, -127.125                             # just past it
    c.ks[5], c.kl[5] = 8.0, 7.0                                # 127 with the largest code
    c.k[5, :, :, 3] = 15
    c.ks[6, 1, 17], c.kl[6, 1, 17] = np.nan, np.nan            # one head has a row that is no number
    c.kl[7, 0, 63] = np.inf
    c.ks[8, :, 40:], c.kl[8, :, 40:] = np.nan, np.inf          # behind the last token
    c.ks[9], c.kl[9] = 2.0 ** -20, -(2.0 ** -20) * 7
    table, pos = np.arange(12).reshape(12, 1), np.full(12, 0)
    pos[8] = -24
    check_bounds(env, c, table, pos, 64)


# ------------------------------------------------------------------ the choice
class Bounds:
    def __init__(self, seed, n_pages, Hkv, D):
        rng = np.random.default_rng(seed)
        a, b = rng.integers(-127, 128, (2, n_pages, Hkv, D))
        self.upper, self.lower = np.maximum(a, b).astype(np.int8), np.minimum(a, b).astype(np.int8)
        self.grid = (2.0 ** rng.integers(-6, -3, (n_pages, Hkv))).astype(np.float32)
        self.n_pages, self.Hkv, self.D = n_pages, Hkv, D

    def bytes(self):
        return pg.bounds_bytes(self.upper, self.lower, self.grid)


def oracle_choice(bounds, q, pos, table, P, first, last, count):
    Bn, T, Hq, D = q.shape
    G = Hq // bounds.Hkv
    out = np.zeros((Bn, T, bounds.Hkv, count), np.int32)
    for b in range(Bn):
        for j in range(T):
            n = pg.in_sight(int(pos[b]) + j, P, table.shape[1])
            page = table[b, :n]
            there = (page >= 0) & (page < bounds.n_pages)
            page = np.where(there, page, 0).astype(np.int64)
            for h in range(bounds.Hkv):
                s = pg.scores(q[b, j, h * G:(h + 1) * G], bounds.upper[page, h], bounds.lower[page, h], bounds.grid[page, h], there) if n else np.zeros(0)
                out[b, j, h] = pg.choose(s, first, last, count)
    return out


def check_choice(env, bounds, q, pos, table, P, first, last, count, no_table=False, workspace=None):
    torch, B = env
    Bn, T, Hq, D = q.shape
    out = torch.full((Bn, T, bounds.Hkv, count), -77, dtype=torch.int32, device="cuda")
    B.kv4_select(dev(torch, q), dev(torch, bounds.bytes()), dev(torch, np.asarray(pos, np.int32)), bounds.Hkv, P, count,
                 None if no_table else dev(torch, table.astype(np.int32)), first=first, last=last, blocks=out, workspace=workspace)
    want = oracle_choice(bounds, q, pos, table, P, first, last, count)
    got = out.cpu().numpy()
    assert (got == want).all(), np.argwhere((got != want).any(-1))[:5]
    return got


@pytest.mark.parametrize("Bn,T,Hq,Hkv,D,P,each,first,last,count", [
    (1, 1, 1, 1, 64, 64, 40, 0, 0, 1), (2, 1, 8, 2, 128, 64, 70, 1, 1, 8), (1, 1, 64, 8, 128, 64, 300, 1, 2, 64), (3, 4, 8, 1, 64, 64, 100, 2, 3, 16), (2, 5, 6, 2, 128, 128, 33, 1, 0, 7),
    (1, 3, 7, 1, 128, 64, 65, 0, 4, 4), (1, 17, 4, 4, 64, 64, 90, 1, 1, 20), (2, 2, 32, 2, 64, 256, 50, 0, 1, 5), (1, 3, 17, 1, 128, 64, 64, 1, 1, 9), (1, 2, 80, 2, 64, 64, 129, 3, 0, 30),
    (1, 40, 10, 2, 64, 64, 37, 1, 1, 12), (1, 1, 255, 1, 64, 64, 17, 0, 1, 3), (5, 1, 3, 3, 128, 64, 16, 16, 0, 16), (70, 1, 2, 1, 64, 64, 20, 1, 1, 6), (2, 2, 2, 2, 64, 64, 33, 0, 0, 33)])
def test_choice(env, Bn, T, Hq, Hkv, D, P, each, first, last, count):
    rng = np.random.default_rng(count + T)
    n_pages = Bn * each + 3
    pos = np.r_[each * P - T, rng.integers(-T, each * P, Bn - 1)]
    check_choice(env, Bounds(each, n_pages, Hkv, D), queries(count, Bn, T, Hq, D), pos, shuffled(T, Bn, each, n_pages), P, first, last, count)


@pytest.mark.parametrize("each,count", [(3000, 100), (8192, 64), (8193, 1000), (20000, 37), (9000, 8999)])
def test_choice_of_many_pages(env, each, count):
    b = Bounds(each, each, 1, 64)
    check_choice(env, b, queries(1, 1, 2, 2, 64), np.array([each * 64 - 2]), np.random.default_rng(2).permutation(each).reshape(1, each), 64, 1, 2, count)


@pytest.mark.parametrize("Bn,T,Hkv,each,count", [(90, 3, 1, 24, 7), (3, 50, 2, 70, 20), (1, 260, 1, 2100, 50)])
def test_choice_of_many_rows(env, Bn, T, Hkv, each, count):
    """Pages with few different scores among them."""
    b = Bounds(T, Bn * each, Hkv, 64)
    b.upper[::3], b.lower[::3], b.grid[:] = b.upper[0], b.lower[0], 0.125
    pos = np.r_[each * 64 - T, np.random.default_rng(1).integers(-T, each * 64, Bn - 1)]
    check_choice(env, b, queries(2, Bn, T, 2 * Hkv, 64), pos, shuffled(3, Bn, each, Bn * each), 64, 1, 2, count)


@pytest.mark.parametrize("n", [2000, 9000])
@pytest.mark.parametrize("count", [1, 5, 64, 200])
def test_choice_among_equals(env, n, count):
    """All pages alike, two kinds of them, few different scores: the lower ones are taken."""
    b = Bounds(3, n, 1, 64)
    table, pos, q = np.arange(n).reshape(1, n), np.array([n * 64 - 1]), queries(3, 1, 1, 2, 64)
    b.upper[:], b.lower[:], b.grid[:] = b.upper[0], b.lower[0], 0.25
    check_choice(env, b, q, pos, table, 64, 0, 0, count)
    b.grid[::17] = 0.5
    check_choice(env, b, q, pos, table, 64, 1, 0, count)
    b.grid[:] = 2.0 ** np.random.default_rng(4).integers(-3, 3, b.grid.shape)
    check_choice(env, b, q, pos, table, 64, 0, 1, count)
    check_choice(env, b, np.zeros_like(q), pos, table, 64, 0, 0, count)


def test_choice_at_the_ends(env):
    """Idle and empty sequences, positions past the cache, fewer pages than are asked for, pages that are not there, in order without a table."""
    P, each, T, n_pages = 64, 9, 3, 100
    pos = np.array([-3, -2, -1, 0, 61, 62, 63, 300, 575, 576, 2 ** 31 - 1, -(2 ** 31)])
    b = Bounds(6, n_pages + 20, 2, 64)
    table = shuffled(5, 12, each, n_pages + 20).astype(np.int64)
    q = queries(7, 12, T, 4, 64)
    check_choice(env, b, q, pos, table, P, 1, 1, 4)
    check_choice(env, b, q, pos, table, P, 0, 2, 12)
    check_choice(env, b, q, pos, np.arange(120)[:108].reshape(12, 9), P, 1, 1, 4, no_table=False)
    b = Bounds(6, 108, 2, 64)
    check_choice(env, b, q, pos, np.arange(108).reshape(12, 9), P, 1, 1, 4, no_table=True)
    table = np.where(table < 108, table, -1)
    table[7, 1:4] = [108, 2 ** 31 - 1, -(2 ** 31)]
    check_choice(env, b, q, pos, table, P, 1, 0, 4)
    check_choice(env, b, q, pos, np.full((12, 9), -1), P, 0, 0, 3)


def test_choice_with_what_is_no_number(env):
    b = Bounds(8, 60, 2, 128)
    table, pos = np.arange(60).reshape(1, 60), np.array([60 * 64 - 4])
    q = queries(9, 1, 4, 6, 128)
    q[0, 1, 4, 7], q[0, 2, 0, 0], q[0, 3, 5, 100] = np.nan, np.inf, -np.inf
    check_choice(env, b, q, pos, table, 64, 1, 1, 9)
    for pages in ([5], [5, 0, 59], list(range(3, 12)), list(range(60))):
        b.upper[pages, 1], b.lower[pages, 1], b.grid[pages, 1] = 0, 0, np.nan
        check_choice(env, b, q, pos, table, 64, 1, 1, 9)
        check_choice(env, b, q, pos, table, 64, 0, 0, 1)
        check_choice(env, b, q, pos, table, 64, 5, 4, 9)


@pytest.mark.parametrize("size", [2.0 ** -24, 2.0 ** -14, 1e-3, 60000.0])
def test_choice_by_queries_of_every_size(env, size):
    b = Bounds(10, 200, 1, 64)
    q = np.clip(queries(11, 1, 2, 4, 64) * np.float32(size), -65504, 65504).astype(np.float16)
    q[0, 1, :, 5] = np.float16(size) * np.float16(1.0)
    check_choice(env, b, q, np.array([200 * 64 - 2]), np.arange(200).reshape(1, 200), 64, 0, 0, 20)
    half = np.zeros((1, 1, 2, 64), np.float16)
    half[0, 0, :, 0] = 127                                     # halves are rounded to even
    half[0, 0, :, 1:] = np.arange(126).reshape(2, 63) + 0.5
    half = np.where(half > 127, 0, half).astype(np.float16)
    check_choice(env, b, half, np.array([200 * 64 - 1]), np.arange(200).reshape(1, 200), 64, 0, 0, 20)
    b.grid[:] = 2.0 ** np.random.default_rng(1).integers(-30, 15, b.grid.shape)
    check_choice(env, b, q, np.array([200 * 64 - 2]), np.arange(200).reshape(1, 200), 64, 0, 0, 20)


# ------------------------------------------------------------------ attention over chosen pages
def compare_blocks(got, cache, q, pos, table, blocks, scale=None, rows=None):
    Bn, T, Hq, D = q.shape
    Hkv, P, S = cache.Hkv, cache.P, table.shape[1] * cache.P
    G = Hq // Hkv
    scale = D ** -0.5 if scale is None else scale
    for b in range(Bn) if rows is None else rows:
        tokens = int(min(max(int(pos[b]) + T, 0), S))
        if tokens:
            k, v, present, step = cache.sequence(table[b], tokens)
        for j in range(T):
            at = int(pos[b]) + j
            n = pg.in_sight(at, P, table.shape[1])
            for h in range(Hkv):
                mine = pg.listed(blocks[b, j, h], n, table.shape[1]) if n else []
                t = np.array([e * P + i for e in mine for i in range(P)], dtype=np.int64)
                t = t[t <= min(at, tokens - 1)] if len(t) else t
                t = t[present[t]] if len(t) else t
                out = got[b, j, h * G:(h + 1) * G]
                if len(t) == 0:
                    assert (out == 0).all(), (b, j, h)
                    continue
                x = q[b, j, h * G:(h + 1) * G]
                want = kv.attention(x[None], k[t, h][:, None], v[t, h][:, None], np.ones(len(t), bool), [len(t)], scale)[0]
                size = np.abs(x.astype(np.float64)).sum(-1) * scale * (np.abs(k[t, h]).max() * 2.0)
                bound = (2.0 ** -11 * np.abs(want) + 2.0 ** -25 + (2.0 ** -11 * 8 + len(t) * 2.0 ** -29) * step[t, h].max()
                         + 2 * ((D + 12) * 2.0 ** -24 * size)[:, None] * 2 * np.abs(v[t, h]).max())
                worst = np.abs(out - want) - bound
                assert np.isfinite(out).all() and worst.max() <= 0, (b, j, h, worst.max(), bound.max())


def check_blocks(env, cache, q, pos, table, blocks, scale=None, no_table=False, workspace=None, rows=None, raw=None):
    torch, B = env
    Bn, T, Hq, D = q.shape
    guard = torch.full((q.size + 64,), 123.0, dtype=torch.float16, device="cuda")
    out = guard[32:-32].view(Bn, T, Hq, D)
    out.fill_(float("nan"))
    B.attn_kv4_blocks(dev(torch, q), dev(torch, cache.bytes() if raw is None else raw), dev(torch, np.asarray(pos, np.int32)), dev(torch, blocks.astype(np.int32)), cache.Hkv, cache.P,
                      None if no_table else dev(torch, table.astype(np.int32)), scale, out=out, workspace=workspace)
    torch.cuda.synchronize()
    assert (guard[:32] == 123.0).all() and (guard[-32:] == 123.0).all()
    compare_blocks(out.cpu().numpy().astype(np.float64), cache, q, pos, table, blocks, scale, rows)
    return out


def lists(seed, Bn, T, Hkv, count, pos, P, each):
    rng = np.random.default_rng(seed)
    out = np.full((Bn, T, Hkv, count), -1)
    for b in range(Bn):
        for j in range(T):
            n = pg.in_sight(int(pos[b]) + j, P, each)
            for h in range(Hkv):
                mine = np.sort(rng.permutation(n)[:count])
                out[b, j, h, :len(mine)] = mine
    return out


@pytest.mark.parametrize("Bn,T,Hq,Hkv,D,P,each,count", [
    (1, 1, 1, 1, 64, 64, 1, 1), (2, 1, 4, 2, 128, 64, 9, 3), (1, 1, 8, 1, 64, 64, 30, 8), (2, 4, 32, 4, 128, 64, 20, 5), (3, 3, 7, 1, 64, 128, 7, 2), (1, 2, 16, 1, 128, 64, 12, 12),
    (1, 3, 20, 1, 64, 64, 15, 4), (2, 1, 64, 2, 128, 256, 4, 3), (1, 2, 40, 1, 64, 64, 11, 6), (1, 1, 100, 1, 128, 64, 8, 5), (1, 37, 8, 4, 64, 64, 10, 3), (50, 1, 2, 2, 64, 64, 3, 2),
    (1, 1, 255, 1, 64, 64, 6, 4), (300, 2, 1, 1, 64, 64, 2, 1), (2, 130, 2, 2, 64, 64, 6, 5)])
def test_blocks(env, Bn, T, Hq, Hkv, D, P, each, count):
    rng = np.random.default_rng(count + T)
    pos = np.r_[each * P - T, rng.integers(-T, each * P - T + 1, Bn - 1)]
    n_pages = Bn * each + 1
    check_blocks(env, Cache(D + T, n_pages, Hkv, D, P), queries(T, Bn, T, Hq, D), pos, shuffled(3, Bn, each, n_pages), lists(5, Bn, T, Hkv, count, pos, P, each),
                 rows=range(Bn) if Bn <= 50 else range(0, Bn, 17))


def test_lists_of_every_kind(env):
    """Entries that are negative, out of order, twice the same, behind the row's position, past the cache; empty and idle rows."""
    P, each, count = 64, 8, 5
    rows = [[0, 1, 2, 3, 4], [-1, 0, 1, 2, 3], [-1] * 5, [3, 3, 3, 3, 3], [4, 2, 5, 5, 6], [0, 7, 8, 9, 2 ** 31 - 1], [-(2 ** 31), 2, -5, 4, 6], [7, 0, 7, 0, 7], [1, 2, 2, 1, 3], [6, 7, -1, -1, -1]]
    Bn = len(rows)
    blocks = np.array(rows)[:, None, None, :].repeat(2, 1).repeat(2, 2)
    blocks[:, 1, 1] = blocks[::-1, 1, 1]
    c = Cache(6, Bn * each, 2, 128, P)
    table = shuffled(7, Bn, each, Bn * each)
    for pos in (np.full(Bn, 500), np.arange(Bn) * 55 - 2, np.array([-1, -2, -3, 0, 63, 62, 64, 511, 510, 2 ** 31 - 1])):
        check_blocks(env, c, queries(8, Bn, 2, 4, 128), pos, table, blocks)
    table = table.astype(np.int64)
    table[:, 2], table[3:, 5], table[0] = -1, 10 ** 6, -1
    check_blocks(env, c, queries(8, Bn, 2, 4, 128), np.full(Bn, 500), table, blocks)
    check_blocks(env, c, queries(8, Bn, 2, 4, 128), np.full(Bn, 500), np.arange(Bn * each).reshape(Bn, each), blocks, no_table=True)


@pytest.mark.parametrize("Hq,Hkv,D,P,each,count", [(8, 1, 128, 64, 700, 600), (2, 2, 64, 256, 120, 100), (1, 1, 64, 64, 900, 900), (32, 1, 128, 64, 300, 250)])
def test_long_lists_are_shared_out_and_joined(env, Hq, Hkv, D, P, each, count):
    torch, B = env
    pos = np.array([each * P - 1, each * P // 2])
    c = Cache(9, 2 * each, Hkv, D, P)
    ws = B.alloc_workspace(B.attn_kv4_blocks_workspace_bytes(2, 1, Hq, Hkv, D))
    args = (env, c, queries(10, 2, 1, Hq, D, 2.0), pos, shuffled(11, 2, each, 2 * each), lists(12, 2, 1, Hkv, count, pos, P, each))
    first = check_blocks(*args, workspace=ws)
    assert int(ws[:16384].count_nonzero()) == 0
    assert torch.equal(first, check_blocks(*args, workspace=ws))


def test_all_pages_are_the_whole_context(env):
    torch, B = env
    P, each, T, Hq, Hkv, D = 64, 20, 3, 8, 2, 64
    pos = np.array([each * P - T, 700])
    c = Cache(13, 2 * each, Hkv, D, P)
    q, cache, at = dev(torch, queries(14, 2, T, Hq, D)), dev(torch, c.bytes()), dev(torch, pos.astype(np.int32))
    table = dev(torch, shuffled(15, 2, each, 2 * each).astype(np.int32))
    bounds = B.alloc_kv4_bounds(2 * each, Hkv, D)
    blocks = B.kv4_select(q, bounds, at, Hkv, P, each, table)
    assert (blocks[0] == torch.arange(each, device="cuda")).all() and (blocks[1, :, :, 11:] == -1).all()
    some, all_ = B.attn_kv4_blocks(q, cache, at, blocks, Hkv, P, table).float(), B.attn_kv4(q, cache, at, Hkv, P, table).float()
    v = float(np.abs(c.vs.astype(np.float32)).max())
    assert float((some - all_).abs().max()) <= 2 * (2.0 ** -11 * 8 * v + 2.0 ** -11 * float(all_.abs().max()) + 2.0 ** -14)


def test_pages_that_are_not_listed_may_hold_anything(env):
    P, each, D = 64, 10, 64
    c = Cache(16, each, 2, D, P)
    blocks = np.array([[[[0, 3, 9], [2, 3, 9]]]])
    table, pos, q = np.arange(each).reshape(1, each), np.array([each * P - 30]), queries(17, 1, 1, 6, D)
    want = check_blocks(env, c, q, pos, table, blocks)
    bad = Cache(16, each, 2, D, P)
    for a, x in ((bad.ks, np.nan), (bad.kl, np.inf), (bad.vs, np.inf), (bad.vl, np.nan)):
        for h, mine in ((0, (0, 3, 9)), (1, (2, 3, 9))):
            a[[i for i in range(each) if i not in mine], h] = x
        a[9, :, P - 29:] = x                                   # behind the row's position
    got = check_blocks(env, c, q, pos, table, blocks, raw=bad.bytes())
    env[0].cuda.synchronize()
    assert env[0].equal(want, got)


def test_two_streams_and_graphs(env):
    """Select and attention on two streams at once, and captured with what goes before them; two graphs that share one workspace in turn."""
    torch, B = env
    P, each, Bn, T, Hq, Hkv, D, count = 64, 40, 3, 2, 8, 2, 128, 7
    c = Cache(18, Bn * each, Hkv, D, P)
    table = shuffled(19, Bn, each, Bn * each)
    cache, tab = dev(torch, c.bytes()), dev(torch, table.astype(np.int32))
    full = dev(torch, np.zeros(Bn, np.int32))
    bounds = B.kv4_bounds(cache, full, each * P, B.alloc_kv4_bounds(Bn * each, Hkv, D), Hkv, D, P, tab)
    state = empty_bounds(c)
    oracle_bounds(c, table, np.zeros(Bn, np.int64), each * P, *state)
    reference = Bounds(0, Bn * each, Hkv, D)
    reference.upper, reference.lower, reference.grid = state
    q, pos = dev(torch, queries(20, Bn, T, Hq, D)), torch.tensor([2500, 1000, 300], dtype=torch.int32, device="cuda")
    outs = [torch.empty_like(q) for _ in range(3)]
    picks = [torch.empty((Bn, T, Hkv, count), dtype=torch.int32, device="cuda") for _ in range(3)]
    size = B.attn_kv4_blocks_workspace_bytes(Bn, T, Hq, Hkv, D)
    works, scratch = [B.alloc_workspace(size) for _ in range(3)], [torch.empty(B.kv4_select_workspace_bytes(Bn, T, Hq, Hkv, each), dtype=torch.uint8, device="cuda") for _ in range(3)]

    def call(i, w):
        B.kv4_select(q, bounds, pos, Hkv, P, count, tab, blocks=picks[i], workspace=scratch[w])
        B.attn_kv4_blocks(q, cache, pos, picks[i], Hkv, P, tab, out=outs[i], workspace=works[w])

    sides = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        for i, s in enumerate(sides):
            with torch.cuda.stream(s):
                call(i, i)
    call(2, 2)
    torch.cuda.synchronize()
    assert all(torch.equal(outs[i], outs[2]) and torch.equal(picks[i], picks[2]) for i in range(2))
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for i, g in enumerate(graphs):
        with torch.cuda.graph(g):
            call(i, 0)
    rng = np.random.default_rng(23)
    for r in range(4):
        q_new, at = queries(30 + r, Bn, T, Hq, D), rng.integers(-T, each * P - T, Bn)
        q.copy_(dev(torch, q_new))
        pos.copy_(dev(torch, at.astype(np.int32)))
        for o in outs:
            o.fill_(float("nan"))
        torch.cuda.synchronize()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        call(2, 2)
        torch.cuda.synchronize()
        assert all(torch.equal(outs[i], outs[2]) and torch.equal(picks[i], picks[2]) for i in range(2))
        want = oracle_choice(reference, q_new, at, table, P, 1, 1, count)
        assert (picks[0].cpu().numpy() == want).all()
        compare_blocks(outs[0].cpu().numpy().astype(np.float64), c, q_new, at, table, want)
        assert int(works[0][:16384].count_nonzero()) == 0


def test_a_decoder_over_a_long_context(env):
    """Appends, bounds, choices and attention in a row, as a program runs them: a prompt, draft steps, a verify pass that writes their rows again, and
    a rejection after which the bounds forget what was taken back.  Every stage is held to the oracle on what the stage before it really wrote."""
    torch, B = env
    from tests.test_gpu_kv4 import Plain, place
    Bn, Hq, Hkv, D, P, each, count = 2, 4, 2, 64, 64, 6, 3
    n_pages = Bn * each + 1
    rng = np.random.default_rng(24)
    table = shuffled(25, Bn, each, n_pages)
    tab, cache, bounds = dev(torch, table.astype(np.int32)), B.alloc_kv4_cache(n_pages, Hkv, D, P), B.alloc_kv4_bounds(n_pages, Hkv, D)
    plain = Plain(n_pages, Hkv, D, P)
    c = Cache(0, n_pages, Hkv, D, P)
    state = empty_bounds(c)
    freq = dev(torch, 10000.0 ** (-np.arange(0, D, 2) / D))

    def step(pos, T):
        qkv = rng.standard_normal((Bn, T, (Hq + 2 * Hkv) * D)).astype(np.float16)
        at = dev(torch, pos.astype(np.int32))
        q = B.rope_kv4_append(dev(torch, qkv), freq, at, cache, Hq, Hkv, P, tab)
        B.kv4_bounds(cache, at, T, bounds, Hkv, D, P, tab)
        picked = B.kv4_select(q, bounds, at, Hkv, P, count, tab)
        out = B.attn_kv4_blocks(q, cache, at, picked, Hkv, P, tab)
        x = qkv.reshape(Bn * T, Hq + 2 * Hkv, D)
        where = pos[:, None].astype(np.int64) + np.arange(T)
        turned = kv.rotate(x[:, :Hq + Hkv], where.ravel(), freq.cpu().numpy(), False)
        for b in range(Bn):
            for j in range(T):
                there = place(table, b, int(where[b, j]), P, n_pages)
                if there:
                    plain.put(*there, turned[b * T + j, Hq:], x[b * T + j, Hq + Hkv:])
        assert (cache.cpu().numpy() == plain.bytes()).all()
        c.k, c.ks, c.kl, c.v, c.vs, c.vl = plain.k, plain.ks, plain.kl, plain.v, plain.vs, plain.vl
        oracle_bounds(c, table, pos, T, *state)
        assert (bounds.cpu().numpy() == pg.bounds_bytes(*state)).all()
        reference = Bounds(0, n_pages, Hkv, D)
        reference.upper, reference.lower, reference.grid = state
        queries_ = turned[:, :Hq].reshape(Bn, T, Hq, D)
        want = oracle_choice(reference, queries_, pos, table, P, 1, 1, count)
        assert (picked.cpu().numpy() == want).all()
        compare_blocks(out.cpu().numpy().astype(np.float64), c, queries_, pos, table, want)

    length = np.array([300, 190])
    step(length - 300, 300)                                    # the second one's first rows have no place
    for cycle in range(3):
        for j in range(3):
            step(length + j, 1)
        step(length, 4)
        length = length + np.array([1, 3])                     # the next cycle overwrites what was rejected
