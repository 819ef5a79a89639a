"""Attention behind shared beginnings against the oracle in binary64, on the same cache bytes.

How far an output may be off: as in the attention of one sequence (tests/test_gpu_attn_kv4.py), and for the join of the two parts' sums, in
binary32, a dozen roundings of numbers no larger than the values: 16 * 2^-24 of the largest."""
import contextlib

import numpy as np
import pytest

from oracle import kv4_oracle as kv
from tests.test_gpu_attn_kv4 import Cache, dev, queries

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2410_11305_amd import binding as B
    assert torch.cuda.is_available()
    B.lib()
    return torch, B


def tables(seed, groups, per, each, P, shared, n_pages, apart=False):
    """Rows of pages: those that lie whole in the shared tokens are the same in a group (apart: everyone has pages of its own)."""
    free = list(np.random.default_rng(seed).permutation(n_pages))
    rows = []
    for g in range(groups):
        whole = min(max(int(shared[g]), 0) // P, each)
        for i in range(per):
            before = [] if i == 0 or apart else rows[-1][:whole]
            rows.append(before + [free.pop() for _ in range(each - len(before))])
    return np.array(rows)


def sequence(cache, table, shared, per, b, tokens):
    """(k, v, present, value steps) of a sequence's tokens."""
    mine, first = cache.sequence(table[b], tokens), cache.sequence(table[b - b % per], tokens)
    from_first = np.arange(tokens) < shared[b // per]
    pick = lambda a, c: np.where(from_first.reshape(-1, *[1] * (a.ndim - 1)), c, a)
    return [pick(a, c) for a, c in zip(mine, first)]


def compare(got, cache, q, pos, table, shared, scale=None, rows=None):
    Bn, T, Hq, D = q.shape
    per = Bn // len(shared)
    scale = D ** -0.5 if scale is None else scale
    S = table.shape[1] * cache.P
    for b in range(Bn) if rows is None else rows:
        at = np.int64(pos[b]) + np.arange(T)
        tokens = int(min(max(at[-1] + 1, 0), S))
        if tokens == 0:
            assert (got[b] == 0).all()
            continue
        k, v, present, step = sequence(cache, table, shared, per, b, tokens)
        k, v, step = (np.where(present.reshape(-1, *[1] * (a.ndim - 1)), a, 0.0) for a in (k, v, step))
        want = kv.attention(q[b], k, v, present, at, scale)
        size = np.abs(q[b].astype(np.float64)).sum(-1) * scale * (np.abs(k).max() * 2.0)
        spread = np.abs(v).max()
        bound = (2.0 ** -11 * np.abs(want) + 2.0 ** -25 + (2.0 ** -11 * 8 + tokens * 2.0 ** -29) * step.max()
                 + 2 * ((D + 12) * 2.0 ** -24 * size)[..., None] * 2 * spread + 16 * 2.0 ** -24 * spread)
        assert np.isfinite(got[b]).all(), b
        worst = np.abs(got[b] - want) - bound
        assert worst.max() <= 0, (b, np.unravel_index(worst.argmax(), worst.shape), worst.max(), bound.max())
        for j in range(T):
            if not (kv.visible(int(at[j]), tokens, 0, 0) & present).any():
                assert (got[b, j] == 0).all()


def check(env, cache, q, pos, table, shared, scale=None, no_table=False, workspace=None, rows=None, raw=None):
    """Each sequence with its own reading of the shared tokens, and one reading for all of a group."""
    torch, B = env
    with once_for_all(B):
        check_one(env, cache, q, pos, table, shared, scale, no_table, workspace, rows, raw)
    return check_one(env, cache, q, pos, table, shared, scale, no_table, workspace, rows, raw)


@contextlib.contextmanager
def once_for_all(B, tokens=0):
    B.debug_set_plan("QSPEC_ATTN_SHARED", str(tokens))
    try:
        yield
    finally:
        B.debug_set_plan("QSPEC_ATTN_SHARED", None)


def check_one(env, cache, q, pos, table, shared, scale=None, no_table=False, workspace=None, rows=None, raw=None):
    torch, B = env
    Bn, T, Hq, D = q.shape
    guard = torch.full((q.size + 64,), 123.0, dtype=torch.float16, device="cuda")
    out = guard[32:-32].view(Bn, T, Hq, D)
    out.fill_(float("nan"))
    B.attn_kv4_shared(dev(torch, q), dev(torch, cache.bytes() if raw is None else raw), dev(torch, np.asarray(pos, np.int32)), dev(torch, np.asarray(shared, np.int32)),
                      cache.Hkv, cache.P, None if no_table else dev(torch, table.astype(np.int32)), scale, out=out, workspace=workspace)
    torch.cuda.synchronize()
    assert (guard[:32] == 123.0).all() and (guard[-32:] == 123.0).all()
    compare(out.cpu().numpy().astype(np.float64), cache, q, pos, table, shared, scale, rows)
    return out


@pytest.mark.parametrize("groups,per,T,Hq,Hkv,D,P,shared", [
    (1, 4, 1, 4, 4, 128, 16, [37]), (1, 2, 1, 2, 1, 64, 64, [64]), (2, 3, 1, 8, 2, 128, 16, [33, 0]), (1, 8, 4, 4, 4, 64, 32, [70]), (1, 5, 1, 7, 1, 128, 64, [129]),
    (3, 2, 2, 16, 2, 64, 16, [100, 1, 48]), (1, 33, 1, 8, 8, 64, 16, [31]), (1, 2, 17, 4, 2, 128, 32, [90]), (2, 4, 9, 8, 1, 128, 64, [65, 200]), (1, 1, 1, 4, 2, 64, 16, [50]),
    (4, 1, 3, 6, 2, 128, 16, [5, 0, 17, 40]), (1, 70, 1, 20, 1, 64, 64, [150]), (1, 3, 40, 2, 1, 64, 16, [25]), (7, 5, 1, 2, 2, 64, 16, [9, 16, 15, 17, 32, 31, 1])])
def test_groups_rows_and_lengths(env, groups, per, T, Hq, Hkv, D, P, shared):
    """Shared tokens that end inside pages and steps or on their borders; own tokens from the rows of the call alone to a few hundred."""
    rng = np.random.default_rng(per * T + D)
    Bn = groups * per
    own = np.r_[0, rng.integers(0, 200, Bn - 1)]
    pos = np.repeat(shared, per) + own
    each = -(-(int(pos.max()) + T) // P)
    c = Cache(T + D, Bn * each, Hkv, D, P)
    check(env, c, queries(D, Bn, T, Hq, D), pos, tables(1, groups, per, each, P, shared, Bn * each), shared, rows=range(Bn) if Bn <= 20 else range(0, Bn, 7))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("groups,per,T,Hq,Hkv,n", [(1, 18, 1, 16, 8, 700), (3, 6, 4, 16, 8, 90), (2, 9, 2, 64, 8, 1400), (1, 17, 4, 64, 8, 300), (1, 150, 8, 8, 1, 40)])
def test_an_item_to_a_compute_unit(env, groups, per, T, Hq, Hkv, D, n):
    """129 to 256 items, of every size up to 32 rows and more."""
    P, shared, rng = 64, [n - 20 * g for g in range(groups)], np.random.default_rng(n)
    Bn = groups * per
    pos = np.repeat(shared, per) + rng.integers(-3, 900, Bn)
    each = -(-(int(pos.max()) + T) // P)
    table = tables(1, groups, per, each, P, shared, Bn * each)
    used, inverse = np.unique(table, return_inverse=True)
    c = Cache(T + D, len(used), Hkv, D, P)
    check(env, c, queries(D, Bn, T, Hq, D), pos, inverse.reshape(table.shape), shared, rows=range(0, Bn, 5))


@pytest.mark.parametrize("T", [1, 3])
def test_groups_that_share_little_beside_groups_that_share_much(env, T):
    torch, B = env
    P, per, shared, Hkv, D = 64, 3, [700, 40, 0, 399, 400, -3], 2, 64
    rng = np.random.default_rng(T)
    pos = np.repeat(np.maximum(shared, 0), per) + rng.integers(-2, 300, len(shared) * per)
    each = -(-(int(pos.max()) + T) // P)
    table = tables(1, len(shared), per, each, P, shared, len(pos) * each)
    c = Cache(T, len(pos) * each, Hkv, D, P)
    for tokens in (400, 701, 1 << 20):
        with once_for_all(B, tokens):
            check_one(env, c, queries(D, len(pos), T, 4, D), pos, table, shared)


def test_one_long_sequence_among_short_ones(env):
    """Its items have more parts than theirs."""
    P, per, shared, D = 256, 9, [300], 64
    pos = np.array([20011, 300, 310, 400, 299, 5000, 1000, 350, 12345])
    each = -(-(int(pos.max()) + 2) // P)
    table = np.full((per, each), -1)
    for i in range(per):
        table[i, :-(-(int(pos[i]) + 2) // P)] = np.arange(-(-(int(pos[i]) + 2) // P)) + table.max() + 1
    c = Cache(3, int(table.max()) + 1, 16, D, P)
    check(env, c, queries(4, per, 2, 16, D), pos, table, shared)


@pytest.mark.parametrize("T", [1, 6])
def test_rows_in_front_of_the_end_of_what_is_shared(env, T):
    """Rows that see part of the shared tokens, all of them but one, none; idle sequences, the first of its group among them; positions and
    shared numbers past the cache and in front of it."""
    P, each, per = 16, 12, 6
    shared = np.array([100, 3000, -5, 2 ** 31 - 1, -(2 ** 31)])
    pos = np.array([-T, 0, 50, 98, 99, 100,  10, 190, -T, 63, 64, 65,  -1, 0, 20, 150, -T, 191,  5, 80, -(2 ** 31), 2 ** 31 - 1, 192, 200,  30, 31, 32, 33, 34, 35])
    Bn = len(pos)
    c = Cache(3, Bn * each, 2, 64, P)
    table = tables(2, len(shared), per, each, P, np.minimum(shared, each * P), Bn * each)
    check(env, c, queries(4, Bn, T, 6, 64), pos, table, shared)


def test_tables_that_differ_and_no_table(env):
    """What is shared is read through the first row, whatever the others name there."""
    P, each, per, shared = 32, 8, 3, [100, 65]
    pos = np.array([120, 200, 101, 65, 70, 250])
    c = Cache(5, 6 * each, 2, 128, P)
    check(env, c, queries(5, 6, 2, 4, 128), pos, tables(3, 2, per, each, P, shared, 6 * each, apart=True), shared)
    check(env, c, queries(5, 6, 2, 4, 128), pos, np.arange(6 * each).reshape(6, each), shared, no_table=True)


def test_missing_pages(env):
    P, each, n_pages, per, shared = 16, 12, 60, 2, [70, 70]
    table = tables(6, 2, per, each, P, shared, n_pages).astype(np.int64)
    table[0, [1, 5]] = [-1, n_pages]                          # shared ones of the first group
    table[1, [2, 6]] = -7                                     # one that is not read, one of its own
    table[2, :] = 10 ** 6
    c = Cache(7, n_pages, 2, 128, P)
    for T in (1, 5, 20):
        check(env, c, queries(T, 4, T, 4, 128), np.array([160, 120, 100, 90]), table, shared)


@pytest.mark.parametrize("groups,per,T,Hq,Hkv,D,n,own", [(1, 8, 1, 8, 1, 128, 20011, 700), (1, 3, 1, 2, 2, 64, 30000, 5000), (2, 20, 2, 4, 1, 128, 6000, 300), (1, 2, 4, 4, 2, 64, 100, 9000)])
def test_long_sequences_are_shared_out_and_joined(env, groups, per, T, Hq, Hkv, D, n, own):
    torch, B = env
    P, Bn, shared = 256, groups * per, [n - 300 * g for g in range(groups)]
    rng = np.random.default_rng(n)
    pos = np.repeat(shared, per) + rng.integers(0, own, Bn)
    each = -(-(int(pos.max()) + T) // P)
    table = tables(8, groups, per, each, P, shared, Bn * each)
    used = np.unique(table)
    table = np.searchsorted(used, table)                      # (pages that nobody has are left out)
    c = Cache(n, len(used), Hkv, D, P)
    ws = B.alloc_workspace(B.attn_kv4_shared_workspace_bytes(Bn, T, Hq, Hkv, D, groups))
    args = (env, c, queries(n, Bn, T, Hq, D, 2.0), pos, table, shared)
    first = check(*args, workspace=ws, rows=range(0, Bn, 7))
    assert int(ws[:16384].count_nonzero()) == 0
    again = check(*args, workspace=ws, rows=[0])
    assert torch.equal(first, again)
    with once_for_all(B):
        first = check_one(*args, workspace=ws, rows=range(0, Bn, 7))
        assert int(ws[:16384].count_nonzero()) == 0
        assert torch.equal(first, check_one(*args, workspace=ws, rows=[0]))


def test_agrees_with_the_attention_of_each_alone(env):
    """The same tokens in pages of everyone's own."""
    torch, B = env
    P, each, per, T, Hq, Hkv, D = 64, 20, 4, 2, 8, 2, 128
    shared, pos = [777], np.array([800, 1100, 900, 777])
    c = Cache(9, per * each, Hkv, D, P)
    table = np.arange(per * each).reshape(per, each)
    for a in (c.k, c.v, c.ks, c.kl, c.vs, c.vl):
        rows = a.reshape((per, each) + a.shape[1:]).swapaxes(2, 3)
        flat = np.ascontiguousarray(rows).reshape((per, each * P, Hkv) + a.shape[3:])
        flat[1:, :777] = flat[0, :777]
        a[:] = flat.reshape((per * each, P, Hkv) + a.shape[3:]).swapaxes(1, 2)
    q = queries(9, per, T, Hq, D)
    args = [dev(torch, q), dev(torch, c.bytes()), dev(torch, pos.astype(np.int32))]
    alone = B.attn_kv4(*args, Hkv, P, dev(torch, table.astype(np.int32))).float()
    both = B.attn_kv4_shared(*args, dev(torch, np.array(shared, np.int32)), Hkv, P, dev(torch, table.astype(np.int32))).float()
    v = c.sequence(table[0], 800)[3].max()
    # each is off by its weights' rounding about the codes' middle, and by its own
    assert float((alone - both).abs().max()) <= 2 * (2.0 ** -11 * 8 * v + 2.0 ** -11 * float(alone.abs().max()) + 2.0 ** -14)


@pytest.mark.parametrize("T", [1, 4, 20])
def test_rows_nobody_sees_may_hold_anything(env, T):
    """Behind the last token of a sequence, and in its own page's places of the shared tokens."""
    P, each, per, shared, D = 16, 12, 2, [100], 64
    pos = np.array([150 - T, 120 - T])
    table = np.arange(2 * each).reshape(2, each)
    table[1, :6] = table[0, :6]
    c = Cache(9, 2 * each, 1, D, P)
    want = check(env, c, queries(T, 2, T, 3, D), pos, table, shared)
    hidden = np.ones(2 * each * P, bool)
    hidden[:150] = False
    own = each * P + np.arange(100, 120)
    hidden[own] = False
    bad = Cache(9, 2 * each, 1, D, P)
    for a, x in ((bad.ks, np.nan), (bad.kl, np.inf), (bad.vs, np.inf), (bad.vl, np.nan)):
        a.reshape(-1)[hidden] = x
    got = check(env, c, queries(T, 2, T, 3, D), pos, table, shared, raw=bad.bytes())
    torch, _ = env
    assert torch.equal(want, got)
    with once_for_all(env[1]):
        args = (env, c, queries(T, 2, T, 3, D), pos, table, shared)
        assert torch.equal(check_one(*args), check_one(*args, raw=bad.bytes()))


@pytest.mark.parametrize("bad", [60000.0, np.inf, np.nan])
@pytest.mark.parametrize("T,G", [(1, 3), (5, 4), (20, 2)])
def test_idle_sequences_do_not_bring_tokens_in(env, T, G, bad):
    """Shared tokens behind every row, of steps of fp16's largest size or that are no numbers, beside sequences that are not running."""
    P, each, shared, D = 16, 12, [150], 64
    pos = np.array([-T, 40, -T - 5, 60 - T, -T])
    table = tables(5, 1, 5, each, P, shared, 5 * each)
    c = Cache(21, 5 * each, 1, D, P)
    for token in range(max(int(pos.max()) + T, 41 + T), 150):
        c.vs[table[0, token // P], 0, token % P], c.vl[table[0, token // P], 0, token % P] = bad, -bad
        c.ks[table[0, token // P], 0, token % P] = bad
    check(env, c, queries(T, 5, T, G, D), pos, table, shared)


def test_what_is_no_number_shows_where_it_is_seen(env):
    torch, B = env
    P, each, shared, D, Hq, Hkv = 16, 8, [50], 64, 4, 2
    pos = np.array([30, 60, -1, 90])
    table = tables(4, 1, 4, each, P, shared, 4 * each)
    c = Cache(11, 4 * each, Hkv, D, P)
    q = queries(3, 4, 1, Hq, D)

    def run(q, c):
        call = lambda: B.attn_kv4_shared(dev(torch, q), dev(torch, c.bytes()), dev(torch, pos.astype(np.int32)), dev(torch, np.array(shared, np.int32)), Hkv, P,
                                         dev(torch, table.astype(np.int32))).isnan().cpu().numpy()
        one = call()
        with once_for_all(B):
            two = call()
        assert (one == two).all()
        return one

    odd = q.copy()
    odd[1, 0, 2, 5], odd[2, 0, 0, 0] = np.nan, np.inf
    got = run(odd, c)
    want = np.zeros(got.shape, bool)
    want[1, 0, 2] = True                                      # (a row that sees nothing gets zeros, whatever its query)
    assert (got == want).all()
    for token, which in ((40, "ks"), (10, "vl")):             # a shared token: of the rows at or behind it
        d = Cache(11, 4 * each, Hkv, D, P)
        getattr(d, which)[table[0, token // P], 1, token % P] = np.nan
        got = run(q, d)
        want = np.zeros(got.shape, bool)
        want[pos >= token, 0, 2:] = True
        assert (got == want).all(), token
    d = Cache(11, 4 * each, Hkv, D, P)
    d.vs[table[3, 70 // P], 0, 70 % P] = np.nan               # a token of the last sequence's own
    got = run(q, d)
    want = np.zeros(got.shape, bool)
    want[3, 0, :2] = True
    assert (got == want).all()


@pytest.mark.parametrize("tokens", [0, 900, 1 << 30])
def test_two_streams_with_a_workspace_each_and_a_graph(env, tokens):
    """One reading of the shared tokens for all of a group, of the groups that share 900 and more, of none."""
    with once_for_all(env[1], tokens):
        two_streams_and_a_graph(env)


def two_streams_and_a_graph(env):
    torch, B = env
    groups, per, T, Hq, Hkv, D, P, n = 2, 3, 4, 8, 2, 128, 64, 2500
    Bn, each = groups * per, -(-n // P)
    c = Cache(20, Bn * each, Hkv, D, P)
    table = np.random.default_rng(1).permutation(Bn * each).reshape(Bn, each)
    cache, tab = dev(torch, c.bytes()), dev(torch, table.astype(np.int32))
    pos = torch.tensor([2400, 2000, 2100, 1000, 1500, 2496], dtype=torch.int32, device="cuda")
    shared = torch.tensor([1999, 1000], dtype=torch.int32, device="cuda")
    size = B.attn_kv4_shared_workspace_bytes(Bn, T, Hq, Hkv, D, groups)
    q = dev(torch, queries(21, Bn, T, Hq, D))
    outs, works = [torch.empty_like(q) for _ in range(3)], [B.alloc_workspace(size) for _ in range(3)]
    call = lambda i: B.attn_kv4_shared(q, cache, pos, shared, Hkv, P, tab, out=outs[i], workspace=works[i])
    sides = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        for i, s in enumerate(sides):
            with torch.cuda.stream(s):
                call(i)
    call(2)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[2]) and torch.equal(outs[1], outs[2])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(0)
    rng = np.random.default_rng(22)
    for r in range(4):
        q_new = queries(30 + r, Bn, T, Hq, D)
        q.copy_(dev(torch, q_new))
        sh = rng.integers(0, 1500, groups)
        at = rng.integers(0, n - T, Bn)
        pos.copy_(dev(torch, at.astype(np.int32)))
        shared.copy_(dev(torch, sh.astype(np.int32)))
        outs[0].fill_(float("nan"))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        call(2)
        torch.cuda.synchronize()
        assert torch.equal(outs[0], outs[2])
        compare(outs[0].cpu().numpy().astype(np.float64), c, q_new, at, table, sh)
        assert int(works[0][:16384].count_nonzero()) == 0


@pytest.mark.parametrize("what", ["zero", "constant", "subnormal", "huge", "mixed", "shared large", "own large"])
def test_value_steps_of_every_size(env, what):
    """Constant rows, fp16's smallest and largest, and the two parts' sums on references that lie far apart."""
    P, each, per, shared, D, Hkv = 64, 16, 3, [500], 128, 2
    pos = np.array([900, 520, 1000])
    table = tables(1, 1, per, each, P, shared, per * each)
    c = Cache(10, per * each, Hkv, D, P)
    if what == "zero":
        c.vs[:], c.vl[:], c.ks[:], c.kl[:] = 0, 0, 0, 0
    elif what == "constant":
        c.vs[:] = 0
    elif what == "subnormal":
        c.vs[:], c.vl[:] = 2.0 ** -24, -7 * 2.0 ** -24
    elif what == "huge":
        c.vs[:], c.vl[:] = 8000.0, -60000.0
    elif what == "mixed":
        c.vs[:] = (2.0 ** np.random.default_rng(1).integers(-20, 12, c.vs.shape)).astype(np.float16)
        c.vl[:] = -8 * c.vs.astype(np.float32)
    else:
        first = np.zeros(per * each, bool)
        first[table[0, :8]] = True
        large = first if what == "shared large" else ~first
        c.vs[large], c.vs[~large] = 1000.0, 2.0 ** -20
        c.vl[large], c.vl[~large] = -8000.0, 0.0
    check(env, c, queries(11, per, 2, 4, D), pos, table, shared)


@pytest.mark.parametrize("size,scale", [(0.0, None), (60.0, None), (1e-3, 100.0), (2.0 ** -24, 1e6), (1.0, 1e-6)])
def test_queries_of_every_size(env, size, scale):
    P, each, per, shared, D = 32, 20, 3, [300], 128
    c = Cache(12, per * each, 2, D, P)
    check(env, c, queries(13, per, 3, 4, D, size), np.array([600, 310, 200]), tables(2, 1, per, each, P, shared, per * each), shared, scale=scale)


def test_caches_of_more_than_four_gib(env):
    """The pages at both ends and past the 32-bit offsets: shared attention, bounds, attention over chosen pages."""
    torch, B = env
    from oracle import kv4_pages_oracle as pg
    from tests.test_gpu_kv4_pages import Bounds, compare_blocks, empty_bounds, oracle_bounds, oracle_choice
    P, Hkv, D, each, T, Hq = 256, 8, 128, 2, 2, 16
    page = B.kv4_page_bytes(Hkv, D, P)
    n_pages = (5 << 30) // page
    small = Cache(17, 4, Hkv, D, P)
    cache, bounds = torch.zeros((n_pages, page), dtype=torch.uint8, device="cuda"), B.alloc_kv4_bounds(n_pages, Hkv, D)
    where = np.array([n_pages - 1, 3, n_pages // 2 + 1, n_pages - 7])
    cache[torch.from_numpy(where).cuda()] = dev(torch, small.bytes())
    table, small_table = where[[[0, 1], [0, 2]]], np.array([[0, 1], [0, 2]])
    q, pos = queries(18, 2, T, Hq, D), np.array([500, 400])
    at, tab = dev(torch, pos.astype(np.int32)), dev(torch, table.astype(np.int32))
    shared = [300]
    small.k[2, :, :44], small.v[2, :, :44] = 0, 0             # (not read: shared)
    for tokens in (0, 1 << 30):
        with once_for_all(B, tokens):
            got = B.attn_kv4_shared(dev(torch, q), cache, at, dev(torch, np.array(shared, np.int32)), Hkv, P, tab)
        compare(got.cpu().numpy().astype(np.float64), small, q, pos, small_table, shared)
    small = Cache(17, 4, Hkv, D, P)
    one = dev(torch, np.array([[where[3], where[0]], [where[2], where[1]]], dtype=np.int32))
    own = np.array([[3, 0], [2, 1]])
    B.kv4_bounds(cache, dev(torch, np.zeros(2, np.int32)), 500, bounds, Hkv, D, P, one)
    state = empty_bounds(small)
    oracle_bounds(small, own, np.zeros(2, np.int64), 500, *state)
    assert (bounds[torch.from_numpy(where).cuda()].cpu().numpy() == pg.bounds_bytes(*state)).all()
    picked = B.kv4_select(dev(torch, q), bounds, at, Hkv, P, 1, one, first=0, last=0)
    reference = Bounds(0, 4, Hkv, D)
    reference.upper, reference.lower, reference.grid = state
    want = oracle_choice(reference, q, pos, own, P, 0, 0, 1)
    assert (picked.cpu().numpy() == want).all()
    got = B.attn_kv4_blocks(dev(torch, q), cache, at, picked, Hkv, P, one)
    compare_blocks(got.cpu().numpy().astype(np.float64), small, q, pos, own, want)


def test_one_workspace_serves_all_in_turn(env):
    torch, B = env
    from paper_2410_11305_amd import synth
    M, N, K = 200, 1024, 4096
    codes, scales, x = synth.generic_case(23, M, N, K)
    blob, xd = B.pack_weights(dev(torch, codes), dev(torch, scales)), dev(torch, x)
    c = Cache(24, 40, 2, 128, 64)
    cache, pos, q = dev(torch, c.bytes()), torch.tensor([2500, 2000], dtype=torch.int32, device="cuda"), dev(torch, queries(25, 2, 1, 8, 128))
    table = torch.arange(40, dtype=torch.int32, device="cuda").repeat(2, 1)

    def shared_once(w):
        with once_for_all(B):
            return B.attn_kv4_shared(q, cache, pos, shared, 2, 64, table, workspace=w)

    shared = torch.tensor([1900], dtype=torch.int32, device="cuda")
    blocks = torch.arange(0, 40, 2, dtype=torch.int32, device="cuda").repeat(2, 1, 2, 1)
    ws = B.alloc_workspace(max(B.workspace_bytes(M, N, K), B.attn_kv4_workspace_bytes(2, 1, 8, 2, 128), B.attn_kv4_shared_workspace_bytes(2, 1, 8, 2, 128, 1),
                               B.attn_kv4_blocks_workspace_bytes(2, 1, 8, 2, 128)))
    calls = [lambda w: B.gemm_w4a16(blob, xd, N, workspace=w), lambda w: B.attn_kv4(q, cache, pos, 2, 64, table, workspace=w),
             lambda w: B.attn_kv4_shared(q, cache, pos, shared, 2, 64, table, workspace=w), shared_once,
             lambda w: B.attn_kv4_blocks(q, cache, pos, blocks, 2, 64, table, workspace=w)]
    alone = [call(None) for call in calls]
    for _ in range(3):
        for call, want in zip(calls, alone):
            assert torch.equal(call(ws), want)
            assert int(ws[:16384].count_nonzero()) == 0


def test_tensors_that_do_not_fit_are_refused(env):
    torch, B = env
    cache, pos, q = B.alloc_kv4_cache(8, 2, 64, 64), torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros((2, 1, 4, 64), dtype=torch.float16, device="cuda")
    bounds, shared, blocks = B.alloc_kv4_bounds(8, 2, 64), torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros((2, 1, 2, 3), dtype=torch.int32, device="cuda")
    bad = [lambda: B.attn_kv4_shared(q, cache, pos, shared.long(), 2, 64), lambda: B.attn_kv4_shared(q, cache, pos, shared.cpu(), 2, 64), lambda: B.attn_kv4_shared(q.float(), cache, pos, shared, 2, 64),
           lambda: B.attn_kv4_shared(q, cache, pos, shared, 2, 64, out=q[:1]), lambda: B.attn_kv4_blocks(q, cache, pos, blocks[:, :, :1], 2, 64), lambda: B.attn_kv4_blocks(q, cache, pos, blocks.long(), 2, 64),
           lambda: B.attn_kv4_blocks(q, cache, pos, blocks.transpose(1, 2), 2, 64), lambda: B.kv4_bounds(cache, pos, 1, bounds[:4], 2, 64, 64), lambda: B.kv4_bounds(cache, pos, 1, bounds[:, 16:], 2, 64, 64),
           lambda: B.kv4_bounds_read(bounds, pos, 1, 2, 64, 64, upper=torch.zeros((2, 1, 2, 64), device="cuda")), lambda: B.kv4_select(q, bounds, pos, 2, 64, 3, blocks=blocks[..., :2]),
           lambda: B.kv4_select(q, bounds, pos, 2, 64, 3, page_table=torch.zeros((3, 4), dtype=torch.int32, device="cuda")), lambda: B.kv4_select(q, bounds.float(), pos, 2, 64, 3)]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    for call in (lambda: B.attn_kv4_shared(q, cache, pos, torch.zeros(3, dtype=torch.int32, device="cuda"), 2, 64), lambda: B.kv4_select(q, bounds, pos, 2, 64, 3, first=2, last=2),
                 lambda: B.kv4_select(q, bounds, pos, 2, 64, 0), lambda: B.attn_kv4_blocks(q, B.alloc_kv4_cache(8, 2, 64, 32), pos, blocks, 2, 32)):
        with pytest.raises(B.QSpecError):
            call()
