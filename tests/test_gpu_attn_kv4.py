"""Attention over the 4-bit cache against the oracle in binary64, on the same cache bytes.

How far an output may be off (derived from the arithmetic, nothing measured):
  fp16 result                      2^-11 of it (and half the smallest subnormal)
  weights rounded to fp16          2^-11 of a weight times a code about its middle, 8 steps at most: 2^-11 * 8 * largest step;
                                   weights below fp16's normal range are off by 2^-25 where the largest is 2^7 or more
  scores in binary32               D products and a few more operations on magnitudes that sum to S: (D + 12) 2^-24 S of a
                                   logarithm of a weight, on either side of the quotient, times the spread of the values
"""
import numpy as np
import pytest

from oracle import kv4_oracle as kv
from tests.test_attn_division import NEIGHBOURS

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2410_11305_amd import binding as B
    assert torch.cuda.is_available()
    B.lib()
    return torch, B


def dev(torch, a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


class Cache:
    """Random pages: codes, steps and lows, the bytes, and what a sequence reads from them."""

    def __init__(self, seed, n_pages, Hkv, D, P, spread=1.0):
        rng = np.random.default_rng(seed)
        self.n_pages, self.Hkv, self.D, self.P = n_pages, Hkv, D, P
        self.k, self.v = (rng.integers(0, 16, (n_pages, Hkv, P, D)).astype(np.uint8) for _ in range(2))
        step = lambda: (rng.uniform(0.1, 0.4, (n_pages, Hkv, P)) * spread).astype(np.float16)
        self.ks, self.vs = step(), step()
        self.kl = (-self.ks.astype(np.float32) * rng.uniform(6, 9, self.ks.shape)).astype(np.float16)
        self.vl = (-self.vs.astype(np.float32) * rng.uniform(6, 9, self.vs.shape)).astype(np.float16)

    def bytes(self):
        return kv.cache_bytes(self.k, self.ks, self.kl, self.v, self.vs, self.vl, self.P)

    def sequence(self, row, tokens):
        """(k, v, present, largest value step) of the first `tokens` tokens of a table's row."""
        n = -(-tokens // self.P)
        there = np.array([0 <= p < self.n_pages for p in row[:n]], dtype=bool)
        pages = np.where(there, row[:n], 0).astype(np.int64)
        flat = lambda a: a[pages].swapaxes(1, 2).reshape((n * self.P,) + a.shape[1:2] + a.shape[3:])[:tokens]
        k = kv.values(flat(self.k), flat(self.ks), flat(self.kl))
        v = kv.values(flat(self.v), flat(self.vs), flat(self.vl))
        return k, v, np.repeat(there, self.P)[:tokens], flat(self.vs).astype(np.float64)


def check(env, cache, q, pos, table, scale=None, window=0, sinks=0, no_table=False, workspace=None, poison=None, rows=None):
    """Runs the call and compares; returns the output."""
    torch, B = env
    Bn, T, Hq, D = q.shape
    raw = cache.bytes()
    if poison is not None:
        raw = poison(raw)
    guard = torch.full((q.size + 64,), 123.0, dtype=torch.float16, device="cuda")
    out = guard[32:-32].view(Bn, T, Hq, D)
    out.fill_(float("nan"))
    B.attn_kv4(dev(torch, q), dev(torch, raw), dev(torch, pos.astype(np.int32)), cache.Hkv, cache.P, None if no_table else dev(torch, table.astype(np.int32)),
               scale, window, sinks, out=out, workspace=workspace)
    torch.cuda.synchronize()
    assert (guard[:32] == 123.0).all() and (guard[-32:] == 123.0).all()
    got = out.cpu().numpy().astype(np.float64)
    compare(got, cache, q, pos, table, scale, window, sinks, rows)
    return out


def compare(got, cache, q, pos, table, scale, window, sinks, rows=None):
    Bn, T, Hq, D = q.shape
    scale = D ** -0.5 if scale is None else scale
    S = table.shape[1] * cache.P
    group = Hq // cache.Hkv
    for b in range(Bn) if rows is None else rows:
        at = np.int64(pos[b]) + np.arange(T)
        tokens = int(min(max(at[-1] + 1, 0), S))
        if tokens == 0:
            assert (got[b] == 0).all()
            continue
        k, v, present, step = cache.sequence(table[b], tokens)
        seen = np.zeros(tokens, bool)
        for p in at:
            seen |= kv.visible(int(p), tokens, window, sinks) & present
        k, v, step = (np.where(seen.reshape(-1, *[1] * (a.ndim - 1)), a, 0.0) for a in (k, v, step))
        want = kv.attention(q[b], k, v, present, at, scale, window, sinks)
        size = np.abs(q[b].astype(np.float64)).sum(-1) * scale * (np.abs(k).max() * 2.0)             # magnitudes before they cancel: code * step and low
        spread = np.abs(v).max()
        bound = (2.0 ** -11 * np.abs(want) + 2.0 ** -25 + (2.0 ** -11 * 8 + tokens * 2.0 ** -29) * step.max()
                 + 2 * ((D + 12) * 2.0 ** -24 * size)[..., None] * 2 * spread)
        assert np.isfinite(got[b]).all(), b
        worst = np.abs(got[b] - want) - bound
        assert worst.max() <= 0, (b, np.unravel_index(worst.argmax(), worst.shape), worst.max(), bound.max())
        for j in range(T):
            if not (kv.visible(int(at[j]), tokens, window, sinks) & present).any():
                assert (got[b, j] == 0).all()


def queries(seed, Bn, T, Hq, D, size=1.0):
    return (np.random.default_rng(seed).standard_normal((Bn, T, Hq, D)) * size).astype(np.float16)


def shuffled(seed, Bn, each, n_pages):
    return np.random.default_rng(seed).permutation(n_pages)[:Bn * each].reshape(Bn, each)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 255, 256, 257])
def test_one_token_over_short_caches(env, D, n):
    each = -(-n // 16) + 1
    c = Cache(n + D, 3 * each + 2, 2, D, 16)
    check(env, c, queries(n, 3, 1, 4, D), np.array([n - 1, 0, n // 2]), shuffled(1, 3, each, 3 * each + 2))


@pytest.mark.parametrize("Bn,T,Hq,Hkv,D,P,n", [
    (2, 4, 8, 8, 128, 64, 200), (1, 5, 32, 32, 128, 64, 600), (3, 4, 8, 1, 128, 32, 300), (2, 3, 7, 1, 64, 16, 100), (1, 9, 16, 2, 64, 256, 500),
    (2, 16, 4, 4, 128, 16, 40), (2, 17, 4, 4, 128, 16, 40), (1, 33, 4, 4, 64, 32, 90), (1, 64, 4, 2, 128, 64, 70), (1, 100, 8, 2, 64, 64, 100),
    (1, 67, 3, 3, 128, 128, 400), (5, 2, 40, 8, 128, 64, 700), (40, 1, 4, 2, 64, 16, 90), (300, 1, 2, 2, 64, 16, 30), (600, 2, 1, 1, 64, 16, 20), (1, 1, 128, 1, 64, 16, 50)])
def test_rows_heads_and_lengths(env, Bn, T, Hq, Hkv, D, P, n):
    """n tokens at most, the first sequence the longest; the pages end inside a step, the steps inside a page."""
    rng = np.random.default_rng(Bn + T)
    pos = np.r_[n - T, rng.integers(-1, n - T + 1, Bn - 1)]
    each = -(-n // P)
    c = Cache(T + D, Bn * each + 1, Hkv, D, P)
    check(env, c, queries(D, Bn, T, Hq, D), pos, shuffled(T, Bn, each, Bn * each + 1), rows=range(Bn) if Bn <= 40 else range(0, Bn, 17))


@pytest.mark.parametrize("window,sinks", [(1, 0), (16, 0), (33, 0), (100, 4), (37, 40), (300, 1), (64, 300), (5000, 3), (40, 16), (7, 500)])
@pytest.mark.parametrize("T,G,D", [(1, 1, 128), (5, 4, 64), (70, 1, 128)])
def test_windows_and_sinks(env, window, sinks, T, G, D):
    n = 700
    c = Cache(window + T, 45, 1, D, 32)
    check(env, c, queries(window, 2, T, G, D), np.array([n - T, 120 - T]), shuffled(2, 2, 22, 45), window=window, sinks=sinks)


@pytest.mark.parametrize("Bn,T,Hq,Hkv,D,n,window", [(1, 1, 8, 1, 128, 20000, 0), (1, 1, 1, 1, 64, 30011, 0), (2, 4, 4, 2, 64, 9000, 0), (1, 40, 2, 1, 128, 6000, 0),
                                                   (3, 2, 16, 2, 128, 4000, 3500), (1, 8, 4, 1, 64, 12345, 9000), (1, 3, 2, 2, 128, 1100, 0)])
def test_long_sequences_are_shared_out_and_joined(env, Bn, T, Hq, Hkv, D, n, window):
    torch, B = env
    each = -(-n // 256)
    c = Cache(n, Bn * each, Hkv, D, 256)
    ws = B.alloc_workspace(B.attn_kv4_workspace_bytes(Bn, T, Hq, Hkv, D))
    pos = np.array([n - T, n // 2, n - 300][:Bn])
    args = (env, c, queries(n, Bn, T, Hq, D, 2.0), pos, shuffled(3, Bn, each, Bn * each), None, window, 4 if window else 0)
    first = check(*args, workspace=ws)
    assert int(ws[:16384].count_nonzero()) == 0
    again = check(*args, workspace=ws)                        # the counters are back at zero, and the order of arrival does not show
    assert torch.equal(first, again)


def test_lengths_of_every_kind_side_by_side(env):
    """Idle, empty, one token, a full cache, positions past its end, one long sequence among short ones."""
    T, P, each = 3, 16, 200
    pos = np.array([-3, -2, -(2 ** 31), 0, 3197, 3198, 3300, 5, 3000, 2 ** 31 - 5, 40, -1])
    Bn = len(pos)
    c = Cache(5, Bn * each, 2, 64, P)
    table = shuffled(4, Bn, each, Bn * each)
    for window, sinks in ((0, 0), (50, 2)):
        check(env, c, queries(6, Bn, T, 6, 64), pos, table, window=window, sinks=sinks)


def test_missing_pages(env):
    """Entries outside the cache: their tokens are not there; a sequence without any page."""
    P, each, n_pages = 16, 12, 40
    table = shuffled(5, 3, each, n_pages).astype(np.int64)
    table[0, [0, 3, 4, 11]] = [-1, n_pages, 2 ** 31 - 1, -(2 ** 31)]
    table[1, :] = -1
    table[2, 5:] = 10 ** 6
    c = Cache(7, n_pages, 2, 128, P)
    for T in (1, 5, 20):
        check(env, c, queries(T, 3, T, 4, 128), np.array([190 - T, 150, 100]), table)
    check(env, c, queries(2, 3, 1, 4, 128), np.array([190, 150, 100]), table, window=30, sinks=3)


def test_pages_in_sequence_order(env):
    c = Cache(8, 12, 2, 64, 64)
    check(env, c, queries(3, 3, 2, 4, 64), np.array([254, 0, 100]), np.arange(12).reshape(3, 4), no_table=True)


@pytest.mark.parametrize("T", [1, 4, 40])
def test_rows_nobody_sees_may_hold_anything(env, T):
    """NaN and infinities in the steps and lows behind the last token, in front of the window, and in pages of others."""
    P, each, n, D = 16, 20, 250, 64
    table = np.arange(each).reshape(1, each)
    c = Cache(9, each + 2, 1, D, P)
    for window in (0, 60):
        hidden = np.ones((each + 2) * P, bool)
        for p in range(n - T, n):
            hidden[:each * P] &= ~kv.visible(p, each * P, window, 3 if window else 0)
        c2 = Cache(9, each + 2, 1, D, P)
        for a, bad in ((c2.ks, np.nan), (c2.kl, np.inf), (c2.vs, np.inf), (c2.vl, np.nan)):
            a.reshape(-1)[hidden] = bad
        check(env, c, queries(T, 1, T, 3, D), np.array([n - T]), table, window=window, sinks=3 if window else 0, poison=lambda raw: c2.bytes())


@pytest.mark.parametrize("what", ["zero", "constant", "subnormal", "huge", "mixed", "late"])
def test_value_steps_of_every_size(env, what):
    """Steps of zero (constant rows), fp16's smallest and largest, and a large one that turns up late."""
    n, D, P = 1000, 128, 64
    c = Cache(10, 16, 2, D, P)
    if what == "zero":
        c.vs[:], c.vl[:], c.ks[:], c.kl[:] = 0, 0, 0, 0
    elif what == "constant":
        c.vs[:] = 0
    elif what == "subnormal":
        c.vs[:], c.vl[:] = 2.0 ** -24, -7 * 2.0 ** -24
    elif what == "huge":
        c.vs[:] = 8000.0
        c.vl[:] = -60000.0
    elif what == "mixed":
        c.vs[:] = (2.0 ** np.random.default_rng(1).integers(-20, 12, c.vs.shape)).astype(np.float16)
        c.vl[:] = -8 * c.vs.astype(np.float32)
    else:
        c.vs[:12], c.vs[12:] = 2.0 ** -20, 1000.0
        c.vl[:12], c.vl[12:] = 0.0, -8000.0
    check(env, c, queries(11, 1, 2, 4, D), np.array([n - 2]), np.arange(16).reshape(1, 16))


@pytest.mark.parametrize("size,scale", [(0.0, None), (60.0, None), (1e-3, 100.0), (2.0 ** -24, 1e6), (600.0, 1e-3), (1.0, 1e-6)])
def test_queries_of_every_size(env, size, scale):
    """Zeros (every token weighs the same), scores of hundreds (one token weighs everything), subnormals."""
    c = Cache(12, 20, 2, 128, 32)
    check(env, c, queries(13, 1, 3, 4, 128, size), np.array([600]), np.arange(20).reshape(1, 20), scale=scale)


def test_one_large_feature(env):
    """A feature thousands of times the others: the common factor of a row keeps the small ones."""
    q = queries(14, 1, 2, 2, 128)
    q[..., 7] = 30000.0
    c = Cache(15, 10, 1, 128, 32)
    c.k[..., 7] = 5                                           # the same for every token, so that the others decide
    c.ks[:], c.kl[:] = 0.25, -2.0
    check(env, c, q, np.array([300]), np.arange(10).reshape(1, 10))


def test_rising_scores_move_the_reference(env):
    """Keys that score higher and higher: the running maximum moves all the way."""
    n, D, P = 2048, 64, 64
    c = Cache(16, 32, 1, D, P)
    c.k[:] = 8
    c.ks[:] = np.linspace(0.01, 2.0, n).reshape(32, 1, P).astype(np.float16)
    c.kl[:] = 0
    check(env, c, np.full((1, 1, 2, D), 1.0, np.float16), np.array([n - 1]), np.arange(32).reshape(1, 32))
    c.ks[:] = c.ks[::-1, :, ::-1].copy()
    check(env, c, np.full((1, 1, 2, D), 1.0, np.float16), np.array([n - 1]), np.arange(32).reshape(1, 32))


def test_cache_of_more_than_four_gib(env):
    torch, B = env
    P, Hkv, D, each = 256, 8, 128, 2
    page = B.kv4_page_bytes(Hkv, D, P)
    n_pages = (5 << 30) // page
    small = Cache(17, 4, Hkv, D, P)
    cache = torch.zeros((n_pages, page), dtype=torch.uint8, device="cuda")
    where = [n_pages - 1, 3, n_pages // 2 + 1, n_pages - 7]
    cache[torch.tensor(where, device="cuda")] = dev(torch, small.bytes())
    table = np.array([[where[0], where[1]], [where[2], where[3]]])
    q, pos = queries(18, 2, 2, 16, D), np.array([500, 300])
    got = B.attn_kv4(dev(torch, q), cache, dev(torch, pos.astype(np.int32)), Hkv, P, dev(torch, table.astype(np.int32)))
    compare(got.cpu().numpy().astype(np.float64), small, q, pos, np.array([[0, 1], [2, 3]]), None, 0, 0)
    # the append finds the same places
    qkv = np.random.default_rng(19).standard_normal((2, 1, (16 + 2 * Hkv) * D)).astype(np.float16)
    B.rope_kv4_append(dev(torch, qkv), None, dev(torch, pos.astype(np.int32)), cache, 16, Hkv, P, dev(torch, table.astype(np.int32)))
    raw = cache[torch.tensor(where, device="cuda")].cpu().numpy()
    for b in range(2):
        page_at, slot = b * 2 + int(pos[b]) // P, int(pos[b]) % P
        heads = qkv[b, 0].reshape(-1, D)
        small.k[page_at, :, slot], small.ks[page_at, :, slot], small.kl[page_at, :, slot] = kv.quantise(heads[16:16 + Hkv])
        small.v[page_at, :, slot], small.vs[page_at, :, slot], small.vl[page_at, :, slot] = kv.quantise(heads[16 + Hkv:])
    assert (raw == small.bytes()).all()


def test_two_streams_with_a_workspace_each_and_a_graph(env):
    torch, B = env
    Bn, T, Hq, Hkv, D, P, n = 2, 4, 8, 2, 128, 64, 3000
    each = -(-n // P)
    c = Cache(20, Bn * each, Hkv, D, P)
    table = shuffled(6, Bn, each, Bn * each)
    cache, tab = dev(torch, c.bytes()), dev(torch, table.astype(np.int32))
    pos = torch.tensor([n - T, 1000], dtype=torch.int32, device="cuda")
    size = B.attn_kv4_workspace_bytes(Bn, T, Hq, Hkv, D)
    q = dev(torch, queries(21, Bn, T, Hq, D))
    outs, works = [torch.empty_like(q) for _ in range(3)], [B.alloc_workspace(size) for _ in range(3)]
    call = lambda i: B.attn_kv4(q, cache, pos, Hkv, P, tab, out=outs[i], workspace=works[i])
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
        at = rng.integers(0, n - T, Bn)
        pos.copy_(dev(torch, at.astype(np.int32)))
        outs[0].fill_(float("nan"))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        call(2)
        torch.cuda.synchronize()
        assert torch.equal(outs[0], outs[2])
        compare(outs[0].cpu().numpy().astype(np.float64), c, q_new, at, table, None, 0, 0)
        assert int(works[0][:16384].count_nonzero()) == 0


def test_one_workspace_serves_products_and_attention_in_turn(env):
    torch, B = env
    from paper_2410_11305_amd import synth
    M, N, K = 200, 1024, 4096
    codes, scales, x = synth.generic_case(23, M, N, K)
    blob, xd = B.pack_weights(dev(torch, codes), dev(torch, scales)), dev(torch, x)
    c = Cache(24, 40, 2, 128, 64)
    cache, pos, q = dev(torch, c.bytes()), torch.tensor([2500], dtype=torch.int32, device="cuda"), dev(torch, queries(25, 1, 1, 8, 128))
    ws = B.alloc_workspace(max(B.workspace_bytes(M, N, K), B.attn_kv4_workspace_bytes(1, 1, 8, 2, 128)))
    own = B.gemm_w4a16(blob, xd, N), B.attn_kv4(q, cache, pos, 2, 64)
    for _ in range(3):
        y = B.gemm_w4a16(blob, xd, N, workspace=ws)
        o = B.attn_kv4(q, cache, pos, 2, 64, workspace=ws)
        assert torch.equal(y, own[0]) and torch.equal(o, own[1])


def test_binding_checks_shapes_on_the_device(env):
    torch, B = env
    c = Cache(26, 4, 2, 64, 16)
    good = dict(q=dev(torch, queries(1, 2, 1, 4, 64)), cache=dev(torch, c.bytes()), pos=torch.zeros(2, dtype=torch.int32, device="cuda"), Hkv=2, page_size=16)
    B.attn_kv4(**good)
    for bad in (dict(q=good["q"][:1]), dict(q=good["q"].float()), dict(pos=good["pos"].long()), dict(cache=good["cache"][:, :-16]),
                dict(page_table=torch.zeros((2, 2), dtype=torch.int64, device="cuda")), dict(out=torch.empty((2, 1, 4, 128), dtype=torch.float16, device="cuda")),
                dict(q=torch.cat((good["q"], good["q"]), -1)[..., ::2]), dict(workspace=torch.empty(100, device="cuda"))):
        with pytest.raises(ValueError):
            B.attn_kv4(**{**good, **bad})
    with pytest.raises(B.QSpecError) as e:
        B.attn_kv4(**{**good, "workspace": B.alloc_workspace(1024)})
    assert e.value.status == B.ERR_WORKSPACE
    for bad in (dict(Hkv=3), dict(page_size=24), dict(window=-1), dict(sinks=2), dict(scale=0.0)):
        with pytest.raises((B.QSpecError, ValueError)):
            B.attn_kv4(**{**good, **bad})


def test_as_many_query_heads_to_a_key_head_as_are_taken(env):
    """255, and rows that the blocks of rows cut inside a token."""
    c = Cache(11, 9, 2, 64, 32)
    check(env, c, queries(12, 1, 3, 510, 64), np.array([250]), shuffled(5, 1, 9, 9))


def test_thousands_of_sequences(env):
    """More entries than lanes many times over, most of them idle."""
    Bn, P = 5000, 16
    rng = np.random.default_rng(13)
    pos = np.where(rng.random(Bn) < 0.9, -1, rng.integers(0, 16, Bn))
    pos[[0, 7, Bn - 1]] = 15, 0, 3
    c = Cache(14, 64, 1, 64, P)
    table = rng.integers(0, 64, (Bn, 1))                       # (pages may be read by many)
    check(env, c, queries(15, Bn, 1, 2, 64), pos, table, rows=np.r_[0, 7, Bn - 1, range(0, Bn, 119)])


@pytest.mark.parametrize("Bn,T,Hq,Hkv,D,first", [(2, 300, 64, 64, 64, (0, 0)), (2, 300, 64, 64, 64, (0, 9)), (1, 1100, 32, 32, 64, (0,)), (3, 200, 50, 50, 128, (5, 5, 5)),
                                                (1, 700, 96, 48, 64, (-40,)), (1, 330, 90, 90, 64, (900,)), (4, 1000, 8, 8, 64, (0, 0, 0, 0))])
def test_prompts_of_more_blocks_than_workgroups(env, Bn, T, Hq, Hkv, D, first):
    """Blocks of rows that are dealt out whole, and (lengths or histories that differ) ones that are not."""
    torch, B = env
    P, n = 64, T + max(first)
    each = -(-n // P)
    c = Cache(T, Bn * each, Hkv, D, P)
    args = (env, c, queries(T, Bn, T, Hq, D), np.array(first), shuffled(T, Bn, each, Bn * each))
    ws = B.alloc_workspace(B.attn_kv4_workspace_bytes(Bn, T, Hq, Hkv, D))
    a = check(*args, workspace=ws, rows=[0, Bn - 1])
    assert torch.equal(a, check(*args, workspace=ws, rows=[0])) and int(ws[:16384].count_nonzero()) == 0
    check(*args, window=150, sinks=3, workspace=ws, rows=[0])


@pytest.mark.parametrize("Bn,T,Hq,Hkv,D,n", [(130, 1, 5, 5, 64, 90), (256, 1, 6, 3, 64, 70), (90, 6, 8, 8, 128, 100), (66, 3, 64, 8, 64, 150), (80, 20, 7, 7, 64, 90),
                                            (40, 40, 14, 14, 64, 60), (120, 4, 40, 5, 128, 60)])
@pytest.mark.parametrize("lengths", ["alike", "ragged", "one long"])
def test_batches_of_more_items_than_workgroups(env, Bn, T, Hq, Hkv, D, n, lengths):
    """Items that are dealt out whole in the order of their lengths, and ones that are not."""
    torch, B = env
    rng = np.random.default_rng(Bn)
    pos = np.full(Bn, n - T) if lengths == "alike" else rng.integers(-T, n - T + 1, Bn)
    P, each = 64, -(-n // 64)
    table = shuffled(T, Bn, each, Bn * each)
    if lengths == "one long":
        pos[5], each = 3000, 48
        table = np.c_[table, rng.integers(0, Bn * table.shape[1], (Bn, each - table.shape[1]))]
    c = Cache(T + Hq, Bn * -(-n // 64), Hkv, D, P)
    args = (env, c, queries(T, Bn, T, Hq, D), pos, table)
    first = check(*args, rows=[0, 5, Bn // 2, Bn - 1])
    assert torch.equal(first, check(*args, rows=[0]))


@pytest.mark.parametrize("T,Hq,Hkv,n", NEIGHBOURS)
def test_neighbouring_items_of_many_parts_are_joined_apart(env, T, Hq, Hkv, n):
    """The last workgroup of an item's parts is the first of the next one's (which calls those are: the division's test)."""
    torch, B = env
    each, D = -(-n // 256), 64
    c = Cache(n, each, Hkv, D, 256)
    ws = B.alloc_workspace(B.attn_kv4_workspace_bytes(1, T, Hq, Hkv, D))
    args = (env, c, queries(n, 1, T, Hq, D, 2.0), np.array([n - T]), shuffled(3, 1, each, each))
    first = check(*args, workspace=ws)
    assert int(ws[:16384].count_nonzero()) == 0
    assert torch.equal(first, check(*args, workspace=ws)) and int(ws[:16384].count_nonzero()) == 0


@pytest.mark.parametrize("window,sinks", [(2 ** 31 - 1, 0), (2 ** 31 - 1, 3), (2 ** 30 + 7, 1)])
@pytest.mark.parametrize("T,G,D", [(6, 1, 64), (20, 2, 128), (70, 1, 64)])
def test_windows_as_large_as_they_come(env, window, sinks, T, G, D):
    """No token is behind them, also where a block begins with rows in front of the sequence."""
    c = Cache(31, 12, 1, D, 32)
    check(env, c, queries(32, 4, T, G, D), np.array([-5, 1 - T, 0, 90]), shuffled(8, 4, 3, 12)[:, [0, 1, 2, 2, 2, 2]], window=window, sinks=sinks)


def test_windows_of_rows_far_past_the_cache(env):
    """A window that still reaches the cache from there."""
    T = 4
    for pos in (2 ** 30 + 5, 2 ** 31 - 2 ** 20, 2 ** 31 - 1 - T):
        c = Cache(33, 4, 2, 64, 64)
        got = check(env, c, queries(34, 1, T, 4, 64), np.array([pos]), np.arange(4).reshape(1, 4), window=pos - 150, sinks=5)
        assert (got != 0).all()


@pytest.mark.parametrize("T,G,n", [(1, 1, 100), (1, 8, 3000), (4, 4, 700), (20, 1, 5000), (70, 1, 400), (3, 1, 20000)])
@pytest.mark.parametrize("what", ["key", "value"])
def test_a_token_that_is_no_number_shows(env, T, G, n, what):
    """NaN for step and low of a token that every row sees: NaN, in the sums of one workgroup and in joined ones; the other head keeps its result."""
    torch, B = env
    P, D, Hkv = 64, 64, 2
    each = -(-n // P)
    c = Cache(37, each, Hkv, D, P)
    q, pos, table = dev(torch, queries(38, 1, T, G * Hkv, D)), torch.tensor([n - T], dtype=torch.int32, device="cuda"), torch.arange(each, dtype=torch.int32, device="cuda").view(1, -1)
    want = B.attn_kv4(q, dev(torch, c.bytes()), pos, Hkv, P, table)
    for at in (0, n // 3, n - T):
        d = Cache(37, each, Hkv, D, P)
        for a in (d.ks, d.kl) if what == "key" else (d.vs, d.vl):
            a[at // P, 0, at % P] = np.nan
        got = B.attn_kv4(q, dev(torch, d.bytes()), pos, Hkv, P, table)
        assert got[:, :, :G].isnan().all() and torch.equal(got[:, :, G:], want[:, :, G:]), at


@pytest.mark.parametrize("T,G,n", [(1, 1, 1), (1, 8, 3000), (4, 4, 700), (20, 1, 5000), (70, 1, 400)])
def test_a_query_that_is_no_number_shows(env, T, G, n):
    """A NaN or an infinity in one feature of one row: NaN there, the other rows and heads keep their results."""
    torch, B = env
    P, D, Hkv = 64, 128, 2
    each = -(-n // P)
    c = Cache(39, each, Hkv, D, P)
    c.kl[:] = 0.5                                             # all keys positive: a negative infinity would weigh every token with zero
    q = queries(40, 1, T, G * Hkv, D)
    cache, pos, table = dev(torch, c.bytes()), torch.tensor([n - T], dtype=torch.int32, device="cuda"), torch.arange(each, dtype=torch.int32, device="cuda").view(1, -1)
    want = B.attn_kv4(dev(torch, q), cache, pos, Hkv, P, table).cpu().numpy()
    j, h = T // 2, G * Hkv - 1
    for bad in (np.nan, np.inf, -np.inf):
        for d in (0, 70, D - 1):
            p = q.copy()
            p[0, j, h, d] = bad
            got = B.attn_kv4(dev(torch, p), cache, pos, Hkv, P, table).cpu().numpy()
            assert np.isnan(got[0, j, h]).all(), (bad, d)
            got[0, j, h] = want[0, j, h]
            compare(got.astype(np.float64), c, q, np.array([n - T]), np.arange(each).reshape(1, each), None, 0, 0)


def test_rows_that_see_nothing_stay_zero_whatever_the_query(env):
    torch, B = env
    c = Cache(41, 2, 1, 64, 16)
    q = np.full((2, 3, 2, 64), np.nan, np.float16)
    got = B.attn_kv4(dev(torch, q), dev(torch, c.bytes()), torch.tensor([-3, -2], dtype=torch.int32, device="cuda"), 1, 16, torch.tensor([[0], [1]], dtype=torch.int32, device="cuda"))
    assert (got[0] == 0).all() and (got[1, :2] == 0).all() and got[1, 2].isnan().all()


@pytest.mark.parametrize("T,G,first", [(1, 1, 89), (4, 2, 2996), (20, 1, 1980), (70, 1, 230), (70, 1, -3)])
def test_scores_past_what_is_told_apart(env, T, G, first):
    """Scores of up to 2^26: the token with the largest weighs everything, where it leads by more than their rounding.  Past 2^27 a row is no
    number, but for rows that see nothing."""
    torch, B = env
    P, D = 64, 64
    each = -(-(first + T) // P)
    c, table, pos = Cache(43, each, 1, D, P), np.arange(each).reshape(1, each), np.array([first])
    q = queries(44, 1, T, G, D)
    k, v, _, step = c.sequence(table[0], first + T)
    s = q[0].astype(np.float64) @ k[:, 0].T                   # [T, G, tokens]
    s[np.broadcast_to(np.arange(first + T) > first + np.arange(T)[:, None, None], s.shape)] = -np.inf
    sees = np.arange(T) + first >= 0
    fits = float(np.float32(2.0 ** 26 / np.abs(s[np.isfinite(s)]).max()))
    got = check(env, c, q, pos, table, scale=fits).cpu().numpy()[0].astype(np.float64)
    with np.errstate(invalid="ignore"):
        lead = np.sort(s, -1)[..., -1] - (np.sort(s, -1)[..., -2] if first + T > 1 else -np.inf)
    rounding = (D + 12) * 2.0 ** -24 * np.abs(q[0].astype(np.float64)).sum(-1) * np.abs(k).max() * 4
    for j, h in np.argwhere((lead > rounding + 64 / fits) & sees[:, None]):
        want = v[s[j, h].argmax(), 0]
        assert (np.abs(got[j, h] - want) <= 2.0 ** -11 * np.abs(want) + 2.0 ** -11 * 8 * step.max()).all(), (j, h)
    for scale in (float(2.0 ** 27 / np.abs(s.max(-1)[sees]).min()), 1e10):
        out = B.attn_kv4(dev(torch, q), dev(torch, c.bytes()), dev(torch, pos.astype(np.int32)), 1, P, dev(torch, table.astype(np.int32)), scale).cpu().numpy()[0]
        assert np.isnan(out[sees]).all() and (out[~sees] == 0).all()


@pytest.mark.parametrize("T,G,D,window", [(3, 1, 64, 0), (9, 1, 128, 4), (20, 1, 64, 0), (40, 1, 64, 0), (70, 1, 128, 0), (100, 2, 64, 0), (70, 1, 128, 9), (20, 1, 128, 6)])
@pytest.mark.parametrize("bad", [(np.nan, np.nan, np.nan, np.nan), (0.25, -2.0, np.inf, 0.0), (0.25, -2.0, 0.25, -np.inf), (0.25, -2.0, np.nan, 0.0)])
def test_what_later_rows_see_does_not_reach_earlier_ones(env, T, G, D, window, bad):
    """A token of the call whose step or low is not finite: rows before it (and rows whose window has passed it) are as if it were not there, the rows
    that see it are not finite."""
    torch, B = env
    first, P, Hkv = 35, 32, 2
    at = first + T // 2
    each = -(-(first + T) // P)
    c, table = Cache(35, each, Hkv, D, P), np.arange(each).reshape(1, each)
    q, pos = queries(36, 1, T, G * Hkv, D), np.array([first])
    clean = c.bytes()
    for a, x in zip((c.ks, c.kl, c.vs, c.vl), bad):
        a[at // P, 1, at % P] = x                             # the second head's alone
    call = lambda raw: B.attn_kv4(dev(torch, q), dev(torch, raw), dev(torch, pos.astype(np.int32)), Hkv, P, dev(torch, table.astype(np.int32)), window=window).cpu().numpy()[0]
    got = call(c.bytes())
    sees = np.array([kv.visible(first + j, each * P, window, 0)[at] for j in range(T)])
    assert sees.any() and not sees.all()
    assert not np.isfinite(got[sees, G:]).any()
    want = Cache(35, each, Hkv, D, P)
    got[sees, G:] = call(clean)[sees, G:]
    compare(got[None].astype(np.float64), want, q, pos, table, None, window, 0)
