"""Rotary append to the 4-bit cache and reading it back, against the oracle: codes, steps and the cache's bytes are decided
exactly, so everything is compared bit for bit."""
import numpy as np
import pytest

from oracle import kv4_oracle as kv

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


class Plain:
    """The cache as arrays of codes, steps and lows."""

    def __init__(self, n_pages, Hkv, D, P):
        self.P = P
        self.k, self.v = (np.zeros((n_pages, Hkv, P, D), np.uint8) for _ in range(2))
        self.ks, self.kl, self.vs, self.vl = (np.zeros((n_pages, Hkv, P), np.float16) for _ in range(4))

    def put(self, page, slot, k, v):
        self.k[page, :, slot], self.ks[page, :, slot], self.kl[page, :, slot] = kv.quantise(k)
        self.v[page, :, slot], self.vs[page, :, slot], self.vl[page, :, slot] = kv.quantise(v)

    def bytes(self):
        return kv.cache_bytes(self.k, self.ks, self.kl, self.v, self.vs, self.vl, self.P)


def place(table, b, at, P, n_pages):
    """(page, slot) of position at, or None."""
    each = table.shape[1]
    if not 0 <= at < each * P:
        return None
    page = int(table[b, at // P])
    return (page, at % P) if 0 <= page < n_pages else None


def run_append(env, qkv, freq, pos, table, n_pages, Hq, Hkv, P, interleaved=False, mscale=1.0, no_table=False, calls=1):
    """Appends on the GPU and in the oracle; returns nothing, compares everything."""
    torch, B = env
    Bn, T, width = qkv.shape
    D = width // (Hq + 2 * Hkv)
    plain = Plain(n_pages, Hkv, D, P)
    cache = B.alloc_kv4_cache(n_pages, Hkv, D, P)
    guard = torch.full((Bn * T * Hq * D + 64,), 123.0, dtype=torch.float16, device="cuda")
    q = guard[32:-32].view(Bn, T, Hq, D)
    args = (dev(torch, qkv), None if freq is None else dev(torch, freq), dev(torch, pos.astype(np.int32)), cache, Hq, Hkv, P,
            None if no_table else dev(torch, table.astype(np.int32)))
    for _ in range(calls):
        B.rope_kv4_append(*args, interleaved=interleaved, mscale=mscale, q=q)
    k_out, v_out = B.kv4_read(cache, args[2], T, Hkv, D, P, args[7])
    torch.cuda.synchronize()
    at = pos[:, None].astype(np.int64) + np.arange(T)
    x = qkv.reshape(Bn * T, Hq + 2 * Hkv, D)
    turned = x[:, :Hq + Hkv] if freq is None else kv.rotate(x[:, :Hq + Hkv], at.ravel(), freq, interleaved, float(np.float32(mscale)))
    assert (q.cpu().numpy().view(np.uint16) == turned[:, :Hq].reshape(Bn, T, Hq, D).view(np.uint16)).all()
    assert (guard[:32] == 123.0).all() and (guard[-32:] == 123.0).all()
    want_k, want_v = np.zeros((2, Bn, T, Hkv, D), np.float16)
    for b in range(Bn):
        for j in range(T):
            there = place(table, b, int(at[b, j]), P, n_pages)
            if there:
                plain.put(*there, turned[b * T + j, Hq:], x[b * T + j, Hq + Hkv:])
                page, slot = there
                half = lambda c, s, l: np.clip(c.astype(np.float32) * s.astype(np.float32)[:, None] + l.astype(np.float32)[:, None], -65504, 65504).astype(np.float16)
                want_k[b, j] = half(plain.k[page, :, slot], plain.ks[page, :, slot], plain.kl[page, :, slot])
                want_v[b, j] = half(plain.v[page, :, slot], plain.vs[page, :, slot], plain.vl[page, :, slot])
    wrong = np.argwhere(cache.cpu().numpy() != plain.bytes())
    assert len(wrong) == 0, (len(wrong), wrong[:4].tolist())
    # (the two roundings of the product and the sum may meet a tie of fp16 that one does not: half a unit of binary32 away)
    for got, want in ((k_out, want_k), (v_out, want_v)):
        g, w = got.cpu().numpy().astype(np.float64), want.astype(np.float64)
        assert np.abs(g - w).max() <= 2.0 ** -10 * np.abs(w).max()
        assert (g != w).mean() < 1e-3


def inputs(seed, Bn, T, Hq, Hkv, D, outliers=True):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((Bn, T, Hq + 2 * Hkv, D)).astype(np.float32)
    if outliers:
        x[..., rng.integers(0, D, 2)] *= 20.0
    return x.astype(np.float16).reshape(Bn, T, -1)


def shuffled(seed, Bn, each, n_pages):
    return np.random.default_rng(seed).permutation(n_pages)[:Bn * each].reshape(Bn, each)


FREQ = lambda rot, theta=10000.0: theta ** (-np.arange(0, rot, 2) / rot)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rot", [0, 16, 48, 64, 128])
def test_rotation_of_a_part_of_the_head(env, D, interleaved, rot):
    if rot > D:
        rot = 32
    x = inputs(rot + D, 2, 3, 6, 3, D)
    run_append(env, x, FREQ(rot) if rot else None, np.array([0, 1000]), shuffled(1, 2, 70, 145), 145, 6, 3, 16, interleaved)


@pytest.mark.parametrize("Bn,T,Hq,Hkv,D,P", [(1, 1, 1, 1, 64, 16), (1, 1, 32, 32, 128, 64), (3, 4, 8, 1, 128, 32), (2, 17, 5, 5, 64, 16),
                                             (1, 130, 4, 2, 128, 64), (9, 2, 7, 1, 64, 256), (1, 33, 40, 8, 128, 16), (128, 4, 2, 1, 64, 16)])
def test_shapes_across_pages(env, Bn, T, Hq, Hkv, D, P):
    rng = np.random.default_rng(T)
    each = (T + 3 * P) // P + 1
    pos = rng.integers(0, 2 * P + 5, Bn)
    run_append(env, inputs(Bn + T, Bn, T, Hq, Hkv, D), FREQ(D), pos, shuffled(2, Bn, each, Bn * each + 3), Bn * each + 3, Hq, Hkv, P)


def test_pages_in_sequence_order(env):
    table = np.arange(12).reshape(3, 4)
    run_append(env, inputs(5, 3, 5, 4, 2, 128), FREQ(128), np.array([0, 13, 50]), table, 12, 4, 2, 16, no_table=True)


def test_far_positions_and_scaled_frequencies(env):
    import torch
    from paper_2410_11305_amd import rope
    for scaling in ("linear", "ntk", "yarn"):
        f, m = rope.frequencies(128, 500000.0, scaling, 8.0, 8192, device="cpu")
        # a table of many pages of which one page exists; positions up to a million
        for at in (131071, 999989):
            table = np.full((1, 62500 + 2), -1)
            table[0, at // 16], table[0, at // 16 + 1] = 1, 0
            run_append(env, inputs(at, 1, 7, 4, 2, 128), f.numpy(), np.array([at]), table, 2, 4, 2, 16, mscale=m)


def test_rows_without_a_place_are_not_stored(env):
    """Idle sequences, rows before 0 and past the last page, entries outside the cache on both sides."""
    table = np.array([[0, 1, 2], [3, -1, 4], [5, 99, 6], [7, 8, 2 ** 31 - 1], [9, 10, 11], [12, 13, 14], [15, 16, 17]])
    pos = np.array([-5, 10, 12, 30, 46, -2, 2 ** 31 - 3])
    run_append(env, inputs(3, 7, 5, 4, 2, 64), FREQ(32), pos, table, 18, 4, 2, 16)


def test_values_that_are_hard_to_quantise(env):
    """Constant rows, zeros, the largest spread there is, steps that are subnormal or round to zero, ties."""
    rows = [np.full(64, -3.25), np.zeros(64), np.r_[65504.0, -65504.0, np.full(62, 2.0 ** -24)], np.arange(64) * 2.0 ** -24,
            np.r_[np.zeros(63), 2.0 ** -24], np.r_[np.zeros(60), np.full(4, 7 * 2.0 ** -24)], np.r_[0.0, 15.0, np.arange(15) + 0.5, np.full(47, 7.0)],
            np.r_[-7.5, 7.5, np.arange(15) - 7.0, np.full(47, 0.5)], np.r_[0.0, 30.0, 2.0 * np.arange(15) + 1.0, np.full(47, 29.0)], np.arange(64) * 31.0,
            -np.arange(64) * 31.0, np.r_[1000.0, np.zeros(63)]]
    x = np.array(rows).astype(np.float16).reshape(1, len(rows), 1, 64)
    qkv = np.concatenate((x, x, x[:, ::-1]), axis=2).reshape(1, len(rows), -1)
    run_append(env, qkv, None, np.array([3]), np.array([[1, 0]]), 2, 1, 1, 16)


def test_many_random_rows(env):
    rng = np.random.default_rng(9)
    x = (rng.standard_normal((1, 600, 3, 128)) * 10.0 ** rng.uniform(-5, 3, (1, 600, 3, 1))).astype(np.float16)
    x[0, ::3] = np.round(x[0, ::3].astype(np.float32) * 4) / 4                 # few distinct values: many ties
    x = np.clip(x.astype(np.float32), -60000, 60000).astype(np.float16)
    run_append(env, x.reshape(1, 600, -1), None, np.array([1]), np.arange(10).reshape(1, 10), 10, 1, 1, 64)


def test_appending_again_overwrites(env):
    """The verify pass at the draft pass's positions."""
    run_append(env, inputs(4, 2, 4, 2, 1, 64), FREQ(64), np.array([14, 3]), shuffled(3, 2, 2, 4), 4, 2, 1, 16, calls=3)


def test_binding_checks_shapes_on_the_device(env):
    torch, B = env
    cache = B.alloc_kv4_cache(4, 2, 64, 16)
    pos, qkv = torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros((2, 1, 8 * 64), dtype=torch.float16, device="cuda")
    good = dict(qkv=qkv, inv_freq=None, pos=pos, cache=cache, Hq=4, Hkv=2, page_size=16)
    B.rope_kv4_append(**good)
    for bad in (dict(qkv=qkv[:1]), dict(qkv=qkv.float()), dict(qkv=qkv.transpose(0, 1)), dict(pos=pos.long()), dict(cache=cache[:, 1:]),
                dict(page_table=torch.zeros((3, 2), dtype=torch.int32, device="cuda")), dict(q=torch.empty((2, 1, 4, 128), dtype=torch.float16, device="cuda")),
                dict(inv_freq=torch.ones(8, device="cuda")), dict(pos=pos.cpu()), dict(qkv=torch.cat((qkv, qkv), -1)[..., ::2])):
        with pytest.raises(ValueError):
            B.rope_kv4_append(**{**good, **bad})
    with pytest.raises(B.QSpecError):
        B.rope_kv4_append(**{**good, "inv_freq": torch.ones(5, dtype=torch.float64, device="cuda")})
    with pytest.raises(ValueError):
        B.kv4_read(cache, pos, 2, 2, 64, 16, k=torch.empty((2, 1, 2, 64), dtype=torch.float16, device="cuda"))
    with pytest.raises(B.QSpecError):
        B.kv4_read(cache, pos, 0, 2, 64, 16)


@pytest.mark.parametrize("rot,interleaved", [(64, False), (64, True), (32, False), (16, True)])
def test_rotated_queries_keep_what_is_no_number(env, rot, interleaved):
    """NaN stays NaN and infinities what the rotation makes of them: infinite, or NaN beside another one or at an angle of zero."""
    torch, B = env
    rng, Hq, T, D = np.random.default_rng(50), 5, 9, 64
    x = rng.standard_normal((T, Hq + 2, D)).astype(np.float16)
    bad = rng.random((T, Hq, D)) < 0.1
    x[:, :Hq][bad] = rng.choice([np.nan, np.inf, -np.inf], bad.sum())
    cache, pos = B.alloc_kv4_cache(1, 1, D, 16), torch.zeros(1, dtype=torch.int32, device="cuda")
    q = B.rope_kv4_append(dev(torch, x.reshape(1, T, -1)), dev(torch, FREQ(rot)), pos, cache, Hq, 1, 16, interleaved=interleaved)[0].cpu().numpy()
    with np.errstate(invalid="ignore"):
        want = kv.rotate(x[:, :Hq], np.arange(T), FREQ(rot), interleaved)
    np.testing.assert_array_equal(q, want)
    assert np.isnan(want).any() and np.isinf(want).any()


def run_without_numbers(env, x, freq, pos, table, n_pages, Hq, Hkv, P, interleaved=False):
    """run_append for heads x fp16 [T, Hq + 2 Hkv, D] of one sequence that hold infinities and NaN: a NaN is a NaN, whatever its bits, but in the cache."""
    torch, B = env
    T, heads, D = x.shape
    plain, cache = Plain(n_pages, Hkv, D, P), B.alloc_kv4_cache(n_pages, Hkv, D, P)
    at, tab = dev(torch, np.array([pos], dtype=np.int32)), dev(torch, table.astype(np.int32))
    q = B.rope_kv4_append(dev(torch, x.reshape(1, T, -1)), None if freq is None else dev(torch, freq), at, cache, Hq, Hkv, P, tab, interleaved=interleaved)
    k, v = B.kv4_read(cache, at, T, Hkv, D, P, tab)
    with np.errstate(over="ignore", invalid="ignore"):
        turned = x[:, :Hq + Hkv] if freq is None else kv.rotate(x[:, :Hq + Hkv], pos + np.arange(T), freq, interleaved)
    np.testing.assert_array_equal(q[0].cpu().numpy(), turned[:, :Hq])
    for j in range(T):
        plain.put(*place(table, 0, pos + j, P, n_pages), turned[j, Hq:], x[j, Hq + Hkv:])
    assert (cache.cpu().numpy() == plain.bytes()).all()
    for got, rows in ((k, turned[:, Hq:]), (v, x[:, Hq + Hkv:])):
        assert (got[0].isnan().cpu().numpy() == ~np.isfinite(rows).all(-1, keepdims=True)).all()
    return turned


@pytest.mark.parametrize("D,rot,interleaved", [(64, 64, False), (128, 64, True), (128, 128, False), (64, 0, False)])
def test_values_that_are_no_numbers(env, D, rot, interleaved):
    """A query keeps NaN and infinities where the rotation leaves them; a key or value row that has one is stored with NaN for step and low and codes
    of zero, and reads back as NaN; the rows beside it are what they were."""
    rng = np.random.default_rng(51)
    Hq, Hkv, T = 3, 2, 24
    x = rng.standard_normal((T, Hq + 2 * Hkv, D)).astype(np.float16)
    for j, bad in enumerate((np.nan, np.inf, -np.inf) * 7):
        for h in range(j % 3, Hq + 2 * Hkv, 3):
            x[j, h, rng.integers(0, D)] = bad
    x[22, :, 5], x[22, :, 7] = np.inf, -np.inf                # both
    x[23] = np.nan
    turned = run_without_numbers(env, x, FREQ(rot) if rot else None, 13, np.array([[1, 2, 0]]), 3, Hq, Hkv, 16, interleaved)
    assert np.isnan(turned).any() and np.isinf(turned).any() and np.isfinite(turned).all(-1).any()


def test_rotation_past_the_largest_number(env):
    """A rotated key that leaves fp16's range is an infinity: its row has no numbers either."""
    x = np.full((2, 3, 64), 1.0, np.float16)
    x[1, :2, 0] = x[1, :2, 32] = 60000.0
    turned = run_without_numbers(env, x, FREQ(64), 40, np.array([[0, 1, 2]]), 3, 1, 1, 16)
    assert np.isinf(turned[1]).any() and np.isfinite(turned[0]).all()


def test_steps_and_lows_that_are_no_numbers_read_back_as_such(env):
    torch, B = env
    plain = Plain(1, 1, 64, 16)
    plain.k[:], plain.v[:] = 3, 15
    plain.ks[:], plain.kl[:], plain.vs[:], plain.vl[:] = 1.0, 2.0, 8737.6, -65504.0
    for slot, (step, low) in enumerate(((np.nan, np.nan), (np.inf, 0.0), (0.0, -np.inf), (1.0, np.nan))):
        plain.ks[0, 0, slot], plain.kl[0, 0, slot], plain.vs[0, 0, slot], plain.vl[0, 0, slot] = step, low, step, low
    k, v = B.kv4_read(dev(torch, plain.bytes()), torch.zeros(1, dtype=torch.int32, device="cuda"), 5, 1, 64, 16)
    np.testing.assert_array_equal(k[0, :, 0, 0].cpu().numpy(), [np.nan, np.inf, -np.inf, np.nan, 5.0])
    np.testing.assert_array_equal(v[0, :, 0, 0].cpu().numpy(), [np.nan, np.inf, -np.inf, np.nan, 65504.0])    # (15 * 8736 - 65504 = 65536, a finite value: held)
