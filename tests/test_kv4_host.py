"""Host-side checks of the 4-bit cache, attention and sampling entry points that need no GPU: sizes, refusals before
anything is launched, the frequencies, and pins of the oracle."""
import math

import numpy as np
import pytest

from oracle import kv4_oracle as kv
from oracle import sample_oracle as so
from paper_2410_11305_amd import binding as B
from paper_2410_11305_amd import rope

A = 4096          # any 16-byte aligned non-null address: rejected before use


def append(**k):
    a = dict(qkv=A, freq=A, pos=A, table=A, B=2, T=3, Hq=8, Hkv=2, D=128, rot=128, inter=0, mscale=1.0, page=64, each=4, pages=9, q=A, cache=A)
    a.update(k)
    return B.lib().qspec_rope_kv4_append(*a.values(), None)


def read(**k):
    a = dict(cache=A, pos=A, table=A, B=2, T=3, Hkv=2, D=128, page=64, each=4, pages=9, k=A, v=A)
    a.update(k)
    return B.lib().qspec_kv4_read(*a.values(), None)


def attend(**k):
    a = dict(q=A, cache=A, pos=A, table=A, B=2, T=3, Hq=8, Hkv=2, D=128, page=64, each=4, pages=9, scale=0.1, window=0, sinks=0, out=A, ws=A, nws=1 << 30)
    a.update(k)
    return B.lib().qspec_attn_kv4(*a.values(), None)


def choose(**k):
    a = dict(logits=A, u=A, t=A, k=A, p=A, m=A, draft=A, B=2, gamma=3, V=100, n=A, out=A, ws=A, nws=1 << 20)
    a.update(k)
    return B.lib().qspec_sample(*a.values(), None)


def test_sizes():
    assert B.kv4_page_bytes(8, 128, 64) == 8 * 64 * 136
    assert B.kv4_page_bytes(1, 64, 16) == 16 * 72
    for bad in ((0, 128, 64), (8, 96, 64), (8, 128, 8), (8, 128, 48), (8, 128, 0), (1 << 20, 128, 64)):
        assert B.kv4_page_bytes(*bad) == 0
    assert B.attn_kv4_workspace_bytes(2, 1, 8, 2, 128) > 16384
    assert B.attn_kv4_workspace_bytes(2, 1, 8, 3, 128) == 0
    assert B.attn_kv4_workspace_bytes(2, 1, 8, 2, 80) == 0
    assert B.sample_workspace_bytes(3, 4, 1000) == 60
    assert B.sample_workspace_bytes(3, -1, 1000) == 0 and B.sample_workspace_bytes(3, 0, 1 << 22) == 0


@pytest.mark.parametrize("call", [append, read, attend])
def test_cache_shapes_are_refused(call):
    for bad in (dict(B=0), dict(T=0), dict(D=96), dict(page=24), dict(page=8), dict(each=0), dict(pages=0), dict(Hkv=0),
                dict(table=None, pages=7), dict(page=1 << 15, each=1 << 16), dict(T=(1 << 20) + 1, B=1, D=64)):
        assert call(**bad) == B.ERR_SHAPE, bad
    assert call(cache=A + 8) == B.ERR_ALIGN and call(pos=A + 2) == B.ERR_ALIGN and call(table=A + 2) == B.ERR_ALIGN
    assert call(cache=None) == B.ERR_NULL and call(pos=None) == B.ERR_NULL


def test_append_refusals():
    for bad in (dict(rot=24), dict(rot=144), dict(rot=-16), dict(inter=2), dict(mscale=0.0), dict(mscale=-1.0),
                dict(mscale=math.inf), dict(mscale=math.nan), dict(Hq=0), dict(B=1 << 20, T=4, table=A)):
        assert append(**bad) == B.ERR_SHAPE, bad
    assert append(qkv=None) == append(q=None) == append(freq=None) == B.ERR_NULL
    assert append(qkv=A + 8) == append(q=A + 8) == append(freq=A + 8) == B.ERR_ALIGN


def test_read_refusals():
    assert read(k=None) == read(v=None) == B.ERR_NULL
    assert read(k=A + 4) == read(v=A + 4) == B.ERR_ALIGN
    assert read(B=1 << 14, T=1 << 14) == B.ERR_SHAPE


def test_attention_refusals():
    for bad in (dict(Hq=9), dict(Hq=0), dict(Hq=1), dict(scale=0.0), dict(scale=-1.0), dict(scale=math.nan), dict(scale=1e11),
                dict(window=-1), dict(sinks=-1), dict(sinks=4), dict(B=1 << 14, T=1 << 14)):
        assert attend(**bad) == B.ERR_SHAPE, bad
    assert attend(q=None) == attend(out=None) == attend(ws=None) == B.ERR_NULL
    assert attend(q=A + 2) == attend(out=A + 8) == attend(ws=A + 4) == B.ERR_ALIGN
    assert attend(nws=B.attn_kv4_workspace_bytes(2, 3, 8, 2, 128) - 1) == B.ERR_WORKSPACE


def test_attention_refuses_more_work_than_it_counts():
    """B * blocks * Hkv * (tokens / 32 + 64) from 2^31 on."""
    size = dict(B=1024, T=4, Hq=64, Hkv=64, D=64, page=64, nws=1)                # (the workspace is looked at first: what is not refused for its size is for that)
    assert attend(**{**size, "nws": 1 << 30}, each=1 << 14, table=A) == B.ERR_SHAPE
    assert attend(**size, each=1 << 9, table=A) == B.ERR_WORKSPACE
    assert attend(B=3, T=1 << 20, Hq=1, Hkv=1, D=64, page=1 << 12, each=1 << 18, table=A) == B.ERR_SHAPE


def test_sample_refusals():
    for bad in (dict(B=0), dict(gamma=-1), dict(gamma=0), dict(V=0), dict(V=(1 << 21) + 1), dict(B=20000)):
        assert choose(**bad) == B.ERR_SHAPE, bad
    assert choose(logits=None) == choose(u=None) == choose(out=None) == choose(n=None) == choose(ws=None) == B.ERR_NULL
    assert choose(logits=A + 2) == choose(u=A + 2) == choose(t=A + 1) == choose(k=A + 2) == choose(draft=A + 2) == choose(ws=A + 8) == B.ERR_ALIGN
    assert choose(nws=31) == B.ERR_WORKSPACE


def test_binding_refuses_tensors_that_do_not_fit():
    import torch
    cache, pos = torch.zeros((4, B.kv4_page_bytes(2, 64, 16)), dtype=torch.uint8), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="GPU"):
        B.attn_kv4(torch.zeros((2, 1, 4, 64), dtype=torch.float16), cache, pos, 2, 16)
    with pytest.raises(B.QSpecError):
        B.attn_kv4(torch.zeros((2, 1, 4, 96), dtype=torch.float16), cache, pos, 2, 16)
    with pytest.raises(B.QSpecError):
        B.rope_kv4_append(torch.zeros((2, 1, 100), dtype=torch.float16), None, pos, cache, 4, 2, 16)
    with pytest.raises(B.QSpecError):
        B.alloc_kv4_cache(4, 2, 96, 16)


# ------------------------------------------------------------------ frequencies
def test_plain_linear_and_ntk_frequencies():
    f, m = rope.frequencies(8, 10000.0, device="cpu")
    assert m == 1.0 and np.allclose(f.numpy(), [1.0, 0.1, 0.01, 0.001], rtol=1e-15)
    g, m = rope.frequencies(8, 10000.0, "linear", 4.0, device="cpu")
    assert m == 1.0 and np.allclose(g.numpy() * 4.0, f.numpy(), rtol=1e-15)
    n, m = rope.frequencies(8, 10000.0, "ntk", 4.0, device="cpu")
    assert m == 1.0 and n[0] == 1.0 and abs(float(n[-1] * 4.0 / f[-1]) - 1.0) < 1e-14       # the slowest pair exactly factor times slower


def test_yarn_frequencies():
    rot, theta, factor, original = 128, 10000.0, 16.0, 4096
    f, _ = rope.frequencies(rot, theta, device="cpu")
    y, m = rope.frequencies(rot, theta, "yarn", factor, original, device="cpu")
    assert abs(m - (0.1 * math.log(16.0) + 1.0)) < 1e-15
    turns, ratio = original * f / (2 * math.pi), y / f
    # the blend runs over whole indices around the two bounds
    assert torch_all(ratio[turns > 32 * theta ** (2 / rot)] == 1.0)
    assert torch_all((ratio[turns < 1 / theta ** (2 / rot)] * factor - 1.0).abs() < 1e-14)
    assert torch_all(ratio[1:] <= ratio[:-1])


@pytest.mark.parametrize("rot,theta,factor,original", [(128, 10000.0, 8.0, 131072), (16, 10000.0, 4.0, 32768), (64, 10000.0, 32.0, 4096), (128, 500000.0, 8.0, 8192),
                                                      (64, 500.0, 2.0, 2 ** 20)])
def test_yarn_blend_where_every_pair_makes_a_turn(rot, theta, factor, original):
    """The blend is a straight line over the index, also where its end lies past the last pair: what lies before is not squeezed."""
    f, _ = rope.frequencies(rot, theta, device="cpu")
    y, _ = rope.frequencies(rot, theta, "yarn", factor, original, device="cpu")
    index = lambda turns: rot * math.log(original / (turns * 2 * math.pi)) / (2 * math.log(theta))
    low, high = max(math.floor(index(32.0)), 0), min(math.ceil(index(1.0)), rot - 1)
    want = [min(max((i - low) / (high - low), 0.0), 1.0) for i in range(rot // 2)]
    share = (1.0 - (y / f).numpy()) / (1.0 - 1.0 / factor)
    assert np.abs(share - want).max() < 1e-12
    turns = (original * f / (2 * math.pi)).numpy()
    assert (share[turns > theta ** (2 / rot)] < 1.0).all()    # only pairs of about one turn and fewer are divided by the whole factor


def torch_all(t):
    return t.numel() > 0 and bool(t.all())


@pytest.mark.parametrize("bad", [dict(rot=7), dict(rot=0), dict(rot=8, theta=1.0), dict(rot=8, scaling="other"), dict(rot=8, scaling="linear", factor=0.5),
                                 dict(rot=8, scaling="ntk", factor=math.inf), dict(rot=8, scaling="yarn", original=0), dict(rot=8, scaling="yarn", fast=1.0)])
def test_bad_frequencies_are_refused(bad):
    with pytest.raises(ValueError):
        rope.frequencies(device="cpu", **bad)


# ------------------------------------------------------------------ pins of the oracle
def test_oracle_quantiser_decides_in_rational_arithmetic():
    rng = np.random.default_rng(1)
    rows = [rng.standard_normal(64) * 10.0 ** rng.integers(-6, 4) for _ in range(200)]
    rows += [np.array([0.0, 15.0] + [k + 0.5 for k in range(15)] + [7.0] * 47), np.full(64, -3.25), np.zeros(64),
             np.array([65504.0, -65504.0] + [2.0 ** -24] * 62), np.arange(64) * 2.0 ** -24, np.arange(64) * 31.0]
    for r in rows:
        x = r.astype(np.float16)
        codes, step, low = kv.quantise(x)
        assert codes.tolist() == kv.quantise_exactly(x)
        if step > 2.0 ** -14:
            assert np.abs(kv.values(codes, step, low) - x.astype(np.float64)).max() <= float(step) * (0.5 + 15 * 2.0 ** -11)


def test_oracle_rows_that_hold_no_number():
    x = np.zeros((4, 64), np.float16)
    x[0, 3], x[1, 63], x[2, 0], x[3, 7] = np.nan, np.inf, -np.inf, 15.0
    codes, step, low = kv.quantise(x)
    assert step.view(np.uint16)[:3].tolist() == low.view(np.uint16)[:3].tolist() == [0x7E00] * 3 and not codes[:3].any()
    assert step[3] == 1.0 and low[3] == 0.0 and codes[3].tolist() == [15 if i == 7 else 0 for i in range(64)]
    assert np.isnan(kv.values(codes, step, low)[:3]).all()


def test_oracle_rotation_keeps_lengths_and_differences_of_positions():
    rng = np.random.default_rng(2)
    f = 10000.0 ** (-np.arange(0, 32, 2) / 32.0)
    x = rng.standard_normal((1, 2, 64)).astype(np.float16)
    for inter in (False, True):
        at = lambda p: kv.rotate(x, np.array([p]), f, inter).astype(np.float64)[0]
        assert (at(0) == x[0]).all() and (at(977)[:, 32:] == x[0, :, 32:]).all()
        d = [float(at(p)[0] @ at(p + 5)[1]) for p in (0, 100, 5000)]
        assert max(d) - min(d) < 64 * 2 * 9 * 2.0 ** -11                  # products of two values rounded to 11 bits


def test_oracle_cache_bytes_of_one_row():
    k = np.zeros((1, 1, 16, 64), np.uint8)
    v = np.zeros_like(k)
    k[0, 0, 3, 8:16] = range(1, 9)
    v[0, 0, 5, 16:24] = range(8, 16)
    z = np.zeros((1, 1, 16), np.float16)
    ks = z.copy(); ks[0, 0, 3] = 1.0
    raw = kv.cache_bytes(k, ks, z, v, z, z, 16)[0]
    words = raw.view(np.uint32)
    assert words[3 * 8 + 1] == 0x86427531 and words[128 + 2 * 16 + 5] == 0xFDB9ECA8
    assert raw.view(np.uint16)[(1024 + 3 * 8) // 2] == 0x3C00 and np.count_nonzero(words) == 3


def test_oracle_sampling_limits_by_hand():
    row = np.log(np.array([0.1, 0.4, 0.2, 0.3])).astype(np.float64)
    pick = lambda u, **k: so.sample(row, u, **k)
    assert [pick(u) for u in (0.0, 0.39, 0.41, 0.69, 0.71, 0.89, 0.91)] == [1, 1, 3, 3, 2, 2, 0]
    assert [pick(u, top_k=2) for u in (0.0, 0.57, 0.58, 0.99)] == [1, 1, 3, 3]
    assert [pick(u, top_p=0.65) for u in (0.56, 0.58, 0.99)] == [1, 3, 3]
    assert [pick(u, min_p=0.6) for u in (0.56, 0.58, 0.99)] == [1, 3, 3]
    assert pick(0.99, temperature=0.0) == 1 and pick(0.99, top_p=0.0) == 1 and pick(0.99, top_k=1) == 1
    assert so.sample([1.0, 1.0, 1.0, 1.0], 0.5) == 2 and so.sample([1.0, 1.0, 1.0, 1.0], 0.5, top_p=0.5) == 1
    assert so.sample([-math.inf, math.nan], 0.5) == -1 and so.sample([0.0, math.inf, 1.0, math.inf], 0.5) == 3
    n, out = so.accept(np.array([[4, 5, 6], [4, 5, 6], [4, 5, 6]]), np.array([[4, 5], [4, 6], [5, 5]]))
    assert n.tolist() == [2, 1, 0] and out.tolist() == [[4, 5, 6], [4, 5, -1], [4, -1, -1]]
