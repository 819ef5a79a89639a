"""A decoder's cycle with the operators in a row, as a program runs them: a padded batch of prompts, draft steps on the W4A4
products, a verify pass on the W4A16 products (eager, then as a replayed graph), acceptance, and the next cycle at the positions that
follow.  Every stage is held to the oracle on what the stage before it really wrote."""
import numpy as np
import pytest

from oracle import kv4_oracle as kv
from oracle import sample_oracle as so
from paper_2410_11305_amd import synth
from tests.test_gpu_attn_kv4 import compare, dev
from tests.test_gpu_kv4 import Plain, place

pytestmark = pytest.mark.gpu

BATCH, GAMMA, HQ, HKV, D, PAGE, EACH, V = 3, 3, 4, 2, 64, 16, 6, 1008
HID = HQ * D


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2410_11305_amd import binding as B
    assert torch.cuda.is_available()
    B.lib()
    return torch, B


class Model:
    """One attention layer and a vocabulary product, with everything a cycle needs and the oracle's view of the cache."""

    def __init__(self, torch, B):
        from paper_2410_11305_amd import rope
        self.torch, self.B = torch, B
        rng = np.random.default_rng(0)
        weights = lambda seed, n: B.pack_weights(dev(torch, synth.generic_case(seed, 1, n, HID)[0]), dev(torch, synth.generic_case(seed, 1, n, HID)[1]))
        self.qkv, self.o, self.head = weights(1, (HQ + 2 * HKV) * D), weights(2, HID), weights(3, V)
        self.embed = dev(torch, rng.standard_normal((V, HID)).astype(np.float16))
        self.freq, self.mscale = rope.frequencies(D, 10000.0, "yarn", 4.0, 64)
        self.n_pages = BATCH * EACH + 2
        self.table = rng.permutation(self.n_pages)[:BATCH * EACH].reshape(BATCH, EACH)
        self.tab = dev(torch, self.table.astype(np.int32))
        self.cache = B.alloc_kv4_cache(self.n_pages, HKV, D, PAGE)
        self.plain = Plain(self.n_pages, HKV, D, PAGE)
        T = 64
        self.ws = B.alloc_workspace(max([B.attn_kv4_workspace_bytes(BATCH, t, HQ, HKV, D) for t in (1, GAMMA + 1, T)]
                                        + [B.workspace_bytes(m, n, HID) for m in (BATCH, BATCH * (GAMMA + 1), BATCH * T) for n in ((HQ + 2 * HKV) * D, HID, V)]))

    def product(self, packed, x, N, draft):
        B = self.B
        if draft:
            qa, sa = B.quant_act(x)
            return B.gemm_w4a4(packed, qa, sa, N, workspace=self.ws)
        return B.gemm_w4a16(packed, x, N, workspace=self.ws)

    def forward(self, tokens, pos, draft):
        """tokens int32 [B, T] at positions pos -> every stage's tensor."""
        B, T = self.B, tokens.shape[1]
        x = self.embed[tokens.long()].view(BATCH * T, HID)
        qkv = self.product(self.qkv, x, (HQ + 2 * HKV) * D, draft).view(BATCH, T, -1)
        q = B.rope_kv4_append(qkv, self.freq, pos, self.cache, HQ, HKV, PAGE, self.tab, mscale=self.mscale)
        a = B.attn_kv4(q, self.cache, pos, HKV, PAGE, self.tab, workspace=self.ws)
        y = x + self.product(self.o, a.view(BATCH * T, HID), HID, draft) * 0.05
        return dict(qkv=qkv, q=q, a=a, logits=(self.product(self.head, y, V, draft) * 0.02).view(BATCH, T, V))

    def check(self, stage, pos):
        """The stage's queries, the cache and the attention against the oracle; pos on the host."""
        qkv, T = stage["qkv"].cpu().numpy(), stage["qkv"].shape[1]
        x = qkv.reshape(BATCH * T, HQ + 2 * HKV, D)
        at = pos[:, None].astype(np.int64) + np.arange(T)
        turned = kv.rotate(x[:, :HQ + HKV], at.ravel(), self.freq.cpu().numpy(), False, float(np.float32(self.mscale)))
        assert (stage["q"].cpu().numpy().reshape(BATCH * T, HQ, D) == turned[:, :HQ]).all()
        for b in range(BATCH):
            for j in range(T):
                there = place(self.table, b, int(at[b, j]), PAGE, self.n_pages)
                if there:
                    self.plain.put(*there, turned[b * T + j, HQ:], x[b * T + j, HQ + HKV:])
        assert (self.cache.cpu().numpy() == self.plain.bytes()).all()
        compare(stage["a"].cpu().numpy().astype(np.float64), Reader(self.plain, self.n_pages), turned[:, :HQ].reshape(BATCH, T, HQ, D), pos, self.table, None, 0, 0)


class Reader:
    def __init__(self, plain, n_pages):
        self.p, self.P, self.Hkv, self.D, self.n_pages = plain, PAGE, HKV, D, n_pages

    def sequence(self, row, tokens):
        p, n = self.p, -(-tokens // PAGE)
        flat = lambda a: a[row[:n]].swapaxes(1, 2).reshape((n * PAGE,) + a.shape[1:2] + a.shape[3:])[:tokens]
        return kv.values(flat(p.k), flat(p.ks), flat(p.kl)), kv.values(flat(p.v), flat(p.vs), flat(p.vl)), np.ones(tokens, bool), flat(p.vs).astype(np.float64)


def test_cycles_of_drafts_and_verification(env):
    torch, B = env
    torch.manual_seed(3)
    m, rng = Model(torch, B), np.random.default_rng(5)
    # prompts of 37, 20 and 5 tokens in rows of 37, the shorter ones at the right: their first rows have no place
    length, T = np.array([37, 20, 5]), 37
    prompt = dev(torch, rng.integers(0, V, (BATCH, T)).astype(np.int32))
    pos = length - T
    stage = m.forward(prompt, dev(torch, pos.astype(np.int32)), draft=False)
    m.check(stage, pos)
    assert (stage["a"][2, :32] == 0).all() and (stage["a"][2, 32:] != 0).any()
    temperature = torch.tensor([0.8, 0.0, 1.2], device="cuda")
    top_k, top_p = torch.tensor([0, 0, 50], dtype=torch.int32, device="cuda"), torch.tensor([0.9, 1.0, 1.0], device="cuda")
    knobs = dict(temperature=temperature, top_k=top_k, top_p=top_p)
    host = {k: v.cpu().numpy() for k, v in knobs.items()}
    last = B.sample(stage["logits"][:, -1:].contiguous(), torch.rand((BATCH, 1), device="cuda"), **knobs)[1]
    pos = length.copy()

    verify_in = torch.zeros((BATCH, GAMMA + 1), dtype=torch.int32, device="cuda")
    verify_pos = torch.zeros(BATCH, dtype=torch.int32, device="cuda")
    verify_u = torch.zeros((BATCH, GAMMA + 1), device="cuda")
    graph, accepted = None, []

    def verify():
        s = m.forward(verify_in, verify_pos, draft=False)
        n, out = B.sample(s["logits"], verify_u, draft=verify_in[:, 1:].contiguous(), **knobs)
        return s, n, out

    for cycle in range(5):
        u = torch.rand((BATCH, GAMMA + 1), device="cuda")
        rows = [last]
        for j in range(GAMMA):
            stage = m.forward(rows[-1], dev(torch, (pos + j).astype(np.int32)), draft=True)
            m.check(stage, pos + j)
            rows.append(B.sample(stage["logits"], u[:, j:j + 1].contiguous(), **knobs)[1])
        verify_in.copy_(torch.cat(rows, 1))
        verify_pos.copy_(dev(torch, pos.astype(np.int32)))
        verify_u.copy_(u)
        if graph is None:
            stage, n, out = verify()
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                captured = verify()
        else:
            graph.replay()
            stage, n, out = captured
        torch.cuda.synchronize()
        m.check(stage, pos)                                  # the verify pass's rows have replaced the draft pass's
        logits, uu = stage["logits"].cpu().numpy(), u.cpu().numpy()
        chosen = np.array([[so.sample(logits[b, j], float(uu[b, j]), float(host["temperature"][b]), int(host["top_k"][b]), float(host["top_p"][b]))
                            for j in range(GAMMA + 1)] for b in range(BATCH)])
        n_ref, out_ref = so.accept(chosen, verify_in[:, 1:].cpu().numpy())
        assert n.tolist() == n_ref.tolist() and out.tolist() == out_ref.tolist()
        accepted += n_ref.tolist()
        last = dev(torch, out_ref[np.arange(BATCH), n_ref].astype(np.int32)[:, None])
        pos = pos + n_ref + 1                                 # rows behind the accepted ones are written again before they are seen
    assert max(accepted) > 0 and min(accepted) < GAMMA, accepted   # both ends of the walk are met
