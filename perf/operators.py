"""What a decoder step needs between the quantised products, as cases that can be timed: rotary positions
with the append to a key/value cache held in 4 bits, attention over that cache, and the choice of the next token.

Every pass exists twice.  With `own` false, `run` computes it in its plain form, from elementary tensor operations;
with `own` true it makes the calls a program makes of `paper_2410_11305_amd.binding`.  Both read the same inputs, the
cache in its documented byte layout among them:

  a page holds page_size tokens of every key/value head; per head, D features each,
    page_size rows of D/2 bytes       key codes: 32-bit words of 8 codes, features 8w .. 8w+7 in word w
    page_size / 16 tiles of 8 D bytes value codes: word (w, t) of a tile, features 8w .. 8w+7 of its token t, at w * 16 + t
    page_size rows of 4 fp16          key step, key minimum, value step, value minimum
  code e of a word sits at bit 4 * (4 (e % 2) + e // 2); a value is code * step + minimum

Token t of sequence b lies in row t % page_size of page table[b][t // page_size].
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

# (query heads, key/value heads, features per head) of Llama-shaped blocks
HEADS = {"7b": (32, 32, 128), "70b": (64, 8, 128)}


def _append(name, heads, B, T, first, rot, page, interleaved=False, factor=1.0, theta=10000.0, spread=0):
    Hq, Hkv, D = heads
    return dict(name=name, op="append", Hq=Hq, Hkv=Hkv, D=D, B=B, T=T, first=first, spread=spread, rot=rot, page=page,
                interleaved=interleaved, factor=factor, theta=theta)


def _attention(name, heads, B, T, longest, shortest, page, paged, window=0, sinks=0):
    Hq, Hkv, D = heads
    return dict(name=name, op="attention", Hq=Hq, Hkv=Hkv, D=D, B=B, T=T, longest=longest, shortest=shortest, page=page,
                paged=paged, window=window, sinks=sinks)


def _sample(name, B, gamma, V, accept, masked=0.0):
    return dict(name=name, op="sample", B=B, gamma=gamma, V=V, accept=accept, masked=masked)


def listed():
    return [
        # one user's draft token: latency
        _append("append_7b_b1", HEADS["7b"], 1, 1, 700, 128, 64),
        # the verify pass of the largest decoding configuration: 128 sequences, 3 drafts + 1 each
        _append("append_70b_verify_b128", HEADS["70b"], 128, 4, 30, 128, 64, spread=1900),
        # a chunk of a long document: odd length, far positions, frequencies stretched 8 times, half of each head
        # rotated, neighbouring features paired
        _append("append_prompt_2050", HEADS["7b"], 1, 2050, 120007, 64, 64, interleaved=True, factor=8.0),
        # small batch, short context: four sequences verify three drafts each
        _attention("attend_short_b4_verify", HEADS["7b"], 4, 4, 193, 41, 16, True),
        # the draft pass of 8 sequences, every head with its own keys, a cache laid out in sequence order
        _attention("attend_7b_draft_b8", HEADS["7b"], 8, 1, 2048, 1500, 256, False),
        # the verify pass of 128 ragged sequences with shared key/value heads, pages anywhere
        _attention("attend_70b_verify_b128", HEADS["70b"], 128, 4, 2048, 200, 64, True),
        # one user, a very long context, one token
        _attention("attend_70b_long_b1", HEADS["70b"], 1, 1, 131071, 131071, 256, True),
        # streaming generation: the last 4096 tokens and the first four, smaller heads
        _attention("attend_window_b32", (64, 8, 64), 32, 1, 32768, 2000, 64, True, window=4096, sinks=4),
        # a prompt of odd length attends to itself
        _attention("attend_7b_prompt_2050", HEADS["7b"], 1, 2050, 2050, 2050, 64, True),
        # one user's next token
        _sample("sample_b1", 1, 0, 32000, False),
        # the verify pass's choice for 128 sequences of 3 drafts + 1, and how many drafts it confirms
        _sample("sample_accept_b128", 128, 3, 32000, True),
        # a large vocabulary of which a grammar leaves a part
        _sample("sample_b32_v128256", 32, 0, 128256, False, masked=0.3),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("append", "attention", "attention", "attention", "sample"))
    if op == "sample":
        V = _log_int(rng, 1000, 160000)
        gamma = rng.choice((0, 1, 3, 5))
        B = _log_int(rng, 1, max(1, 512 * 32000 // (V * (gamma + 1))))
        case = _sample("", B, gamma, V, gamma > 0, masked=rng.choice((0.0, 0.0, 0.5)))
    else:
        Hkv = rng.choice((1, 2, 4, 5, 8, 32, 40))
        group = rng.choice((1, 2, 4, 7, 8)) if Hkv <= 8 else 1
        heads = (Hkv * group, Hkv, rng.choice((64, 128, 128)))
        page = rng.choice((16, 32, 64, 128, 256))
        kind = rng.choice(("draft", "verify", "prompt"))
        T = 1 if kind == "draft" else rng.randint(2, 9) if kind == "verify" else _log_int(rng, 33, 2050)
        if op == "append":
            B = _log_int(rng, 1, max(1, 2050 // T if kind == "prompt" else 128))
            rot = rng.choice((16, 32, 64, heads[2]))
            first = _log_int(rng, 1, 60000)
            case = _append("", heads, B, T, first, rot, page, interleaved=rng.random() < 0.5, factor=rng.choice((1.0, 1.0, 4.0, 8.0)),
                           theta=rng.choice((10000.0, 500000.0)), spread=_log_int(rng, 1, 2000))
        else:
            longest = T + _log_int(rng, 1, 131072 if kind != "prompt" else 4096)
            tokens = 140e6 / (Hkv * (heads[2] + 8))                            # of all sequences, by the longest listed pass
            longest = max(T, min(longest, int(tokens)))
            pairs = 32 * 2050 * 2050 / 2                                       # query, key and head, by the listed prompt
            B = _log_int(rng, 1, max(1, min(160, int(tokens / longest), int(pairs / (heads[0] * T * longest)))))
            if T * longest * heads[0] > pairs:
                longest = max(T, int(pairs / (heads[0] * T)))
                T = min(T, longest)
            windowed = rng.random() < 0.35
            case = _attention("", heads, B, T, longest, max(1, int(longest * rng.random())), page, rng.random() < 0.7,
                              window=_log_int(rng, 16, 8192) if windowed else 0, sinks=rng.choice((0, 1, 4, 16)) if windowed else 0)
    del case["name"]
    return case


# ------------------------------------------------------------------ inputs
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _first_positions(case):
    """Position of each sequence's first new token."""
    B = case["B"]
    at = [(i * 0.6180339887498949) % 1.0 for i in range(B)]
    if case["op"] == "append":
        return [case["first"] + int(case["spread"] * a) for a in at]
    low, high = case["shortest"], case["longest"]
    lengths = [max(1, high - int((high - low) * a)) for a in at]               # the first sequence is the longest
    return [n - case["T"] for n in lengths]


def _pages(case):
    """(pages of a sequence, pages of the cache)"""
    each = -(-max(p + case["T"] for p in _first_positions(case)) // case["page"])
    return each, each * case["B"]


def _page_bytes(case):
    return case["Hkv"] * case["page"] * (case["D"] + 8)


def _frequencies(case):
    """theta^(-2i/rot) / factor in radians per position."""
    rot = case["rot"]
    return [case["theta"] ** (-2.0 * i / rot) / case["factor"] for i in range(rot // 2)]


def _random_cache(case, gen, n_pages):
    """A cache as a long run of a model leaves it: codes of every value, steps about a sixth of a deviation."""
    Hkv, P, D = case["Hkv"], case["page"], case["D"]
    cache = torch.randint(0, 256, (n_pages, Hkv, P * (D + 8)), dtype=torch.uint8, device="cuda", generator=gen)
    step = 0.15 + 0.15 * torch.rand((n_pages, Hkv, P, 2), device="cuda", generator=gen)
    minimum = -step * (6.5 + 2.0 * torch.rand((n_pages, Hkv, P, 2), device="cuda", generator=gen))
    cache[:, :, P * D:] = torch.stack((step[..., 0], minimum[..., 0], step[..., 1], minimum[..., 1]), -1).half().view(torch.uint8).flatten(2)
    return cache.view(n_pages, _page_bytes(case))


def prepare(case, seed):
    gen = _generator(seed)
    if case["op"] == "sample":
        return _prepare_sample(case, gen)
    B, T, Hq, Hkv, D = (case[k] for k in ("B", "T", "Hq", "Hkv", "D"))
    each, n_pages = _pages(case)
    state = dict(case, pos=torch.tensor(_first_positions(case), dtype=torch.int32, device="cuda"))
    paged = case["op"] == "append" or case["paged"]
    state["table"] = torch.randperm(n_pages, device="cuda", generator=gen).int().view(B, each) if paged else None
    if case["op"] == "append":
        state["qkv"] = torch.randn((B, T, (Hq + 2 * Hkv) * D), device="cuda", generator=gen).half()
        state["frequencies"] = torch.tensor(_frequencies(case), dtype=torch.float64, device="cuda")
        state["cache"] = torch.zeros((n_pages, _page_bytes(case)), dtype=torch.uint8, device="cuda")
        if own:
            state["q"] = torch.empty((B, T, Hq, D), dtype=torch.float16, device="cuda")
            state["k"], state["v"] = (torch.empty((B, T, Hkv, D), dtype=torch.float16, device="cuda") for _ in range(2))
    else:
        state["q"] = torch.randn((B, T, Hq, D), device="cuda", generator=gen).half()
        state["cache"] = _random_cache(case, gen, n_pages)
        if own:
            from paper_2410_11305_amd import binding
            state["out"] = torch.empty_like(state["q"])
            state["workspace"] = binding.alloc_workspace(binding.attn_kv4_workspace_bytes(B, T, Hq, Hkv, D))
    return state


def _prepare_sample(case, gen):
    B, gamma, V = case["B"], case["gamma"], case["V"]
    rows = gamma + 1
    logits = (torch.randn((B, rows, V), device="cuda", generator=gen) * 2.5).half()
    if case["masked"]:
        logits.masked_fill_(torch.rand((B, rows, V), device="cuda", generator=gen) < case["masked"], float("-inf"))
    uniform = torch.rand((B, rows), device="cuda", generator=gen)
    # requests of every kind side by side
    pick = torch.rand((4, B), device="cuda", generator=gen)
    temperature = torch.where(pick[0] < 0.15, torch.zeros_like(pick[0]), 0.3 + 1.2 * pick[0])
    top_k = torch.where(pick[1] < 0.4, torch.zeros_like(pick[1]), 1 + 200 * pick[1]).int()
    top_p = torch.where(pick[2] < 0.3, torch.ones_like(pick[2]), 0.3 + 0.7 * pick[2])
    min_p = torch.where(pick[3] < 0.6, torch.zeros_like(pick[3]), 0.1 * pick[3])
    state = dict(case, logits=logits, uniform=uniform, temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p, draft=None)
    if case["accept"]:
        top = logits.argmax(dim=2).int()
        miss = torch.rand((B, gamma), device="cuda", generator=gen) >= 0.8
        state["draft"] = torch.where(miss, (top[:, :gamma] + 1) % V, top[:, :gamma]).int().contiguous()
    if own:
        from paper_2410_11305_amd import binding
        state["tokens"] = torch.empty((B, rows), dtype=torch.int32, device="cuda")
        state["n_accept"] = torch.empty((B,), dtype=torch.int32, device="cuda") if case["accept"] else None
        state["workspace"] = torch.empty(max(16, binding.sample_workspace_bytes(B, gamma, V)), dtype=torch.uint8, device="cuda")
    return state


# ------------------------------------------------------------------ one pass
def run(state):
    op = state["op"]
    if own:
        from paper_2410_11305_amd import binding
        if op == "append":
            q = binding.rope_kv4_append(state["qkv"], state["frequencies"], state["pos"], state["cache"], state["Hq"], state["Hkv"],
                                        state["page"], state["table"], interleaved=state["interleaved"], q=state["q"])
            k, v = binding.kv4_read(state["cache"], state["pos"], state["T"], state["Hkv"], state["D"], state["page"], state["table"],
                                    k=state["k"], v=state["v"])
            return q, k, v
        if op == "attention":
            return binding.attn_kv4(state["q"], state["cache"], state["pos"], state["Hkv"], state["page"], state["table"],
                                    window=state["window"], sinks=state["sinks"], out=state["out"], workspace=state["workspace"])
        n_accept, tokens = binding.sample(state["logits"], state["uniform"], state["temperature"], state["top_k"], state["top_p"],
                                          state["min_p"], state["draft"], n_accept=state["n_accept"], out_tokens=state["tokens"],
                                          workspace=state["workspace"])
        return tokens if state["draft"] is None else (n_accept, tokens)
    if op == "append":
        return _plain_append(state)
    return _plain_attention(state) if op == "attention" else _plain_sample(state)


# ---- plain forms
_NIBBLE = [4 * (4 * (e % 2) + e // 2) for e in range(8)]       # bit of code e in its word


def _rounded_half(x):
    """float64 to fp16 in one rounding (the conversion of the library goes through float32)."""
    _, e = torch.frexp(x)
    ulp = torch.ldexp(torch.ones_like(x), torch.clamp(e - 11, min=-24))
    return (torch.round(x / ulp) * ulp).half()


def _token_pages(state, at):
    """Page of each position at [B, ...]."""
    page = at // state["page"]
    each = state["cache"].shape[0] // state["B"] if state["table"] is None else state["table"].shape[1]
    if state["table"] is None:
        return page + torch.arange(state["B"], device="cuda").view(-1, 1) * each
    return torch.gather(state["table"].long(), 1, page)


def _rotate(x, angles, rot, interleaved):
    """x [B, T, H, D] float64, angles [B, T, rot/2]; the first rot features turn in pairs."""
    c, s = torch.cos(angles).unsqueeze(2), torch.sin(angles).unsqueeze(2)
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:rot])
    first, second = a * c - b * s, b * c + a * s
    turned = torch.stack((first, second), -1).flatten(-2) if interleaved else torch.cat((first, second), -1)
    return torch.cat((turned, x[..., rot:]), -1)


def _plain_append(state):
    B, T, Hq, Hkv, D, P = (state[k] for k in ("B", "T", "Hq", "Hkv", "D", "page"))
    x = state["qkv"].view(B, T, Hq + 2 * Hkv, D).double()
    at = state["pos"].long().view(B, 1) + torch.arange(T, device="cuda")
    angles = at.double().unsqueeze(-1) * state["frequencies"]
    turned = _rounded_half(_rotate(x[:, :, :Hq + Hkv], angles, state["rot"], state["interleaved"]))
    q, k, v = turned[:, :, :Hq], turned[:, :, Hq:], state["qkv"].view(B, T, Hq + 2 * Hkv, D)[:, :, Hq + Hkv:]
    words = state["cache"].view(torch.int32).view(-1)
    start = _token_pages(state, at) * (_page_bytes(state) // 4)                                      # [B, T]
    start = start.unsqueeze(-1) + torch.arange(Hkv, device="cuda") * (P * (D + 8) // 4)              # [B, T, Hkv], in words
    row = (at % P).unsqueeze(-1)
    w = torch.arange(D // 8, device="cuda")
    shifts = torch.tensor(_NIBBLE, device="cuda")
    values, params = [], []
    for which, t in enumerate((k, v)):
        t = t.double()
        low, high = t.amin(-1), t.amax(-1)
        step = _rounded_half((high - low) / 15.0)
        wide = step.double()
        codes = torch.where(wide > 0, torch.round((t - low.unsqueeze(-1)) / torch.where(wide > 0, wide, torch.ones_like(wide)).unsqueeze(-1)).permute(3, 0, 1, 2),
                            torch.zeros_like(wide)).permute(1, 2, 3, 0).clamp(0, 15).long()
        packed = (codes.view(B, T, Hkv, D // 8, 8) << shifts).sum(-1)
        packed = torch.where(packed >= 2 ** 31, packed - 2 ** 32, packed).int()
        if which == 0:
            place = start.unsqueeze(-1) + (row * (D // 8)).unsqueeze(-1) + w
        else:
            place = start.unsqueeze(-1) + (P * D // 8 + (row // 16) * (2 * D) + row % 16).unsqueeze(-1) + w * 16
        words[place.flatten()] = packed.flatten()
        params += [step, low.half()]
        values.append((codes.double() * wide.unsqueeze(-1) + low.unsqueeze(-1)).float().half())
    pair = torch.stack(params, -1).contiguous().view(torch.int32)                                    # [B, T, Hkv, 2]
    words[(start.unsqueeze(-1) + (P * D // 4 + row * 2).unsqueeze(-1) + torch.arange(2, device="cuda")).flatten()] = pair.flatten()
    return q.contiguous(), values[0], values[1]


def _plain_cache(state, tokens):
    """Keys and values [B, Hkv, tokens, D] in float32."""
    B, Hkv, D, P = (state[k] for k in ("B", "Hkv", "D", "page"))
    pages = -(-tokens // P)
    index = _token_pages(state, (torch.arange(pages, device="cuda") * P).repeat(B, 1))
    cache = state["cache"].view(-1, Hkv, P * (D + 8))[index]                                         # [B, pages, Hkv, bytes]
    k = cache[..., :P * D // 2].contiguous().view(torch.int32).view(B, pages, Hkv, P, D // 8)
    v = cache[..., P * D // 2:P * D].contiguous().view(torch.int32).view(B, pages, Hkv, P // 16, D // 8, 16).transpose(-1, -2)
    params = cache[..., P * D:].contiguous().view(torch.float16).view(B, pages, Hkv, P, 4).float()
    shifts = torch.tensor(_NIBBLE, dtype=torch.int32, device="cuda")
    out = []
    for words, step in ((k, 0), (v, 2)):
        codes = ((words.reshape(B, pages, Hkv, P, D // 8, 1) >> shifts) & 15).float().flatten(-2)
        x = codes * params[..., step:step + 1] + params[..., step + 1:step + 2]
        out.append(x.permute(0, 2, 1, 3, 4).reshape(B, Hkv, pages * P, D)[:, :, :tokens])
    return out


def _visible(case, at, t):
    """at: positions of the queries, t: positions of the keys."""
    seen = t <= at
    if case["window"]:
        seen = seen & ((t > at - case["window"]) | (t < case["sinks"]))
    return seen


def _plain_attention(state):
    B, T, Hq, Hkv, D = (state[k] for k in ("B", "T", "Hq", "Hkv", "D"))
    tokens = max(p + T for p in _first_positions(state))
    k, v = _plain_cache(state, tokens)
    group = Hq // Hkv
    q = state["q"].float().view(B, T, Hkv, group, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, T * group, D)
    scores = torch.matmul(q, k.transpose(-1, -2)) * (1.0 / math.sqrt(D))
    at = state["pos"].long().view(B, 1) + torch.arange(T, device="cuda")
    seen = _visible(state, at.unsqueeze(-1), torch.arange(tokens, device="cuda"))                    # [B, T, tokens]
    seen = seen.unsqueeze(2).expand(B, T, group, tokens).reshape(B, 1, T * group, tokens)
    scores = scores.masked_fill(~seen, float("-inf"))
    top = scores.amax(-1, keepdim=True)
    weights = torch.exp(scores - torch.where(torch.isinf(top), torch.zeros_like(top), top))
    total = weights.sum(-1, keepdim=True)
    out = torch.matmul(weights, v) / torch.where(total > 0, total, torch.ones_like(total))
    return out.view(B, Hkv, T, group, D).permute(0, 2, 1, 3, 4).reshape(B, T, Hq, D).half()


def _plain_sample(state):
    """Tokens by falling logit, the lowest first among equals; top_k, min_p, then top_p cut that order, and the token
    is the first whose running mass passes uniform * mass.  Sums in 64 bits: a token next to a border is decided by
    the last of them."""
    x = state["logits"].float()
    B, rows, V = x.shape
    x, order = torch.sort(x, dim=-1, descending=True, stable=True)
    per = lambda name: state[name].view(B, 1, 1)
    greedy = per("temperature") <= 0
    top = x[..., :1]
    scaled = (x - top).double() / torch.where(greedy, torch.ones_like(per("temperature")), per("temperature")).double()
    mass = torch.where(x == top, torch.ones_like(scaled), torch.exp(scaled))
    rank = torch.arange(V, device="cuda")
    k = torch.where(greedy, torch.ones_like(per("top_k")), torch.where(per("top_k") > 0, per("top_k"), torch.full_like(per("top_k"), V)))
    keep = (rank < k) & (mass >= per("min_p").double())
    mass = torch.where(keep, mass, torch.zeros_like(mass))
    running = torch.cumsum(mass, -1)
    limit = per("top_p").double() * running[..., -1:]
    keep = keep & ((running - mass < limit) | (per("top_p") >= 1.0) | (rank == 0))
    kept = torch.where(keep, mass, torch.zeros_like(mass)).sum(-1, keepdim=True)
    choice = (keep & (running <= state["uniform"].double().unsqueeze(-1) * kept)).sum(-1, keepdim=True)
    choice = torch.minimum(choice, keep.sum(-1, keepdim=True) - 1)
    tokens = torch.gather(order, -1, choice).squeeze(-1).int()
    if state["draft"] is None:
        return tokens
    gamma = rows - 1
    hit = torch.cumprod((tokens[:, :gamma] == state["draft"]).int(), -1)
    n_accept = hit.sum(-1)
    tokens = torch.where(torch.arange(rows, device="cuda") <= n_accept.unsqueeze(-1), tokens, torch.full_like(tokens, -1))
    return n_accept.int(), tokens


# ------------------------------------------------------------------ the definitions in 64 bits
def exact(case, seed):
    state = prepare(case, seed)
    if case["op"] == "append":
        return _exact_append(case, state)
    return _exact_attention(case, state) if case["op"] == "attention" else _exact_sample(case, state)


def _exact_append(case, state):
    B, T, Hq, Hkv, D, rot = (case[k] for k in ("B", "T", "Hq", "Hkv", "D", "rot"))
    x = state["qkv"].cpu().numpy().reshape(B, T, Hq + 2 * Hkv, D).astype(np.float64)
    at = np.array(_first_positions(case), dtype=np.float64)[:, None] + np.arange(T)
    angle = at[:, :, None, None] * np.array(_frequencies(case))
    turn = np.cos(angle) + 1j * np.sin(angle)
    head = x[:, :, :Hq + Hkv]
    if case["interleaved"]:
        z = (head[..., 0:rot:2] + 1j * head[..., 1:rot:2]) * turn
        head[..., 0:rot:2], head[..., 1:rot:2] = z.real, z.imag
    else:
        z = (head[..., :rot // 2] + 1j * head[..., rot // 2:rot]) * turn
        head[..., :rot // 2], head[..., rot // 2:rot] = z.real, z.imag
    out = [torch.from_numpy(np.ascontiguousarray(head[:, :, :Hq]))]
    for t in (head[:, :, Hq:].astype(np.float16).astype(np.float64), x[:, :, Hq + Hkv:]):
        low = t.min(-1, keepdims=True)
        step = ((t.max(-1, keepdims=True) - low) / 15.0).astype(np.float16).astype(np.float64)
        codes = np.clip(np.rint((t - low) / np.where(step > 0, step, np.inf)), 0, 15)
        out.append(torch.from_numpy(codes * step + low))
    return tuple(out)


def _exact_attention(case, state):
    B, T, Hq, Hkv, D, P = (case[k] for k in ("B", "T", "Hq", "Hkv", "D", "page"))
    each, n_pages = _pages(case)
    table = torch.arange(n_pages, device="cuda").view(B, each) if state["table"] is None else state["table"].long()
    position = [0] * 8                                         # features of a byte pair by bits: undo the order of the codes
    for e in range(8):
        position[4 * (e % 2) + e // 2] = e
    group = Hq // Hkv
    out = torch.zeros((B, T, Hq, D), dtype=torch.float64, device="cuda")
    for b, first in enumerate(_first_positions(case)):
        n = max(first + T, 0)
        if n == 0:
            continue
        pages = state["cache"][table[b, :-(-n // P)]].view(-1, Hkv, P * (D + 8))
        at = torch.arange(first, first + T, device="cuda").view(T, 1, 1)
        key = torch.arange(n, device="cuda")
        seen = (key >= 0) & (key <= at)
        if case["window"]:
            seen &= (at - key < case["window"]) | (key < case["sinks"])
        seen = seen.expand(T, group, n).reshape(T * group, n)
        for h in range(Hkv):
            params = pages[:, h, P * D:].contiguous().view(torch.float16).view(-1, 4)[:n].double()
            both = []
            for raw in (pages[:, h, :P * D // 2].reshape(-1, P, D // 8, 4),
                        pages[:, h, P * D // 2:P * D].reshape(-1, P // 16, D // 8, 16, 4).transpose(2, 3).reshape(-1, P, D // 8, 4)):
                nibbles = torch.stack((raw & 15, raw >> 4), -1).flatten(-2)                      # by bit position
                codes = torch.empty_like(nibbles)
                codes[..., position] = nibbles
                both.append(codes.reshape(-1, D)[:n].double())
            k = both[0] * params[:, :1] + params[:, 1:2]
            v = both[1] * params[:, 2:3] + params[:, 3:]
            q = state["q"][b, :, h * group:(h + 1) * group].double().reshape(T * group, D)
            scores = (q @ k.t().contiguous()) / math.sqrt(D)
            weights = torch.softmax(scores.masked_fill(~seen, float("-inf")), -1).nan_to_num(0.0)
            out[b, :, h * group:(h + 1) * group] = (weights @ v).view(T, group, D)
    return out


def _exact_sample(case, state):
    B, rows, V = case["B"], case["gamma"] + 1, case["V"]
    logits = state["logits"].cpu().numpy().astype(np.float64)
    uniform, temperature, top_k, top_p, min_p = (state[k].cpu().numpy().astype(np.float64)
                                                 for k in ("uniform", "temperature", "top_k", "top_p", "min_p"))
    tokens = np.zeros((B, rows), dtype=np.int32)
    for b in range(B):
        for j in range(rows):
            x = logits[b, j]
            order = np.argsort(-x, kind="stable")
            if temperature[b] <= 0:
                tokens[b, j] = order[0]
                continue
            mass = np.exp((x[order] - x[order[0]]) / temperature[b])
            n = int(np.count_nonzero(mass >= min_p[b]))
            if top_k[b] > 0:
                n = min(n, int(top_k[b]))
            running = np.cumsum(mass[:n])
            if top_p[b] < 1.0:
                n = min(n, int(np.searchsorted(running, top_p[b] * running[-1], side="left")) + 1)
            tokens[b, j] = order[min(int(np.searchsorted(running[:n], uniform[b, j] * running[n - 1], side="right")), n - 1)]
    if state["draft"] is None:
        return torch.from_numpy(tokens)
    draft = state["draft"].cpu().numpy()
    n_accept = np.zeros(B, dtype=np.int32)
    for b in range(B):
        while n_accept[b] < rows - 1 and tokens[b, n_accept[b]] == draft[b, n_accept[b]]:
            n_accept[b] += 1
        tokens[b, n_accept[b] + 1:] = -1
    return torch.from_numpy(n_accept), torch.from_numpy(tokens)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    if case["op"] == "sample":
        n = case["B"] * (case["gamma"] + 1)
        return dict(bytes=2 * n * case["V"] + 8 * n, flops=4 * n * case["V"])
    B, T, Hq, Hkv, D = (case[k] for k in ("B", "T", "Hq", "Hkv", "D"))
    if case["op"] == "append":
        new = B * T * Hkv
        # q, k, v in; q, the cache's rows and their values out
        return dict(bytes=2 * B * T * D * (2 * Hq + 2 * Hkv) + new * (D + 8) + 4 * new * D, flops=3 * B * T * case["rot"] * (Hq + Hkv) + 6 * new * 2 * D)
    read = pairs = 0
    for first in _first_positions(case):
        rows = [p for p in (first, first + T - 1) if p >= 0]
        if not rows:
            continue
        last, window = first + T - 1, case["window"] or (1 << 40)
        low = max(0, rows[0] - window + 1)
        read += last + 1 - low + min(low, case["sinks"])
        for p in range(max(first, 0), last + 1):
            start = max(0, p - window + 1)
            pairs += p + 1 - start + min(start, case["sinks"])
    return dict(bytes=read * Hkv * (D + 8) + 4 * B * T * Hq * D, flops=4 * D * Hq * pairs)
