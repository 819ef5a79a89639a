"""What long contexts add to a decoder step on the 4-bit key/value cache, as cases that can be timed: attention for
sequences that share a prefix, the bounds of each page's keys, the choice of pages by those bounds, and attention over the chosen pages.

Every pass exists twice.  With `own` false, `run` computes it in its plain form, from elementary tensor operations;
with `own` true it makes the calls a program makes of `paper_2410_11305_amd.binding`.  Both read the same inputs in
their documented byte layouts:

  a page of the cache holds page_size tokens of every key/value head; per head, D features each,
    page_size rows of D/2 bytes       key codes: 32-bit words of 8 codes, features 8w .. 8w+7 in word w
    page_size / 16 tiles of 8 D bytes value codes: word (w, t) of a tile, features 8w .. 8w+7 of its token t, at w * 16 + t
    page_size rows of 4 fp16          key step, key minimum, value step, value minimum
  code e of a word sits at bit 4 * (4 (e % 2) + e // 2); a value is code * step + minimum
  the bounds of a page are, per key/value head, D bytes of upper and D bytes of lower codes (signed), then a binary32
    grid for every head, the whole filled up to 16 bytes; a bound is code * grid

Token t of sequence b lies in row t % page_size of page table[b][t // page_size].
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

# (query heads, key/value heads, features per head) of Llama-shaped blocks
HEADS = {"7b": (32, 32, 128), "70b": (64, 8, 128)}


def _shared(name, heads, groups, each, T, prefix, spread, longest, page):
    """`groups` sets of `each` sequences; prefixes of prefix - spread .. prefix tokens, up to `longest` of its own for a sequence."""
    Hq, Hkv, D = heads
    return dict(name=name, op="shared", Hq=Hq, Hkv=Hkv, D=D, groups=groups, B=groups * each, T=T, prefix=prefix, spread=spread,
                longest=longest, page=page)


def _paged(op, name, heads, B, T, longest, shortest, page, **more):
    Hq, Hkv, D = heads
    return dict(name=name, op=op, Hq=Hq, Hkv=Hkv, D=D, B=B, T=T, longest=longest, shortest=shortest, page=page, **more)


def listed():
    return [
        # four samples of one short prompt, one token each: latency
        _shared("shared_7b_4_samples", HEADS["7b"], 1, 4, 1, 500, 0, 40, 16),
        # the verify pass of 8 users behind one system prompt, every head with its own keys
        _shared("shared_7b_verify_b8", HEADS["7b"], 1, 8, 4, 2000, 0, 600, 64),
        # 128 users behind one long prompt that ends inside a page, one token each
        _shared("shared_70b_b128", HEADS["70b"], 1, 128, 1, 8197, 0, 1500, 64),
        # 16 prompts of different lengths, 8 samples each, verify passes, smaller heads
        _shared("shared_16x8_verify", (64, 8, 64), 16, 8, 4, 6000, 4500, 700, 128),
        # the bounds behind one user's append
        _paged("bounds", "bounds_7b_b1", HEADS["7b"], 1, 1, 4000, 4000, 64),
        # ... and behind a chunk of a long document
        _paged("bounds", "bounds_prompt_2050", HEADS["7b"], 1, 2050, 34050, 34050, 64),
        # one user, a long context: 64 of 2048 pages
        _paged("select", "select_70b_b1", HEADS["70b"], 1, 1, 131071, 131071, 64, count=64, first=1, last=2),
        # the verify pass of 32 ragged sequences
        _paged("select", "select_70b_verify_b32", HEADS["70b"], 32, 4, 32768, 3000, 64, count=32, first=1, last=2),
        # one user's draft token on a sixth of a shorter context
        _paged("blocks", "blocks_7b_b1", HEADS["7b"], 1, 1, 6000, 6000, 64, count=16),
        # a long context, one token, 64 of 2048 pages
        _paged("blocks", "blocks_70b_b1_long", HEADS["70b"], 1, 1, 131071, 131071, 64, count=64),
        # drafts of 64 users, larger pages
        _paged("blocks", "blocks_70b_b64", HEADS["70b"], 64, 1, 32768, 1500, 256, count=16),
        # the verify pass of 32 ragged sequences, every row with pages of its own, smaller heads
        _paged("blocks", "blocks_d64_verify_b32", (64, 8, 64), 32, 4, 32768, 3000, 64, count=32),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("shared", "shared", "bounds", "select", "blocks", "blocks"))
    Hkv = rng.choice((1, 2, 4, 5, 8, 32))
    group = rng.choice((1, 2, 4, 7, 8)) if Hkv <= 8 else 1
    heads = (Hkv * group, Hkv, rng.choice((64, 128, 128)))
    T = rng.choice((1, 1, rng.randint(2, 9)))
    tokens = 3e8 / (Hkv * (heads[2] + 8))                          # read in one pass at most, less than by the longest listed one
    if op == "shared":
        page = rng.choice((16, 32, 64, 128, 256))
        each, groups = rng.choice(((1, 3), (2, 8), (7, 4), (8, 16), (33, 1), (64, 1), (128, 1)))
        prefix = _log_int(rng, 1, min(20000, int(tokens / groups)))
        prefix = max(1, min(prefix, int(4e9 / (heads[0] * groups * each * T))))
        longest = T + _log_int(rng, 1, max(1, min(2000, int(tokens / (groups * each)))))
        case = _shared("", heads, groups, each, T, prefix, rng.randint(0, prefix - 1), longest, page)
    else:
        page = rng.choice((64, 64, 128, 256))
        if op == "bounds":
            T = rng.choice((1, 4, _log_int(rng, 10, 2050)))
            B = _log_int(rng, 1, max(1, 2050 // T))
            low = _log_int(rng, 1, 5000)
            longest = T + low + _log_int(rng, 1, 5000)
            case = _paged(op, "", heads, B, T, longest, T + low, page)
        else:
            B = _log_int(rng, 1, 64)
            longest = T + _log_int(rng, 1, max(1, min(131072, int(12 * tokens / B))))
            count = _log_int(rng, 1, max(1, min(96, int(tokens / (B * T * page)))))
            shortest = max(1, int(longest * rng.random()))
            case = _paged(op, "", heads, B, T, longest, shortest, page, count=count)
            if op == "select":
                case["first"] = rng.randint(0, min(2, count))
                case["last"] = rng.randint(0, min(4, count - case["first"]))
    del case["name"]
    return case


# ------------------------------------------------------------------ inputs
def _lengths(case):
    """Tokens of each sequence, the new ones among them."""
    at = [(i * 0.6180339887498949) % 1.0 for i in range(case["B"])]
    if case["op"] == "shared":
        prefixes, each = _prefixes(case), case["B"] // case["groups"]
        low, high = case["T"], case["longest"]
        return [prefixes[i // each] + high - int((high - low) * a) for i, a in enumerate(at)]
    low, high = min(case["shortest"], case["longest"]), case["longest"]
    return [max(case["T"], high - int((high - low) * a)) for a in at]


def _prefixes(case):
    return [case["prefix"] - int(case["spread"] * ((i * 0.6180339887498949) % 1.0)) for i in range(case["groups"])]


def _first_positions(case):
    return [n - case["T"] for n in _lengths(case)]


def _each(case):
    """Pages of a sequence."""
    return -(-max(_lengths(case)) // case["page"])


def _random_cache(case, gen, n_pages):
    """A cache as a long run of a model leaves it: codes of every value, steps about a sixth of a deviation."""
    Hkv, P, D = case["Hkv"], case["page"], case["D"]
    cache = torch.randint(0, 256, (n_pages, Hkv, P * (D + 8)), dtype=torch.uint8, device="cuda", generator=gen)
    step = 0.15 + 0.15 * torch.rand((n_pages, Hkv, P, 2), device="cuda", generator=gen)
    minimum = -step * (6.5 + 2.0 * torch.rand((n_pages, Hkv, P, 2), device="cuda", generator=gen))
    cache[:, :, P * D:] = torch.stack((step[..., 0], minimum[..., 0], step[..., 1], minimum[..., 1]), -1).half().view(torch.uint8).flatten(2)
    return cache.view(n_pages, Hkv * P * (D + 8))


def _bounds_bytes(case):
    return case["Hkv"] * 2 * case["D"] + -(-4 * case["Hkv"] // 16) * 16


def _random_bounds(case, gen, n_pages):
    """Bounds as pages of keys have them: a feature's middle, and a width about it, that differ from page to page."""
    Hkv, D = case["Hkv"], case["D"]
    middle = 20.0 * torch.randn((1, Hkv, D), device="cuda", generator=gen) + 8.0 * torch.randn((n_pages, Hkv, D), device="cuda", generator=gen)
    width = 50.0 + 6.0 * torch.randn((2, n_pages, Hkv, D), device="cuda", generator=gen)
    codes = torch.stack((middle + width[0], middle - width[1]), 2).clamp(-127, 127).round().to(torch.int8)
    grid = torch.where(torch.rand((n_pages, Hkv), device="cuda", generator=gen) < 0.1, 2.0 ** -4, 2.0 ** -5)
    out = torch.zeros((n_pages, _bounds_bytes(case)), dtype=torch.uint8, device="cuda")
    out[:, :Hkv * 2 * D] = codes.view(n_pages, -1).view(torch.uint8)
    out[:, Hkv * 2 * D:Hkv * 2 * D + 4 * Hkv] = grid.view(torch.uint8)
    return out


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    op = case["op"]
    B, T, Hq, Hkv, D = (case[k] for k in ("B", "T", "Hq", "Hkv", "D"))
    each = _each(case)
    state = dict(case, pos=torch.tensor(_first_positions(case), dtype=torch.int32, device="cuda"), lengths=_lengths(case))
    if op == "shared":
        # the pages of a group's whole prefix are the same; the page in which it ends is everyone's own
        prefixes, per = _prefixes(case), B // case["groups"]
        table, n_pages = [], 0
        for b in range(B):
            whole = prefixes[b // per] // case["page"]
            before = table[b - b % per][:whole] if b % per else []
            table.append(before + list(range(n_pages, n_pages + each - len(before))))
            n_pages += each - len(before)
        order = torch.randperm(n_pages, device="cuda", generator=gen).int()
        state["table"] = order[torch.tensor(table, device="cuda")]
        state["shared"] = torch.tensor(prefixes, dtype=torch.int32, device="cuda")
        state["prefixes"] = prefixes
    else:
        n_pages = B * each
        state["table"] = torch.randperm(n_pages, device="cuda", generator=gen).int().view(B, each)
    if op == "select":
        state["bounds"] = _random_bounds(case, gen, n_pages)
    else:
        state["cache"] = _random_cache(case, gen, n_pages)
    if op == "bounds":
        state["bounds"] = torch.zeros((n_pages, _bounds_bytes(case)), dtype=torch.uint8, device="cuda")
        # the plain form keeps them as numbers
        state["upper"], state["lower"] = (torch.zeros((n_pages, Hkv, D), device="cuda") for _ in range(2)) if not own else (
            torch.empty((B, (T - 1) // case["page"] + 2, Hkv, D), device="cuda") for _ in range(2))
        return state
    state["q"] = torch.randn((B, T, Hq, D), device="cuda", generator=gen).half()
    if op == "blocks":
        # a row's pages: the first, its last, and others by chance, in order; -1 where there are not as many
        count = case["count"]
        n = (state["pos"].view(B, 1) + torch.arange(T, device="cuda")) // case["page"] + 1                  # pages in sight
        weight = torch.rand((B, T, Hkv, each), device="cuda", generator=gen)
        index = torch.arange(each, device="cuda")
        n = n.view(B, T, 1, 1)
        weight = torch.where(index >= n, weight - 2.0, torch.where((index == 0) | (index == n - 1), weight + 2.0, weight))
        weight, chosen = torch.topk(weight, min(count, each), dim=-1)
        chosen = torch.where(weight < -0.5, torch.full_like(chosen, each), chosen).sort(-1).values
        blocks = torch.full((B, T, Hkv, count), -1, dtype=torch.int32, device="cuda")
        blocks[..., :chosen.shape[-1]] = torch.where(chosen == each, torch.full_like(chosen, -1), chosen).int()
        state["blocks"] = blocks
    if own:
        from paper_2410_11305_amd import binding
        if op == "select":
            state["out"] = torch.empty((B, T, Hkv, case["count"]), dtype=torch.int32, device="cuda")
            size = binding.kv4_select_workspace_bytes(B, T, Hq, Hkv, each)
        else:
            state["out"] = torch.empty_like(state["q"])
            size = (binding.attn_kv4_shared_workspace_bytes(B, T, Hq, Hkv, D, case["groups"]) if op == "shared"
                    else binding.attn_kv4_blocks_workspace_bytes(B, T, Hq, Hkv, D))
        state["workspace"] = binding.alloc_workspace(size)
    return state


# ------------------------------------------------------------------ one pass
def run(state):
    op = state["op"]
    if own:
        from paper_2410_11305_amd import binding
        if op == "shared":
            return binding.attn_kv4_shared(state["q"], state["cache"], state["pos"], state["shared"], state["Hkv"], state["page"],
                                           state["table"], out=state["out"], workspace=state["workspace"])
        if op == "bounds":
            binding.kv4_bounds(state["cache"], state["pos"], state["T"], state["bounds"], state["Hkv"], state["D"], state["page"], state["table"])
            return binding.kv4_bounds_read(state["bounds"], state["pos"], state["T"], state["Hkv"], state["D"], state["page"], state["table"],
                                           upper=state["upper"], lower=state["lower"])
        if op == "select":
            return binding.kv4_select(state["q"], state["bounds"], state["pos"], state["Hkv"], state["page"], state["count"], state["table"],
                                      first=state["first"], last=state["last"], blocks=state["out"], workspace=state["workspace"])
        return binding.attn_kv4_blocks(state["q"], state["cache"], state["pos"], state["blocks"], state["Hkv"], state["page"], state["table"],
                                       out=state["out"], workspace=state["workspace"])
    return dict(shared=_plain_shared, bounds=_plain_bounds, select=_plain_select, blocks=_plain_blocks)[op](state)


# ---- plain forms
_NIBBLE = [4 * (4 * (e % 2) + e // 2) for e in range(8)]       # bit of code e in its word


def _plain_pages(state, index, keys_only=False):
    """Keys and values [..., P, D] in float32 of the heads' pages of index [..., Hkv]."""
    Hkv, D, P = (state[k] for k in ("Hkv", "D", "page"))
    raw = state["cache"].view(-1, Hkv, P * (D + 8))[index.long(), torch.arange(Hkv, device="cuda")]        # [..., Hkv, bytes]
    shape = raw.shape[:-1]
    params = raw[..., P * D:].contiguous().view(torch.float16).view(*shape, P, 4).float()
    shifts = torch.tensor(_NIBBLE, dtype=torch.int32, device="cuda")
    k = raw[..., :P * D // 2].contiguous().view(torch.int32).view(*shape, P, D // 8)
    v = raw[..., P * D // 2:P * D].contiguous().view(torch.int32).view(*shape, P // 16, D // 8, 16).transpose(-1, -2)
    out = []
    for words, step in ((k, 0), (v, 2))[:1 if keys_only else 2]:
        codes = ((words.reshape(*shape, P, D // 8, 1) >> shifts) & 15).float().flatten(-2)
        out.append(codes * params[..., step:step + 1] + params[..., step + 1:step + 2])
    return out


def _plain_tokens(state, table, tokens):
    """Keys and values [N, Hkv, tokens, D] of the first tokens of the table's rows [N, pages]."""
    Hkv, D, P = (state[k] for k in ("Hkv", "D", "page"))
    pages = -(-tokens // P)
    index = table[:, :pages].unsqueeze(-1).expand(-1, -1, Hkv)
    return [x.permute(0, 2, 1, 3, 4).reshape(-1, Hkv, pages * P, D)[:, :, :tokens] for x in _plain_pages(state, index)]


def _plain_shared(state):
    B, T, Hq, Hkv, D, groups, P = (state[k] for k in ("B", "T", "Hq", "Hkv", "D", "groups", "page"))
    per, G = B // groups, Hq // Hkv
    longest = max(state["prefixes"])
    k1, v1 = _plain_tokens(state, state["table"][::per], longest)                                          # once a group
    # the others from the page in which the prefix ends
    start = state["shared"].long().repeat_interleave(per) // P                                             # [B]
    pages = max((n - 1) // P - state["prefixes"][b // per] // P for b, n in enumerate(state["lengths"])) + 1
    index = (start.view(B, 1) + torch.arange(pages, device="cuda")).clamp(max=state["table"].shape[1] - 1)
    own_table = torch.gather(state["table"].long(), 1, index)
    k2, v2 = _plain_tokens(state, own_table, pages * P)
    q = state["q"].float().view(groups, per * T, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(groups, Hkv, per * T * G, D)
    q2 = state["q"].float().view(B, T, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, T * G, D)
    at = state["pos"].long().view(B, 1) + torch.arange(T, device="cuda")
    s1 = torch.matmul(q, k1.transpose(-1, -2).contiguous()) * (1.0 / math.sqrt(D))
    limit = torch.minimum(at.view(groups, per * T), state["shared"].long().view(groups, 1) - 1)
    seen = torch.arange(longest, device="cuda") <= limit.view(groups, per * T, 1)
    s1 = s1.masked_fill(~seen.unsqueeze(2).expand(-1, -1, G, -1).reshape(groups, 1, per * T * G, longest), float("-inf"))
    s2 = torch.matmul(q2, k2.transpose(-1, -2).contiguous()) * (1.0 / math.sqrt(D))
    t = (start * P).view(B, 1, 1) + torch.arange(pages * P, device="cuda")
    seen = (t <= at.unsqueeze(-1)) & (t >= state["shared"].long().repeat_interleave(per).view(B, 1, 1))
    s2 = s2.masked_fill(~seen.unsqueeze(2).expand(-1, -1, G, -1).reshape(B, 1, T * G, pages * P), float("-inf"))
    s1 = s1.view(groups, Hkv, per, T * G, longest).permute(0, 2, 1, 3, 4).reshape(B, Hkv, T * G, longest)
    top = torch.maximum(s1.amax(-1, keepdim=True), s2.amax(-1, keepdim=True))
    w1, w2 = torch.exp(s1 - top), torch.exp(s2 - top)
    total = w1.sum(-1, keepdim=True) + w2.sum(-1, keepdim=True)
    w1 = w1.view(groups, per, Hkv, T * G, longest).permute(0, 2, 1, 3, 4).reshape(groups, Hkv, per * T * G, longest)
    o1 = torch.matmul(w1, v1).view(groups, Hkv, per, T * G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, T * G, D)
    out = (o1 + torch.matmul(w2, v2)) / total
    return out.view(B, Hkv, T, G, D).permute(0, 2, 1, 3, 4).reshape(B, T, Hq, D).half()


def _power_of_two_grid(top):
    """The smallest power of two with top <= 127 of it; 1 for zeros."""
    m, e = torch.frexp(top)
    e = e - 7 + (m > 127.0 / 128.0).int()
    return torch.where(top > 0, torch.ldexp(torch.ones_like(top), e), torch.ones_like(top))


def _plain_bounds(state):
    B, T, Hkv, D, P = (state[k] for k in ("B", "T", "Hkv", "D", "page"))
    touched = (T - 1) // P + 2
    first = state["pos"].long().view(B, 1) // P
    number = first + torch.arange(touched, device="cuda")                                                  # [B, touched]
    last = state["pos"].long().view(B, 1) + T - 1
    there = (number * P <= last) & (number < state["table"].shape[1])
    page = torch.gather(state["table"].long(), 1, number.clamp(max=state["table"].shape[1] - 1))
    k, = _plain_pages(state, page.unsqueeze(-1).expand(-1, -1, Hkv), keys_only=True)                       # [B, touched, Hkv, P, D]
    seen = (number.unsqueeze(-1) * P + torch.arange(P, device="cuda") <= last.unsqueeze(-1)).view(B, touched, 1, P, 1)
    upper = torch.where(seen, k, torch.full_like(k, float("-inf"))).amax(-2)
    lower = torch.where(seen, k, torch.full_like(k, float("inf"))).amin(-2)
    grid = _power_of_two_grid(torch.maximum(upper.abs(), lower.abs()).amax(-1, keepdim=True))
    upper, lower = torch.ceil(upper / grid) * grid, torch.floor(lower / grid) * grid
    state["upper"][page[there]] = upper[there]
    state["lower"][page[there]] = lower[there]
    keep = there.view(B, touched, 1, 1)
    return torch.where(keep, upper, torch.zeros_like(upper)), torch.where(keep, lower, torch.zeros_like(lower))


def _plain_select(state):
    """Scores of whole numbers: sums below 2^24 are exact in float32."""
    B, T, Hq, Hkv, D, P, count, first, last = (state[k] for k in ("B", "T", "Hq", "Hkv", "D", "page", "count", "first", "last"))
    G, pages = Hq // Hkv, state["table"].shape[1]
    raw = state["bounds"][state["table"].long()]                                                           # [B, pages, bytes]
    codes = raw[..., :Hkv * 2 * D].contiguous().view(torch.int8).view(B, pages, Hkv, 2, D).float().permute(0, 2, 3, 4, 1)       # [B, Hkv, 2, D, pages]
    grid = raw[..., Hkv * 2 * D:Hkv * 2 * D + 4 * Hkv].contiguous().view(torch.float32).permute(0, 2, 1)   # [B, Hkv, pages]
    q = state["q"].float().view(B, T, Hkv, G * D)
    q = torch.round(q / _power_of_two_grid(q.abs().amax(-1, keepdim=True))).view(B, T, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, T * G, D)
    dots = torch.matmul(q.clamp(min=0), codes[:, :, 0].contiguous()) + torch.matmul(q.clamp(max=0), codes[:, :, 1].contiguous())
    score = dots.view(B, Hkv, T, G, pages).amax(3) * grid.unsqueeze(2)                                     # [B, Hkv, T, pages]
    n = ((state["pos"].long().view(B, 1) + torch.arange(T, device="cuda")) // P + 1).view(B, 1, T, 1)
    index = torch.arange(pages, device="cuda")
    score = torch.where((index < first) | (index >= n - last), torch.full_like(score, float("inf")), score)
    score = torch.where(index < n, score, torch.full_like(score, float("-inf")))
    chosen = torch.sort(score, dim=-1, descending=True, stable=True).indices[..., :count]
    rank = torch.arange(chosen.shape[-1], device="cuda")
    chosen = torch.where(rank < n, chosen, torch.full_like(chosen, pages)).sort(-1).values
    out = torch.full((B, Hkv, T, count), -1, dtype=torch.int32, device="cuda")
    out[..., :chosen.shape[-1]] = torch.where(chosen == pages, torch.full_like(chosen, -1), chosen).int()
    return out.permute(0, 2, 1, 3).contiguous()


def _plain_blocks(state):
    B, T, Hq, Hkv, D, P, count = (state[k] for k in ("B", "T", "Hq", "Hkv", "D", "page", "count"))
    G = Hq // Hkv
    blocks = state["blocks"].long()                                                                        # [B, T, Hkv, count]
    table = state["table"].long().view(B, 1, 1, -1).expand(B, T, Hkv, -1)
    page = torch.gather(table, -1, blocks.clamp(min=0)).permute(0, 1, 3, 2)                                # [B, T, count, Hkv]
    k, v = (x.permute(0, 1, 3, 2, 4, 5).reshape(B, T, Hkv, count * P, D) for x in _plain_pages(state, page))
    q = state["q"].float().view(B, T, Hkv, G, D)
    scores = torch.matmul(q, k.transpose(-1, -2).contiguous()) * (1.0 / math.sqrt(D))                      # [B, T, Hkv, G, tokens]
    t = (blocks.unsqueeze(-1) * P + torch.arange(P, device="cuda")).flatten(-2)
    at = (state["pos"].long().view(B, 1) + torch.arange(T, device="cuda")).view(B, T, 1, 1)
    scores = scores.masked_fill(((t < 0) | (t > at)).unsqueeze(-2), float("-inf"))
    weights = torch.exp(scores - scores.amax(-1, keepdim=True))
    out = torch.matmul(weights, v) / weights.sum(-1, keepdim=True)
    return out.reshape(B, T, Hq, D).half()


# ------------------------------------------------------------------ the definitions in 64 bits
def exact(case, seed):
    state = prepare(case, seed)
    return dict(shared=_exact_shared, bounds=_exact_bounds, select=_exact_select, blocks=_exact_blocks)[case["op"]](case, state)


def _exact_rows(case, cache, pages, h):
    """Keys and values [len(pages) * P, D] of head h in float64."""
    Hkv, D, P = case["Hkv"], case["D"], case["page"]
    position = [0] * 8                                         # features of a byte quadruple by bits: undo the order of the codes
    for e in range(8):
        position[4 * (e % 2) + e // 2] = e
    raw = cache.view(-1, Hkv, P * (D + 8))[pages.long(), h]
    params = raw[:, P * D:].contiguous().view(torch.float16).view(-1, 4).double()
    both = []
    for part in (raw[:, :P * D // 2].reshape(-1, P, D // 8, 4),
                 raw[:, P * D // 2:P * D].reshape(-1, P // 16, D // 8, 16, 4).transpose(2, 3).reshape(-1, P, D // 8, 4)):
        nibbles = torch.stack((part & 15, part >> 4), -1).flatten(-2)
        codes = torch.empty_like(nibbles)
        codes[..., position] = nibbles
        both.append(codes.reshape(-1, D).double())
    return both[0] * params[:, :1] + params[:, 1:2], both[1] * params[:, 2:3] + params[:, 3:]


def _exact_shared(case, state):
    B, T, Hq, Hkv, D, P = (case[k] for k in ("B", "T", "Hq", "Hkv", "D", "page"))
    per, G = B // case["groups"], Hq // Hkv
    out = torch.zeros((B, T, Hq, D), dtype=torch.float64, device="cuda")
    for h in range(Hkv):
        for g, prefix in enumerate(_prefixes(case)):
            k1, v1 = (x[:prefix] for x in _exact_rows(case, state["cache"], state["table"][g * per, :-(-prefix // P)], h))
            for b in range(g * per, (g + 1) * per):
                n, skip = state["lengths"][b], prefix // P
                k2, v2 = (x[prefix - skip * P:n - skip * P] for x in _exact_rows(case, state["cache"], state["table"][b, skip:-(-n // P)], h))
                k, v = torch.cat((k1, k2)), torch.cat((v1, v2))
                q = state["q"][b, :, h * G:(h + 1) * G].double().reshape(T * G, D)
                at = torch.arange(n - T, n, device="cuda").view(T, 1, 1)
                seen = (torch.arange(n, device="cuda") <= at).expand(T, G, n).reshape(T * G, n)
                weights = torch.softmax(((q @ k.t().contiguous()) / math.sqrt(D)).masked_fill(~seen, float("-inf")), -1)
                out[b, :, h * G:(h + 1) * G] = (weights @ v).view(T, G, D)
    return out


def _exact_bounds(case, state):
    B, T, Hkv, D, P = (case[k] for k in ("B", "T", "Hkv", "D", "page"))
    touched = (T - 1) // P + 2
    out = torch.zeros((2, B, touched, Hkv, D), dtype=torch.float64, device="cuda")
    for b, n in enumerate(state["lengths"]):
        for i in range(touched):
            page = (n - T) // P + i
            if page * P >= n:
                continue
            for h in range(Hkv):
                keys = _exact_rows(case, state["cache"], state["table"][b, page:page + 1], h)[0][:n - page * P].float().double()
                upper, lower = keys.amax(0), keys.amin(0)
                top = float(torch.maximum(upper.abs(), lower.abs()).max())
                grid = 2.0 ** math.ceil(math.log2(top / 127.0)) if top > 0 else 1.0
                grid = grid * 2.0 if top > 127.0 * grid else grid / 2.0 if 0 < top <= 63.5 * grid else grid
                out[0, b, i, h], out[1, b, i, h] = torch.ceil(upper / grid) * grid, torch.floor(lower / grid) * grid
    return out[0], out[1]


def _exact_select(case, state):
    B, T, Hq, Hkv, D, P, count = (case[k] for k in ("B", "T", "Hq", "Hkv", "D", "page", "count"))
    G = Hq // Hkv
    bounds, table = state["bounds"].cpu().numpy(), state["table"].cpu().numpy()
    q = state["q"].cpu().numpy().astype(np.float64)
    out = np.full((B, T, Hkv, count), -1, dtype=np.int32)
    for b, length in enumerate(state["lengths"]):
        for h in range(Hkv):
            rows = bounds[table[b]]
            codes = rows[:, h * 2 * D:(h + 1) * 2 * D].view(np.int8).astype(np.int64)
            grid = rows[:, Hkv * 2 * D + 4 * h:Hkv * 2 * D + 4 * h + 4].copy().view(np.float32)[:, 0].astype(np.float64)
            for j in range(T):
                x = q[b, j, h * G:(h + 1) * G]
                top, unit = np.abs(x).max(), 1.0
                while top > 127.0 * unit:
                    unit *= 2.0
                while 0 < top <= 63.5 * unit:
                    unit /= 2.0
                x = np.rint(x / unit).astype(np.int64)
                n = (length - T + j) // P + 1
                bound = np.maximum(x, 0) @ codes[:n, :D].T + np.minimum(x, 0) @ codes[:n, D:].T
                score = bound.max(0) * grid[:n]
                score[:case["first"]] = np.inf
                score[max(n - case["last"], 0):] = np.inf
                best = np.sort(np.argsort(-score, kind="stable")[:count])
                out[b, j, h, :len(best)] = best
    return torch.from_numpy(out)


def _exact_blocks(case, state):
    B, T, Hq, Hkv, D, P = (case[k] for k in ("B", "T", "Hq", "Hkv", "D", "page"))
    G = Hq // Hkv
    out = torch.zeros((B, T, Hq, D), dtype=torch.float64, device="cuda")
    listed_pages = state["blocks"].cpu().numpy()
    for b, length in enumerate(state["lengths"]):
        for j in range(T):
            for h in range(Hkv):
                mine = torch.tensor([i for i in listed_pages[b, j, h] if i >= 0], device="cuda")
                k, v = _exact_rows(case, state["cache"], state["table"][b][mine], h)
                t = (mine.view(-1, 1) * P + torch.arange(P, device="cuda")).flatten()
                seen = t <= length - T + j
                scores = state["q"][b, j, h * G:(h + 1) * G].double() @ k.t().contiguous() / math.sqrt(D)
                out[b, j, h * G:(h + 1) * G] = torch.softmax(scores.masked_fill(~seen, float("-inf")), -1) @ v
    return out


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    B, T, Hq, Hkv, D, P = (case[k] for k in ("B", "T", "Hq", "Hkv", "D", "page"))
    lengths = _lengths(case)
    if case["op"] == "shared":
        prefixes, per = _prefixes(case), B // case["groups"]
        read = sum(prefixes) + sum(n - prefixes[b // per] for b, n in enumerate(lengths))
        pairs = sum(T * n - T * (T - 1) // 2 for n in lengths)
        return dict(bytes=read * Hkv * (D + 8) + 4 * B * T * Hq * D, flops=4 * D * Hq * pairs)
    if case["op"] == "bounds":
        pages = sum((n - 1) // P - (n - T) // P + 1 for n in lengths)
        tokens = sum(n - (n - T) // P * P for n in lengths)
        # the keys in; the bounds out, and their values out again
        return dict(bytes=tokens * Hkv * (D // 2 + 4) + pages * Hkv * (2 * D + 4) + B * ((T - 1) // P + 2) * Hkv * 8 * D, flops=4 * tokens * Hkv * D)
    seen = [[(n - T + j) // P + 1 for j in range(T)] for n in lengths]
    if case["op"] == "select":
        return dict(bytes=sum(s[-1] for s in seen) * Hkv * (2 * D + 4) + 2 * B * T * Hq * D + 4 * B * T * Hkv * case["count"],
                    flops=sum(map(sum, seen)) * Hq * 4 * D)
    tokens = sum(min(case["count"], s) * P for row in seen for s in row)      # of every row and head
    return dict(bytes=tokens * Hkv * (D + 8) + 4 * B * T * Hq * D + 4 * B * T * Hkv * case["count"], flops=4 * D * Hq * tokens)
