"""Decoding with drafted tokens over the paged FP8 cache, as measurable cases.

Five operators, in the order in which a serving program runs them in one round of drafting:

  tree     mq_draft_tree: for each drafted token the tokens above it in its sequence's tree, as a mask, and its position
  attend   kv8_tree_attention: attention of the drafted tokens' queries over the history and over those above them
  sample   mq_sample: one token from each row of logits, by temperature, top-k, top-p and min-p, from given uniform numbers
  accept   mq_draft_accept: the path of drafted tokens that the sampled ones confirm
  compact  kv8_compact: the confirmed tokens' keys and values brought together in the cache

The plain forms below compute the same from the formulas with elementary torch operations.

Formulas.  New tokens of sequence b are cu_q[b] .. cu_q[b + 1] - 1, the last of its kv_lens[b] places; start = kv_lens[b] - n.  A token's
parent is an earlier token of its sequence by its number there, or -1.  tree: bit j of a token's words (32 to a word) is set where j is the
token itself or above it, positions = start + the number of tokens above it.  attend: softmax over the visible j of scale * q.k_j, times v_j; a
token sees the places j < start, with a window w > 0 those with j > position - w, and of the new tokens those of its mask.  sample:
tokens in the order of falling logits, the lower index first among equals; w = exp((logit - largest) / temperature); kept are the first k,
of those the ones with less than top_p of their mass before them, and of those the ones with w >= min_p, the first always; the result is
the lowest index up to which the kept tokens have more than u of the kept mass; a temperature of zero gives the first.  accept:
from token 0 on to the lowest child whose token is the one sampled at its parent, while there is one; the path, its length, the token
sampled at its end, and the sequence's new length.  compact: place start + path[i] to place start + i; a page's exponent becomes the
smallest that holds what comes from other pages, at least what it was; codes that come or stay are brought to it with one rounding.
"""
import math
import random

import torch

own = False

# a program keeps one workspace per stream: the largest that the library asks for
WORKSPACE = 64 << 20
E4M3_MAX = 448.0
LOWEST, HIGHEST = -112, 119


def _tree(seqs, nodes, lengths=1):
    return {"kind": "tree", "seqs": seqs, "q_lo": nodes[0], "q_hi": nodes[1], "past_lo": 10, "past_hi": 8000, "lengths": lengths}


def _attend(seqs, nodes, past, Hq=32, Hkv=8, D=128, P=64, window=0, lengths=1):
    return {"kind": "attend", "seqs": seqs, "q_lo": nodes[0], "q_hi": nodes[1], "past_lo": past[0], "past_hi": past[1], "Hq": Hq, "Hkv": Hkv,
            "D": D, "P": P, "window": window, "lengths": lengths}


def _sample(rows, V, dtype="bf16", filters="all"):
    return {"kind": "sample", "rows": rows, "V": V, "dtype": dtype, "filters": filters}


def _accept(seqs, nodes, lengths=1):
    return {"kind": "accept", "seqs": seqs, "q_lo": nodes[0], "q_hi": nodes[1], "past_lo": 10, "past_hi": 8000, "lengths": lengths}


def _compact(seqs, nodes, past, Hkv=8, D=128, P=64, lengths=1):
    return {"kind": "compact", "seqs": seqs, "q_lo": nodes[0], "q_hi": nodes[1], "past_lo": past[0], "past_hi": past[1], "Hkv": Hkv, "D": D,
            "P": P, "lengths": lengths}


def listed():
    return [
        # one request with a tree of sixty drafted tokens
        dict(_tree(1, (60, 60)), name="tree_one"),
        # a decode batch, trees of uneven size
        dict(_tree(200, (8, 150)), name="tree_batch"),
        # one request, a tree of sixty after a short history
        dict(_attend(1, (60, 60), (2000, 2000)), name="attend_one"),
        # a decode batch with small trees after uneven histories
        dict(_attend(64, (8, 26), (100, 8000)), name="attend_batch"),
        # two requests deep in a long context, wide trees, pages of 16
        dict(_attend(2, (64, 64), (100000, 131000), P=16), name="attend_long"),
        # the next token of one request, all settings on (latency)
        dict(_sample(1, 131072), name="sample_one"),
        # a decode batch, every request with its own settings, a vocabulary of odd size
        dict(_sample(64, 151673), name="sample_batch"),
        # every node of the trees of a batch, temperature alone, 32-bit logits
        dict(_sample(500, 100003, "fp32", "temperature"), name="sample_nodes"),
        # acceptance for one request, and over a decode batch
        dict(_accept(1, (60, 60)), name="accept_one"),
        dict(_accept(200, (8, 150)), name="accept_batch"),
        # one request's confirmed tokens
        dict(_compact(1, (60, 60), (2000, 2000)), name="compact_one"),
        # those of a decode batch, pages of 16
        dict(_compact(200, (8, 64), (100, 2000), P=16), name="compact_batch"),
    ]


KINDS = ("tree", "attend", "sample", "accept", "compact")


def _span(rng, lo, hi):
    """A size from lo to hi, spread over the logarithm where the range is wide."""
    return rng.randint(lo, hi) if hi < 10 * max(lo, 1) else min(hi, max(lo, int(math.exp(rng.uniform(math.log(max(lo, 1)), math.log(hi + 1))))))


def draw(rng):
    top = {k: max(_cost(c) for c in listed() if c["kind"] == k) for k in KINDS}
    kind = rng.choice(["tree", "attend", "attend", "attend", "sample", "sample", "sample", "accept", "compact"])
    while True:
        if kind == "sample":
            c = _sample(_span(rng, 1, 512), _span(rng, 300, 262144), rng.choice(["bf16", "fp32"]), rng.choice(["all", "all", "temperature"]))
        else:
            seqs = _span(rng, 1, 200)
            q_hi = _span(rng, 1, 64) if rng.random() < 0.7 else _span(rng, 32, 250)
            nodes, lengths = (rng.randint(1, q_hi), q_hi), rng.randrange(1000)
            past_hi = _span(rng, 1, 131072)
            past = (rng.randint(0, past_hi), past_hi)
            h = {"Hkv": rng.choice([1, 2, 4, 5, 8]), "D": rng.choice([64, 128, 256]), "P": rng.choice([16, 32, 64, 128])}
            if kind in ("tree", "accept"):
                c = (_tree if kind == "tree" else _accept)(seqs, (max(nodes[0], 8), max(q_hi, 12)), lengths)
            elif kind == "compact":
                c = _compact(seqs, nodes, (past[0] // 32, past[1] // 32), lengths=lengths, **h)
            else:
                c = _attend(seqs, nodes, past, Hq=h["Hkv"] * rng.choice([1, 2, 3, 4, 7, 8, 12]), window=rng.choice([0, 0, _span(rng, 16, 16384)]),
                            lengths=lengths, **h)
        if _cost(c) <= top[kind] and _padded(c) <= 1 << 31:
            return c


def _lengths(case):
    """New and earlier tokens of each sequence: the same ones for every seed."""
    r = random.Random(case["lengths"])
    q = [r.randint(case["q_lo"], case["q_hi"]) for _ in range(case["seqs"])]
    return q, [r.randint(case["past_lo"], case["past_hi"]) for _ in range(case["seqs"])]


def _padded(case):
    """Values of the plain form's largest tensor."""
    if case["kind"] == "sample":
        return case["rows"] * case["V"]
    q, past = _lengths(case)
    if case["kind"] in ("tree", "accept"):
        return case["seqs"] * max(q) ** 2
    longest = max(a + b for a, b in zip(q, past)) + case["P"]
    cache = case["seqs"] * longest * case["Hkv"] * case["D"]
    return max(cache, case["seqs"] * max(q) * longest * case["Hq"]) if case["kind"] == "attend" else cache


def work(case):
    if case["kind"] == "sample":
        n = case["rows"] * case["V"]
        return {"bytes": n * (2 if case["dtype"] == "bf16" else 4) + 24 * case["rows"], "flops": 2 * n}
    q, past = _lengths(case)
    T, B = sum(q), case["seqs"]
    if case["kind"] == "tree":  # parents in, masks and positions out
        return {"bytes": T * (8 + 4 * _words(q)) + 8 * B, "flops": T}
    if case["kind"] == "accept":  # parents, tokens and sampled tokens in, the path out
        return {"bytes": 16 * T + 20 * B, "flops": T}
    if case["kind"] == "compact":  # a token's codes of keys and values in and out
        n = sum(_accepted(q))
        return {"bytes": 4 * case["Hkv"] * case["D"] * n + 4 * n, "flops": 2 * case["Hkv"] * case["D"] * n}
    Hq, Hkv, D, w = case["Hq"], case["Hkv"], case["D"], case["window"]
    places = [min(b, w) if w > 0 else b for b in past]
    return {"bytes": 4 * T * Hq * D + 2 * Hkv * D * (sum(places) + T) + 4 * T * _words(q), "flops": 4 * D * Hq * (sum(a * b for a, b in zip(q, places)) + T)}


def _words(q):
    return -(-max(q) // 32)


def _accepted(q):
    """Lengths of the confirmed paths."""
    return [1 + (7 * i + 3) % min(n, 9) for i, n in enumerate(q)]


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 50)


def _exponent(amax):
    """The smallest e with amax <= 448 * 2^e, within its bounds."""
    m, e = torch.frexp(amax)  # amax = m * 2^e, 0.5 <= m < 1; 448 = 0.875 * 2^9
    e = torch.where(m <= 0.875, e - 9, e - 8)
    return torch.where(amax > 0, e, torch.full_like(e, LOWEST)).clamp(LOWEST, HIGHEST)


def _codes(x, e):
    """E4M3 codes of x / 2^e: nearest, ties to even, clipped."""
    return torch.ldexp(x, -e).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)


def _pool(gen, pages, Hkv, P, D):
    """A cache that holds tokens: normal values, a few large channels, magnitudes that differ from head to head and page to page."""
    x = torch.randn(pages, Hkv, P, D, device="cuda", generator=gen)
    x *= torch.exp(0.5 * torch.randn(1, Hkv, 1, 1, device="cuda", generator=gen) + 0.2 * torch.randn(pages, 1, 1, 1, device="cuda", generator=gen))
    x[..., torch.randint(0, D, (2,), device="cuda", generator=gen)] *= 3.0
    e = _exponent(x.abs().amax((2, 3)))
    return _codes(x, e[:, :, None, None]).view(torch.uint8), (e + 127).to(torch.uint8)


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _parents(q_lens, seed):
    """A tree for each sequence: token 0 its root, every other one below one of the few before it."""
    r = random.Random(seed)
    return [-1 if i == 0 else max(0, i - 1 - int(9 * r.random() ** 1.5)) for n in q_lens for i in range(n)]


def _sampling(s, case, gen):
    rows, V = case["rows"], case["V"]
    flat = lambda lo, hi: lo + (hi - lo) * torch.rand(rows, device="cuda", generator=gen)  # noqa: E731
    pick = lambda p: torch.rand(rows, device="cuda", generator=gen) < p  # noqa: E731
    # a wide spread of unlikely tokens, and some likely ones; rows of every degree of certainty
    logits = 2.2 * torch.randn(rows, V, device="cuda", generator=gen)
    likely = torch.randint(0, V, (rows, 12), device="cuda", generator=gen)
    logits.scatter_(1, likely, flat(4.0, 16.0)[:, None] + 2.0 * torch.randn(rows, 12, device="cuda", generator=gen))
    s["logits"] = logits.to(torch.bfloat16) if case["dtype"] == "bf16" else logits
    s["uniform"] = torch.rand(rows, device="cuda", generator=gen)
    s["temperature"] = torch.where(pick(0.1), 0.0, flat(0.5, 1.3))
    s["top_k"] = s["top_p"] = s["min_p"] = None
    if case["filters"] == "all":
        s["top_k"] = torch.where(pick(0.4), 0, torch.exp(flat(0.7, 8.0)).int()).int()
        s["top_p"] = torch.where(pick(0.3), 1.0, flat(0.7, 0.99))
        s["min_p"] = torch.where(pick(0.6), 0.0, flat(0.001, 0.1))
    return s


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": case}
    if case["kind"] == "sample":
        return _sampling(s, case, gen)
    q_lens, past = _lengths(case)
    seqs, T = case["seqs"], sum(q_lens)
    total = [a + b for a, b in zip(q_lens, past)]
    first = [sum(q_lens[:i]) for i in range(seqs + 1)]
    s.update(cu_q=_ints(first), kv_lens=_ints(total), max_q=max(q_lens), words=_words(q_lens))
    if case["kind"] != "compact":
        parents = _parents(q_lens, seed)
        s["parents"] = _ints(parents)
    if case["kind"] == "accept":
        # at most nodes the model wants the token of one of the children
        r = random.Random(seed + 1)
        tokens = [r.randrange(100000) for _ in range(T)]
        sampled = [r.randrange(100000) for _ in range(T)]
        for b in range(seqs):
            for i in range(1, q_lens[b]):
                if r.random() < 0.6:
                    sampled[first[b] + parents[first[b] + i]] = tokens[first[b] + i]
        s.update(tokens=_ints(tokens), sampled=_ints(sampled))
    if case["kind"] in ("tree", "accept"):
        return s
    Hkv, D, P = case["Hkv"], case["D"], case["P"]
    held = [-(-n // P) for n in total]
    pages = sum(held) + 3
    order = torch.randperm(pages, device="cuda", generator=gen).to(torch.int32)
    table = torch.zeros(seqs, max(held), dtype=torch.int32, device="cuda")
    width = torch.arange(max(held), device="cuda")
    table[width[None] < _ints(held)[:, None]] = order[: sum(held)]
    s["page_table"] = table
    s["k_codes"], s["k_scales"] = _pool(gen, pages, Hkv, P, D)
    s["v_codes"], s["v_scales"] = _pool(gen, pages, Hkv, P, D)
    if case["kind"] == "compact":
        r, counts = random.Random(seed), _accepted(q_lens)
        path = [i for n, c in zip(q_lens, counts) for i in [0] + sorted(r.sample(range(1, n), c - 1)) + [-1] * (n - c)]
        s.update(path=_ints(path), counts=_ints(counts))
        return s
    s["tree"], s["positions"] = _tree_plain(s)
    s["q"] = (1.5 * torch.randn(T, case["Hq"], D, device="cuda", generator=gen)).to(torch.bfloat16)
    s["workspace"] = torch.empty(WORKSPACE, dtype=torch.uint8, device="cuda")
    return s


# ---------------------------------------------------------------------------------------------- the plain forms

def _padded_tokens(s):
    """(token of [sequence, number], whether there is one, sequence of a token, its number there)."""
    cu, most = s["cu_q"].long(), s["max_q"]
    step = torch.arange(most, device="cuda")
    live = step < (cu[1:] - cu[:-1])[:, None]
    tokens = next(s[k].shape[0] for k in ("parents", "q", "path") if k in s)
    seq = torch.searchsorted(cu[1:], torch.arange(tokens, device="cuda"), right=True)
    return torch.where(live, cu[:-1, None] + step, 0), live, seq, torch.arange(tokens, device="cuda") - cu[seq]


def _above(s):
    """[sequence, number, number]: 1 where the second is the first or above it: with A the matrix of parents, where (I + A)^n is not 0."""
    at, live, seq, number = _padded_tokens(s)
    parent = torch.where(live, s["parents"].long()[at], -1)
    step = torch.arange(s["max_q"], device="cuda")
    A = ((parent[:, :, None] == step) & (parent >= 0)[:, :, None] & (parent < step)[:, :, None]).double()
    eye = torch.eye(s["max_q"], dtype=torch.float64, device="cuda").expand_as(A)
    return (torch.linalg.matrix_power(eye + A, 1 << (s["max_q"] - 1).bit_length()) > 0).double(), seq, number


def _tree_plain(s):
    above, seq, number = _above(s)
    rows = above[seq, number]  # [T, most]
    bits = torch.nn.functional.pad(rows, (0, 32 * s["words"] - s["max_q"])).view(-1, s["words"], 32).long()
    words = (bits << torch.arange(32, device="cuda")).sum(-1)
    words = torch.where(words >= 1 << 31, words - (1 << 32), words).int()
    n = s["cu_q"][1:] - s["cu_q"][:-1]
    return words, ((s["kv_lens"] - n)[seq] + rows.sum(1).int() - 1).int()


def _accept_plain(s):
    above, seq, number = _above(s)
    at, live, _, _ = _padded_tokens(s)
    step = torch.arange(s["max_q"], device="cuda")
    tokens, sampled = torch.where(live, s["tokens"][at], -1), torch.where(live, s["sampled"][at], -2)
    parent = torch.where(live, s["parents"].long()[at], -1)
    fits = (parent >= 0) & (tokens == sampled.gather(1, parent.clamp(min=0)))
    # a child that fits, unless a lower one of the same parent does
    rival = (parent[:, :, None] == parent[:, None, :]) & fits[:, None, :] & (step[None, None, :] < step[None, :, None])
    fits = (fits & ~rival.any(2)) | (step == 0)
    accepted = (torch.matmul(above, (~fits).double()[:, :, None])[..., 0] == 0) & live
    count = accepted.sum(1)
    path = torch.sort(torch.where(accepted, step, s["max_q"]), 1)[0]
    last = path.gather(1, (count - 1).clamp(min=0)[:, None])[:, 0]
    path = torch.where(step < count[:, None], path, -1)
    n = s["cu_q"][1:] - s["cu_q"][:-1]
    following = sampled.gather(1, last.clamp(max=s["max_q"] - 1)[:, None])[:, 0]
    return {"path": path[seq, number].int(), "counts": count.int(), "next": following.int(), "kv_lens": (s["kv_lens"] - n + count).int()}


def _values(codes, scales, at):
    """Tokens [B, heads, places, D] of the pages `at` [B, W], as the values that they stand for."""
    B, W = at.shape
    _, H, P, D = codes.shape
    x = torch.ldexp(codes[at].view(torch.float8_e4m3fn).float(), scales[at].int()[..., None, None] - 127)
    return x.transpose(1, 2).reshape(B, H, W * P, D)


def _attend_plain(s):
    c = s["case"]
    Hq, Hkv, D = c["Hq"], c["Hkv"], c["D"]
    lens, at, most = s["kv_lens"].long(), s["page_table"].long(), s["max_q"]
    B = at.shape[0]
    n = (s["cu_q"][1:] - s["cu_q"][:-1]).long()
    token, _, seq, number = _padded_tokens(s)
    q = s["q"].float()[token].view(B, most, Hkv, Hq // Hkv, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, -1, D)
    k, v = _values(s["k_codes"], s["k_scales"], at), _values(s["v_codes"], s["v_scales"], at)
    scores = torch.matmul(q, k.transpose(2, 3).contiguous()).view(B, Hkv, Hq // Hkv, most, -1) * D ** -0.5
    start = (lens - n)[:, None, None]
    j = torch.arange(k.shape[2], device="cuda")
    # the j-th place is the i-th new token, whose bit is in word i / 32
    i = (j - start).clamp(0, 32 * s["words"] - 1).expand(B, most, -1)
    words = s["tree"].long()[token]  # [B, most, words]
    seen = ((words.gather(2, i // 32) >> (i % 32)) & 1).bool() & (j >= start) & (j < lens[:, None, None]) & (j - start < 32 * s["words"])
    past = j < start
    if c["window"] > 0:
        past = past & (j > s["positions"].long()[token][..., None] - c["window"])
    seen = seen | past
    scores.masked_fill_(~seen[:, None, None], -math.inf)
    top = scores.amax(-1, keepdim=True)
    p = scores.sub_(torch.where(top == -math.inf, torch.zeros_like(top), top)).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(B, Hkv, -1, p.shape[-1]), v).view(B, Hkv, Hq // Hkv, most, D)
    o = torch.where(total > 0, o / total.clamp(min=1e-30), torch.zeros_like(o))
    return o.permute(0, 3, 1, 2, 4).reshape(B, most, Hq, D)[seq, number].to(torch.bfloat16)


def _sample_plain(s):
    # in 64 bits: a token is decided by which side of a border a sum of up to 262144 terms lies on
    x = s["logits"].double() + 0.0
    rows, V = x.shape
    at, order = torch.sort(x, dim=1, descending=True, stable=True)
    t = s["temperature"].double()[:, None]
    w = torch.exp((at - at[:, :1]) / torch.where(t > 0, t, torch.ones_like(t)))
    rank = torch.arange(V, device="cuda")
    kept = (rank == 0).expand(rows, V) | (t > 0)
    if s["top_k"] is not None:
        k = s["top_k"].long()[:, None]
        kept = kept & ((k <= 0) | (rank < k))
    if s["top_p"] is not None:
        p = s["top_p"].double()[:, None]
        mass = torch.where(kept, w, 0.0).cumsum(1)
        before = torch.nn.functional.pad(mass[:, :-1], (1, 0))
        kept = kept & ((p >= 1) | (before < p * mass[:, -1:]) | (rank == 0))
    if s["min_p"] is not None:
        kept = kept & ((w >= s["min_p"].double()[:, None]) | (rank == 0))
    mass = torch.empty_like(w).scatter_(1, order, torch.where(kept, w, 0.0)).cumsum(1)
    return (mass <= s["uniform"].double()[:, None] * mass[:, -1:]).sum(1).clamp(max=V - 1).int()


def _compact_plain(s):
    c = s["case"]
    P = c["P"]
    cu, lens, pages = s["cu_q"].long(), s["kv_lens"].long(), s["page_table"].long()
    n = cu[1:] - cu[:-1]
    start, count = lens - n, s["counts"].long()
    B, W = pages.shape
    # places of the pages that the new tokens are on: [sequence, page, place in the page]
    touched = (s["max_q"] + P - 2) // P + 1
    page = start[:, None] // P + torch.arange(touched, device="cuda")
    place = page[..., None] * P + torch.arange(P, device="cuda")
    i = place - start[:, None, None]
    there = (i >= 0) & (i < count[:, None, None])
    source = s["path"].long()[(cu[:-1, None, None] + i).clamp(0, s["path"].shape[0] - 1)]
    moved = there & (source != i)
    kept = (i < 0) | (there & ~moved)
    live = moved.any(-1)
    origin = torch.where(moved, start[:, None, None] + source, place.clamp(max=W * P - 1))
    origin_page = pages.gather(1, (origin // P).view(B, -1)).view_as(origin)[live]  # [touched page, place]
    to = pages.gather(1, page.clamp(max=W - 1))[live]
    spot, moved, kept = (origin % P)[live], moved[live], kept[live]
    far = moved & (origin_page != to[:, None])

    def store(codes, scales):
        here = scales[to].int() - 127
        came = scales[origin_page].int() - 127  # [touched page, place, head]
        x = codes[origin_page, :, spot].view(torch.float8_e4m3fn).float()  # [touched page, place, head, D]
        value = torch.ldexp(x, came[..., None])
        size = torch.where(far[:, :, None, None] & value.isfinite(), value.abs(), torch.zeros_like(value)).amax((1, 3))
        e = torch.maximum(here, _exponent(size))
        fresh = _codes(x, (e[:, None] - came)[..., None])
        both = torch.where((moved | kept)[:, :, None, None], fresh.view(torch.uint8), codes[to].transpose(1, 2))
        codes[to] = both.transpose(1, 2)
        scales[to] = (e + 127).to(torch.uint8)

    store(s["k_codes"], s["k_scales"])
    store(s["v_codes"], s["v_scales"])


def _cache_of(s):
    # the updated cache whole: codes as the E4M3 values that they are, scales as the bytes that hold their exponents
    return {"k_codes": s["k_codes"].view(torch.float8_e4m3fn), "k_scales": s["k_scales"],
            "v_codes": s["v_codes"].view(torch.float8_e4m3fn), "v_scales": s["v_scales"]}


def run(state):
    s, c = state, state["case"]
    kind = c["kind"]
    if own:
        import paper_2605_20315_amd as mq

        if kind == "tree":
            return mq.mq_draft_tree(s["parents"], s["cu_q"], s["kv_lens"], s["words"])
        if kind == "attend":
            return mq.kv8_tree_attention(s["q"], s["k_codes"], s["k_scales"], s["v_codes"], s["v_scales"], s["page_table"], s["cu_q"],
                                         s["kv_lens"], s["tree"], c["D"] ** -0.5, window=c["window"], positions=s["positions"], workspace=s["workspace"])
        if kind == "sample":
            return mq.mq_sample(s["logits"], s["uniform"], s["temperature"], s["top_k"], s["top_p"], s["min_p"])
        if kind == "accept":
            return dict(zip(("path", "counts", "next", "kv_lens"), mq.mq_draft_accept(s["parents"], s["tokens"], s["sampled"], s["cu_q"], s["kv_lens"])))
        mq.kv8_compact(s["k_codes"], s["k_scales"], s["v_codes"], s["v_scales"], s["page_table"], s["cu_q"], s["kv_lens"], s["path"], s["counts"])
        return _cache_of(s)
    if kind == "compact":
        _compact_plain(s)
        return _cache_of(s)
    return {"tree": _tree_plain, "attend": _attend_plain, "sample": _sample_plain, "accept": _accept_plain}[kind](s)


# ---------------------------------------------------------------------------------------------- in 64 bits

def _e4m3_value(byte):
    """Values of E4M3 codes from their bits."""
    byte = byte.long()
    sign, exponent, mantissa = byte >> 7, (byte >> 3) & 15, (byte & 7).double()
    size = torch.where(exponent == 0, mantissa * 2.0 ** -9, (1 + mantissa / 8) * torch.exp2((exponent - 7).double()))
    return torch.where(sign == 1, -size, size)


def _e4m3_round(x):
    """The nearest E4M3 value, ties to even, clipped."""
    size = x.abs().clamp(max=E4M3_MAX)
    step = torch.exp2((torch.frexp(size)[1] - 4).clamp(min=-9).double())
    return torch.copysign(torch.round(size / step) * step, x)


def _walk(parents):
    """The tokens above each of one sequence's, itself first."""
    out = []
    for i, p in enumerate(parents):
        out.append([i] + (out[p] if 0 <= p < i else []))
    return out


def _each(case, s):
    """(sequence, first token, new tokens, earlier ones)."""
    first = 0
    for b, (n, start) in enumerate(zip(*_lengths(case))):
        yield b, first, n, start
        first += n


def _exact_tree(case, s):
    words, positions = [], []
    for b, first, n, start in _each(case, s):
        for above in _walk(s["parents"][first : first + n].tolist()):
            number = sum(1 << j for j in above)
            row = [(number >> (32 * w)) & 0xFFFFFFFF for w in range(s["words"])]
            words.append([r - (1 << 32) if r >> 31 else r for r in row])
            positions.append(start + len(above) - 1)
    return _ints(words), _ints(positions)


def _exact_accept(case, s):
    path, counts, following, lens = [], [], [], []
    for b, first, n, start in _each(case, s):
        parents, tokens, sampled = (s[k][first : first + n].tolist() for k in ("parents", "tokens", "sampled"))
        way = [0]
        while True:
            child = [i for i in range(way[-1] + 1, n) if parents[i] == way[-1] and tokens[i] == sampled[way[-1]]]
            if not child:
                break
            way.append(child[0])
        path += way + [-1] * (n - len(way))
        counts.append(len(way))
        following.append(sampled[way[-1]])
        lens.append(start + len(way))
    return {"path": _ints(path), "counts": _ints(counts), "next": _ints(following), "kv_lens": _ints(lens)}


def _exact_attend(case, s):
    Hq, Hkv, D, P = case["Hq"], case["Hkv"], case["D"], case["P"]
    out = []
    for b, first, n, start in _each(case, s):
        total = start + n
        at = s["page_table"][b, : -(-total // P)].long()
        walks = _walk(_parents(_lengths(case)[0], s["seed"])[first : first + n])
        hidden = torch.ones(n, total, dtype=torch.bool, device="cuda")
        depth = torch.tensor([len(w) - 1 for w in walks], device="cuda")[:, None]
        j = torch.arange(start, device="cuda")[None]
        hidden[:, :start] = (j <= start + depth - case["window"]) if case["window"] > 0 else False
        hidden[[i for i, w in enumerate(walks) for _ in w], [start + a for w in walks for a in w]] = False
        heads = []
        for h in range(Hkv):
            k, v = (((_e4m3_value(s[x + "_codes"][at, h]) * torch.exp2(s[x + "_scales"][at, h].double() - 127)[:, None, None]).reshape(-1, D)[:total]) for x in "kv")
            for g in range(h * (Hq // Hkv), (h + 1) * (Hq // Hkv)):
                a = (s["q"][first : first + n, g].double() @ k.t()) / math.sqrt(D)
                heads.append(torch.softmax(a.masked_fill_(hidden, -math.inf), 1) @ v)
        out.append(torch.stack(heads, 1))
    return torch.cat(out)


def _exact_sample(case, s):
    tokens = []
    for r in range(case["rows"]):
        x = s["logits"][r].double()
        best = int((x == x.max()).nonzero()[0])
        t = float(s["temperature"][r])
        if not t > 0:
            tokens.append(best)
            continue
        p = torch.softmax(x / t, 0)
        ranks = torch.argsort(-x, stable=True)
        if s["top_k"] is not None and int(s["top_k"][r]) > 0:
            ranks = ranks[: int(s["top_k"][r])]
        if s["top_p"] is not None and float(s["top_p"][r]) < 1:
            share = p[ranks] / p[ranks].sum()
            ranks = ranks[(share.cumsum(0) - share < float(s["top_p"][r])).cumprod(0).bool()]
        if s["min_p"] is not None:
            ranks = torch.cat([ranks[:1], ranks[1:][p[ranks[1:]] >= float(s["min_p"][r]) * p[best]]])
        chosen = ranks.sort()[0]
        mass = p[chosen].cumsum(0)
        tokens.append(int(chosen[min(int(torch.searchsorted(mass, float(s["uniform"][r]) * mass[-1], right=True)), len(chosen) - 1)]))
    return _ints(tokens)


def _exact_compact(case, s):
    P = case["P"]
    out = {}
    for x in "kv":
        values, exps = _e4m3_value(s[x + "_codes"]), s[x + "_scales"].long() - 127
        new_values, new_exps = values.clone(), exps.clone()
        for b, first, n, start in _each(case, s):
            count = int(s["counts"][b])
            path = s["path"][first : first + count].tolist()
            table = s["page_table"][b].tolist()
            spot = lambda place: (table[place // P], place % P)  # noqa: E731
            for number in range(start // P, (start + count - 1) // P + 1):
                to, base = table[number], number * P
                places = [start + i for i in range(count) if path[i] != i and (start + i) // P == number]
                if not places:
                    continue
                came = {j: spot(start + path[j - start]) for j in places}
                e = exps[to]
                for j, (page, at) in came.items():
                    if page != to:
                        size = values[page, :, at].abs().amax(1) * torch.exp2(exps[page].double())
                        e = torch.maximum(e, torch.where(size > 0, torch.ceil(torch.log2(size / E4M3_MAX)), LOWEST).clamp(LOWEST, HIGHEST).long())
                stay = [j - base for j in range(base, places[0])]
                new_values[to, :, stay] = _e4m3_round(values[to][:, stay] * torch.exp2((exps[to] - e).double())[:, None, None])
                for j, (page, at) in came.items():
                    new_values[to, :, j - base] = _e4m3_round(values[page, :, at] * torch.exp2((exps[page] - e).double())[:, None])
                new_exps[to] = e
        out[x + "_codes"], out[x + "_scales"] = new_values, (new_exps + 127).to(torch.uint8)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    s["seed"] = seed
    return {"tree": _exact_tree, "attend": _exact_attend, "sample": _exact_sample, "accept": _exact_accept, "compact": _exact_compact}[case["kind"]](case, s)
