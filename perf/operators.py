"""The attention half of a decoder block between its linear layers, and those layers for a few tokens, as measurable cases.

Three operators, in the order in which a serving program runs them in every block:

  append   kv8_append: the position rotation of the queries and keys of new tokens, and their keys and values appended to a
           paged cache of FP8 E4M3 codes with one power-of-two scale for each page and head
  attend   kv8_attention: attention of the new tokens' queries over that cache, causal, with an optional window
  matvec   nvfp4_matvec: BF16 activations of a few tokens times NVFP4 weights (the output and MLP projections of a decode step)

The plain forms below compute the same from the formulas with elementary torch operations in 32 bits.

Formulas.  Rotation by the table's cosines c and sines s at a token's position, for the pairs (a, b) of a head's first R elements
(elements i and R/2 + i, or 2i and 2i + 1 where interleaved): a' = a c - b s, b' = b c + a s, each step in 32 bits and the result
rounded once to BF16.  A page's scale is 2^e with the smallest e of -112 .. 119 that brings its largest finite magnitude to 448
or below, and at least the scale that the page had where it holds earlier tokens; those tokens' codes are brought to the new
scale with one rounding.  A code is the nearest E4M3 value of x / 2^e (ties to even, clipped to +-448).  Scales are kept as the
byte e + 127.  Attention: softmax over the visible j of scale * q.k_j, times v_j; a query at position p sees 0 <= j <= p and, with
a window w > 0, p - w < j; one that sees nothing gives zeros.  The cache's last q_len tokens are the queries' own.
"""
import math
import random

import torch

own = False

# a program keeps one workspace per stream: the largest that the library asks for
WORKSPACE = 64 << 20
E4M3_MAX = 448.0
LOWEST, HIGHEST = -112, 119


def _append(seqs, q, past, Hq=32, Hkv=8, D=128, P=64, rot=128, interleaved=False, lengths=1):
    return {"kind": "append", "seqs": seqs, "q_lo": q[0], "q_hi": q[1], "past_lo": past[0], "past_hi": past[1], "Hq": Hq, "Hkv": Hkv,
            "D": D, "P": P, "rot": rot, "interleaved": interleaved, "lengths": lengths}


def _attend(seqs, q, past, Hq=32, Hkv=8, D=128, P=64, window=0, lengths=1):
    return {"kind": "attend", "seqs": seqs, "q_lo": q[0], "q_hi": q[1], "past_lo": past[0], "past_hi": past[1], "Hq": Hq, "Hkv": Hkv,
            "D": D, "P": P, "window": window, "lengths": lengths}


def _matvec(M, K, N, layout="ktile", out="bf16"):
    return {"kind": "matvec", "M": M, "K": K, "N": N, "layout": layout, "out": out}


def listed():
    return [
        # one request generating: its token's keys and values go into the cache (all latency)
        dict(_append(1, (1, 1), (1000, 1000)), name="append_one"),
        # a decode batch of 200 requests, one token each, somewhere inside a page
        dict(_append(200, (1, 1), (16, 1000)), name="append_batch"),
        # a long prompt at once, into empty pages (the last one in part)
        dict(_append(1, (8111, 8111), (0, 0)), name="append_prompt"),
        # prompts and generated tokens together, a quarter of each head rotated in interleaved pairs, small pages
        dict(_append(24, (1, 700), (0, 900), Hq=28, Hkv=4, D=64, P=16, rot=16, interleaved=True), name="append_mixed"),
        # one request generating, a short history
        dict(_attend(1, (1, 1), (1000, 1000)), name="attend_one"),
        # a decode batch of uneven histories
        dict(_attend(64, (1, 1), (100, 8000)), name="attend_batch"),
        # two requests deep in a long context, three tokens each (drafted ones among them), pages of 16
        dict(_attend(2, (3, 3), (100000, 131000), P=16), name="attend_long"),
        # a long prompt over itself
        dict(_attend(1, (8192, 8192), (0, 0)), name="attend_prompt"),
        # three prompts' next chunks over a sliding window, smaller heads
        dict(_attend(3, (300, 700), (8000, 24000), Hq=16, Hkv=4, D=64, P=32, window=4096), name="attend_chunks"),
        # one token through the query, key and value projection
        dict(_matvec(1, 4096, 6144), name="matvec_one"),
        # a decode batch of nine through the gate and up projection, canonical byte order
        dict(_matvec(9, 4096, 28672, layout="linear"), name="matvec_batch"),
        # a decode batch of forty through a wide down projection, 32-bit sums out
        dict(_matvec(40, 25600, 5120, out="fp32"), name="matvec_wide"),
    ]


def _span(rng, lo, hi):
    """A size from lo to hi, spread over the logarithm where the range is wide."""
    return rng.randint(lo, hi) if hi < 10 * max(lo, 1) else min(hi, max(lo, int(math.exp(rng.uniform(math.log(max(lo, 1)), math.log(hi + 1))))))


def _draw_heads(rng):
    Hkv, group = rng.choice([1, 2, 4, 5, 8]), rng.choice([1, 2, 3, 4, 7, 8, 12])
    return {"Hkv": Hkv, "Hq": Hkv * group, "D": rng.choice([64, 128, 256]), "P": rng.choice([16, 32, 64, 128])}


def draw(rng):
    top = {k: max(_cost(c) for c in listed() if c["kind"] == k) for k in ("append", "attend", "matvec")}
    kind = rng.choice(["append", "attend", "attend", "matvec"])
    while True:
        if kind == "matvec":
            c = _matvec(_span(rng, 1, 64), 64 * _span(rng, 16, 448), _span(rng, 500, 28672), rng.choice(["ktile", "linear"]), rng.choice(["bf16", "fp32"]))
        else:
            seqs, h = _span(rng, 1, 200), _draw_heads(rng)
            one = rng.random() < 0.5
            q_hi = rng.randint(1, 4) if one else _span(rng, 2, 8192 // seqs + 2)
            past_hi = _span(rng, 1, 131072 if kind == "attend" else 4096)
            q, past = (rng.randint(1, q_hi) if not one else q_hi, q_hi), (rng.randint(0, past_hi), past_hi)
            if kind == "append":
                rot = rng.choice([h["D"], h["D"] // 2, h["D"] // 4])
                c = _append(seqs, q, past, rot=rot, interleaved=rng.random() < 0.5, lengths=rng.randrange(1000), **h)
            else:
                c = _attend(seqs, q, past, window=rng.choice([0, 0, _span(rng, 16, 16384)]), lengths=rng.randrange(1000), **h)
        if _cost(c) <= top[kind] and _padded(c) <= 1 << 31:
            return c


def _lengths(case):
    """New and earlier tokens of each sequence: the same ones for every seed."""
    r = random.Random(case["lengths"])
    q = [r.randint(case["q_lo"], case["q_hi"]) for _ in range(case["seqs"])]
    return q, [r.randint(case["past_lo"], case["past_hi"]) for _ in range(case["seqs"])]


def _padded(case):
    """Values of the plain form's largest tensor."""
    if case["kind"] == "matvec":
        return case["N"] * case["K"]
    q, past = _lengths(case)
    longest = max(a + b for a, b in zip(q, past)) + case["P"]
    cache = case["seqs"] * longest * case["Hkv"] * case["D"]
    return max(cache, case["seqs"] * max(q) * longest * case["Hq"]) if case["kind"] == "attend" else cache


def _visible(q, past, window):
    """(query, key) pairs of one sequence that the mask leaves, and keys that any query sees."""
    first, total = past, past + q
    if window <= 0:
        return q * past + q * (q + 1) // 2, total
    pairs = sum(min(p + 1, window) for p in range(first, total))
    return pairs, total - max(0, first - window + 1)


def work(case):
    if case["kind"] == "matvec":
        M, K, N = case["M"], case["K"], case["N"]
        return {"bytes": N * K * 9 / 16 + 2 * M * K + (2 if case["out"] == "bf16" else 4) * M * N, "flops": 2 * M * N * K}
    q, past = _lengths(case)
    T, Hq, Hkv, D = sum(q), case["Hq"], case["Hkv"], case["D"]
    if case["kind"] == "append":
        # BF16 queries in and out, keys and values in, codes out; the table's rows
        return {"bytes": T * (4 * Hq * D + 6 * Hkv * D + 4 * case["rot"]), "flops": 3 * T * (Hq + Hkv) * case["rot"] + 2 * T * Hkv * D}
    pairs = [_visible(a, b, case["window"]) for a, b in zip(q, past)]
    return {"bytes": 4 * T * Hq * D + 2 * Hkv * D * sum(n for _, n in pairs), "flops": 4 * D * Hq * sum(p for p, _ in pairs)}


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
    """A cache that holds earlier tokens: normal values, a few large channels, magnitudes that differ from head to head and page to page."""
    x = torch.randn(pages, Hkv, P, D, device="cuda", generator=gen)
    x *= torch.exp(0.5 * torch.randn(1, Hkv, 1, 1, device="cuda", generator=gen) + 0.2 * torch.randn(pages, 1, 1, 1, device="cuda", generator=gen))
    x[..., torch.randint(0, D, (2,), device="cuda", generator=gen)] *= 3.0
    e = _exponent(x.abs().amax((2, 3)))
    return _codes(x, e[:, :, None, None]).view(torch.uint8), (e + 127).to(torch.uint8)


def _angles(max_pos, rot):
    """cos and sin of position * 500000^(-2i/R), angles in 64 bits: the table that a program keeps."""
    f = 500000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot)
    a = torch.arange(max_pos, dtype=torch.float64, device="cuda")[:, None] * f
    return torch.cat([a.cos(), a.sin()], 1).float()


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *shape: torch.randn(*shape, device="cuda", generator=gen)  # noqa: E731
    if case["kind"] == "matvec":
        M, K, N = case["M"], case["K"], case["N"]
        x = normal(M, K)
        x[:, torch.randint(0, K, (max(1, K // 1000),), device="cuda", generator=gen)] *= 20.0  # outlier channels
        codes, scales, alpha = _weights(normal(N, K) * K ** -0.5)
        if case["layout"] == "ktile":
            codes = codes.view(N, K // 64, 32).transpose(0, 1).contiguous().view(N, K // 2)
            scales = scales.view(N, K // 64, 4).transpose(0, 1).contiguous().view(N, K // 16)
        return {"case": case, "x": x.to(torch.bfloat16), "codes": codes, "scales": scales, "alpha": alpha}
    q_lens, past = _lengths(case)
    seqs, Hq, Hkv, D, P = case["seqs"], case["Hq"], case["Hkv"], case["D"], case["P"]
    T = sum(q_lens)
    total = [a + b for a, b in zip(q_lens, past)]
    held = [-(-n // P) for n in total]
    pages = sum(held) + 3
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    order = torch.randperm(pages, device="cuda", generator=gen).to(torch.int32)
    table = torch.zeros(seqs, max(held), dtype=torch.int32, device="cuda")
    width = torch.arange(max(held), device="cuda")
    table[width[None] < ints(held)[:, None]] = order[: sum(held)]
    s = {"case": case, "page_table": table, "cu_q": ints([0] + [sum(q_lens[: i + 1]) for i in range(seqs)]), "kv_lens": ints(total), "max_q": max(q_lens)}
    s["k_codes"], s["k_scales"] = _pool(gen, pages, Hkv, P, D)
    s["v_codes"], s["v_scales"] = _pool(gen, pages, Hkv, P, D)
    if case["kind"] == "attend":
        s["q"] = (1.5 * normal(T, Hq, D)).to(torch.bfloat16)
        s["workspace"] = torch.empty(WORKSPACE, dtype=torch.uint8, device="cuda")
        return s
    # what the projection hands over: queries, keys and values of a token side by side
    qkv = normal(T, Hq + 2 * Hkv, D)
    qkv *= torch.exp(0.5 * normal(1, Hq + 2 * Hkv, 1))
    qkv = qkv.to(torch.bfloat16)
    s["q"], s["k"], s["v"] = qkv[:, :Hq], qkv[:, Hq : Hq + Hkv], qkv[:, Hq + Hkv :]
    s["table"] = _angles(max(total), case["rot"])
    return s


def _weights(w):
    """NVFP4 codes, block scales and tensor scale of a weight matrix."""
    N, K = w.shape
    alpha = w.abs().amax().reshape(1) / 2688.0
    scales = (w.view(N, K // 16, 16).abs().amax(2) / (6.0 * alpha)).clamp(max=E4M3_MAX).to(torch.float8_e4m3fn)
    y = w.view(N, K // 16, 16) / (alpha * scales.float()).clamp(min=1e-30)[:, :, None]
    steps = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device=w.device)
    c = (torch.bucketize(y.abs(), steps) + 8 * (y < 0)).to(torch.uint8).view(N, K // 2, 2)
    return (c[..., 0] | (c[..., 1] << 4)).contiguous(), scales.view(torch.uint8), alpha


# ---------------------------------------------------------------------------------------------- the plain forms

def _rotate(x, cs, interleaved):
    """x [T, H, D] turned by the table rows cs [T, R]."""
    R = cs.shape[1]
    c, s = cs[:, None, : R // 2], cs[:, None, R // 2 :]
    x = x.float()
    a, b = (x[..., 0:R:2], x[..., 1:R:2]) if interleaved else (x[..., : R // 2], x[..., R // 2 : R])
    a2, b2 = a * c - b * s, b * c + a * s
    turned = torch.stack([a2, b2], -1).flatten(-2) if interleaved else torch.cat([a2, b2], -1)
    return torch.cat([turned, x[..., R:]], -1).to(torch.bfloat16)


def _append_plain(s):
    c = s["case"]
    P = c["P"]
    cu, lens, pages = s["cu_q"].long(), s["kv_lens"].long(), s["page_table"].long()
    n = cu[1:] - cu[:-1]
    start = lens - n
    T, B = s["q"].shape[0], n.shape[0]
    seq = torch.searchsorted(cu[1:], torch.arange(T, device="cuda"), right=True)
    cs = s["table"][start[seq] + torch.arange(T, device="cuda") - cu[seq]]
    # slots of the pages that the new tokens touch: [sequence, page, place in the page]
    touched = (s["max_q"] + P - 2) // P + 1
    page = start[:, None] // P + torch.arange(touched, device="cuda")
    slot = page[..., None] * P + torch.arange(P, device="cuda")
    new = (slot >= start[:, None, None]) & (slot < lens[:, None, None])
    old = (slot < start[:, None, None]) & new.any(-1, keepdim=True)
    token = (cu[:-1, None, None] + slot - start[:, None, None]).clamp(0, T - 1)
    live = new.any(-1)
    at = pages.gather(1, page.clamp(max=pages.shape[1] - 1))[live]

    def store(x, codes, scales):
        x = x.float()[token[live]].transpose(1, 2)  # [touched page, head, place, D]
        is_new, is_old = new[live][:, None, :, None], old[live][:, None, :, None]
        size = torch.where(is_new & x.isfinite(), x.abs(), torch.zeros_like(x)).amax((2, 3))
        before = scales[at].int() - 127
        e = torch.where(is_old.any(2)[..., 0], torch.maximum(_exponent(size), before), _exponent(size))
        kept = _codes(codes[at].view(torch.float8_e4m3fn).float(), (e - before)[:, :, None, None])
        fresh = _codes(x, e[:, :, None, None])
        both = torch.where(is_new, fresh.view(torch.uint8), torch.where(is_old, kept.view(torch.uint8), codes[at]))
        codes[at] = both
        scales[at] = (e + 127).to(torch.uint8)

    q = _rotate(s["q"], cs, c["interleaved"])
    store(_rotate(s["k"], cs, c["interleaved"]), s["k_codes"], s["k_scales"])
    store(s["v"], s["v_codes"], s["v_scales"])
    return q


def _values(codes, scales, at):
    """Tokens [B, heads, places, D] of the pages `at` [B, W], as the values that they stand for."""
    B, W = at.shape
    _, H, P, D = codes.shape
    x = torch.ldexp(codes[at].view(torch.float8_e4m3fn).float(), scales[at].int()[..., None, None] - 127)
    return x.transpose(1, 2).reshape(B, H, W * P, D)


def _attend_plain(s):
    c = s["case"]
    Hq, Hkv, D = c["Hq"], c["Hkv"], c["D"]
    cu, lens, at = s["cu_q"].long(), s["kv_lens"].long(), s["page_table"].long()
    B, T, most = at.shape[0], s["q"].shape[0], s["max_q"]
    n = cu[1:] - cu[:-1]
    step = torch.arange(most, device="cuda")
    token = (cu[:-1, None] + step).clamp(max=T - 1)
    q = s["q"].float()[token].view(B, most, Hkv, Hq // Hkv, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, -1, D)
    k, v = _values(s["k_codes"], s["k_scales"], at), _values(s["v_codes"], s["v_scales"], at)
    scores = torch.matmul(q, k.transpose(2, 3)).view(B, Hkv, Hq // Hkv, most, -1) * D ** -0.5
    pos = (lens - n)[:, None] + step
    j = torch.arange(k.shape[2], device="cuda")
    seen = (j <= pos[..., None]) & (j < lens[:, None, None])
    if c["window"] > 0:
        seen &= j > pos[..., None] - c["window"]
    scores.masked_fill_(~seen[:, None, None], -math.inf)
    top = scores.amax(-1, keepdim=True)
    p = scores.sub_(torch.where(top == -math.inf, torch.zeros_like(top), top)).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(B, Hkv, -1, p.shape[-1]), v).view(B, Hkv, Hq // Hkv, most, D)
    o = torch.where(total > 0, o / total.clamp(min=1e-30), torch.zeros_like(o))
    o = o.permute(0, 3, 1, 2, 4).reshape(B, most, Hq, D)
    row = torch.searchsorted(cu[1:], torch.arange(T, device="cuda"), right=True)
    return o[row, torch.arange(T, device="cuda") - cu[row]].to(torch.bfloat16)


def _matvec_plain(s):
    c = s["case"]
    N, K = c["N"], c["K"]
    codes, scales = s["codes"], s["scales"]
    if c["layout"] == "ktile":
        codes = codes.view(K // 64, N, 32).transpose(0, 1).reshape(N, K // 2)
        scales = scales.view(K // 64, N, 4).transpose(0, 1).reshape(N, K // 16)
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], device="cuda")
    q = torch.stack([grid[(codes & 15).int()], grid[(codes >> 4).int()]], -1).view(N, K // 16, 16)
    w = (q * scales.view(torch.float8_e4m3fn).float()[..., None]).view(N, K)
    y = torch.matmul(s["x"].float(), w.t()) * s["alpha"]
    return y.to(torch.bfloat16) if c["out"] == "bf16" else y


def _state_of(s, q):
    # the updated cache whole: codes as the E4M3 values that they are, scales as the bytes that hold their exponents
    return {"q": q, "k_codes": s["k_codes"].view(torch.float8_e4m3fn), "k_scales": s["k_scales"],
            "v_codes": s["v_codes"].view(torch.float8_e4m3fn), "v_scales": s["v_scales"]}


def run(state):
    s, c = state, state["case"]
    if own:
        import paper_2605_20315_amd as mq

        if c["kind"] == "append":
            return _state_of(s, mq.kv8_append(s["q"], s["k"], s["v"], s["k_codes"], s["k_scales"], s["v_codes"], s["v_scales"],
                                              s["page_table"], s["cu_q"], s["kv_lens"], s["table"], interleaved=c["interleaved"]))
        if c["kind"] == "attend":
            return mq.kv8_attention(s["q"], s["k_codes"], s["k_scales"], s["v_codes"], s["v_scales"], s["page_table"], s["cu_q"],
                                    s["kv_lens"], c["D"] ** -0.5, window=c["window"], workspace=s["workspace"])
        return mq.nvfp4_matvec(s["x"], s["codes"], s["scales"], s["alpha"], mq.MQ_OUT_BF16 if c["out"] == "bf16" else mq.MQ_OUT_FP32,
                               layout=mq.MQ_LAYOUT_KTILE if c["layout"] == "ktile" else mq.MQ_LAYOUT_LINEAR)
    if c["kind"] == "append":
        return _state_of(s, _append_plain(s))
    return _attend_plain(s) if c["kind"] == "attend" else _matvec_plain(s)


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


def _exact_append(case, s):
    P, R, Hkv = case["P"], case["rot"], case["Hkv"]
    q_lens, past = _lengths(case)
    f = 500000.0 ** (-torch.arange(0, R, 2, dtype=torch.float64, device="cuda") / R)
    k_out, v_out = _e4m3_value(s["k_codes"]), _e4m3_value(s["v_codes"])
    k_e, v_e = s["k_scales"].long() - 127, s["v_scales"].long() - 127
    q_out, first = [], 0
    for b, (n, start) in enumerate(zip(q_lens, past)):
        angle = (start + torch.arange(n, dtype=torch.float64, device="cuda"))[:, None] * f
        turn = torch.polar(torch.ones_like(angle), angle)[:, None]

        def rotated(x):
            x = x.double().clone()
            if case["interleaved"]:
                z = torch.complex(x[..., 0:R:2], x[..., 1:R:2]) * turn
                x[..., 0:R:2], x[..., 1:R:2] = z.real, z.imag
            else:
                z = torch.complex(x[..., : R // 2], x[..., R // 2 : R]) * turn
                x[..., : R // 2], x[..., R // 2 : R] = z.real, z.imag
            return x

        q_out.append(rotated(s["q"][first : first + n]))
        k = rotated(s["k"][first : first + n]).to(torch.bfloat16).double()  # the cache takes the BF16 keys
        v = s["v"][first : first + n].double()
        done = 0
        while done < n:
            place = (start + done) % P
            count = min(P - place, n - done)
            page = int(s["page_table"][b, (start + done) // P])
            for new, codes, exps in ((k, k_out, k_e), (v, v_out, v_e)):
                part = new[done : done + count].transpose(0, 1)
                size = part.abs().amax((1, 2))
                e = torch.ceil(torch.log2(size / E4M3_MAX)).clamp(LOWEST, HIGHEST).long()
                if place:
                    e = torch.maximum(e, exps[page])
                    codes[page, :, :place] = _e4m3_round(codes[page, :, :place] * torch.exp2((exps[page] - e).double())[:, None, None])
                codes[page, :, place : place + count] = _e4m3_round(part * torch.exp2(-e.double())[:, None, None])
                exps[page] = e
            done += count
        first += n
    return {"q": torch.cat(q_out), "k_codes": k_out, "k_scales": (k_e + 127).to(torch.uint8), "v_codes": v_out, "v_scales": (v_e + 127).to(torch.uint8)}


def _exact_attend(case, s):
    q_lens, past = _lengths(case)
    Hq, Hkv, D, P = case["Hq"], case["Hkv"], case["D"], case["P"]
    out, first = [], 0
    for b, (n, start) in enumerate(zip(q_lens, past)):
        total = start + n
        at = s["page_table"][b, : -(-total // P)].long()
        p = start + torch.arange(n, device="cuda")[:, None]
        j = torch.arange(total, device="cuda")[None]
        hidden = (j > p) | (j <= p - case["window"]) if case["window"] > 0 else j > p
        heads = []
        for h in range(Hkv):
            k, v = (((_e4m3_value(s[x + "_codes"][at, h]) * torch.exp2(s[x + "_scales"][at, h].double() - 127)[:, None, None]).reshape(-1, D)[:total]) for x in "kv")
            for g in range(h * (Hq // Hkv), (h + 1) * (Hq // Hkv)):
                a = (s["q"][first : first + n, g].double() @ k.t()) / math.sqrt(D)
                heads.append(torch.softmax(a.masked_fill_(hidden, -math.inf), 1) @ v)
        out.append(torch.stack(heads, 1))
        first += n
    return torch.cat(out)


def _exact_matvec(case, s):
    N, K = case["N"], case["K"]
    codes, scales = s["codes"].long().reshape(-1), s["scales"].reshape(-1)
    n, k = torch.arange(N, device="cuda")[:, None], torch.arange(K, device="cuda")[None]
    if case["layout"] == "ktile":
        byte, block = ((k // 64) * N + n) * 32 + (k % 64) // 2, ((k // 64) * N + n) * 4 + (k % 64) // 16
    else:
        byte, block = n * (K // 2) + k // 2, n * (K // 16) + k // 16
    code = (codes[byte] >> (4 * (k % 2))) & 15
    exponent, mantissa = (code >> 1) & 3, (code & 1).double()
    size = torch.where(exponent == 0, mantissa / 2, (1 + mantissa / 2) * torch.exp2((exponent - 1).double()))
    w = torch.where(code >= 8, -size, size) * _e4m3_value(scales)[block]
    return (s["x"].double() @ w.t()) * s["alpha"].double()


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "append":
        return _exact_append(case, s)
    if case["kind"] == "attend":
        return _exact_attend(case, s)
    return _exact_matvec(case, s)
