"""Plain definitions, in NumPy and 64 bits, of decoding with drafted tokens: trees, attention over them, sampling, acceptance, compaction."""
import numpy as np

import _kv8_ref as ref


def above(parents):
    """For each of one sequence's tokens the numbers from itself up to its root."""
    out = []
    for i, p in enumerate(parents):
        out.append([i] + (out[p] if 0 <= p < i else []))
    return out


def tree(parents, cu_q, kv_lens, words, window=0):
    masks, positions = np.zeros((len(parents), words), np.uint32), np.zeros(len(parents), np.int32)
    for b in range(len(kv_lens)):
        n, start = cu_q[b + 1] - cu_q[b], kv_lens[b] - (cu_q[b + 1] - cu_q[b])
        for i, way in enumerate(above(parents[cu_q[b] : cu_q[b + 1]])):
            t = cu_q[b] + i
            positions[t] = start + (len(way) - 1 if i < 32 * words else i)
            if i < 32 * words:
                for j in way[: window if window > 0 else None]:
                    masks[t, j // 32] |= np.uint32(1 << (j % 32))
    return masks.view(np.int32), positions


def random_parents(r, n, spread=9, roots=0.0):
    return [-1 if i == 0 or r.random() < roots else int(r.integers(max(0, i - spread), i)) for i in range(n)]


def tree_attention(q, kc, ks, vc, vs, page_table, cu_q, kv_lens, masks, scale, window=0, positions=None):
    """(y, a, s) as _kv8_ref.attention gives them."""
    pages, Hkv, P, D = kc.shape
    T, Hq, _ = q.shape
    G, masks = Hq // Hkv, masks.view(np.uint32)
    y, a, s = np.zeros(q.shape), np.zeros(q.shape), np.zeros((T, Hq, 1))
    for b in range(len(kv_lens)):
        n = cu_q[b + 1] - cu_q[b]
        start = int(kv_lens[b]) - int(n)
        j = np.array([j for j in range(min(kv_lens[b], page_table.shape[1] * P)) if 0 <= page_table[b, j // P] < pages], dtype=np.int64)
        at = page_table[b, j // P] if len(j) else j
        sees = np.zeros((n, len(j)), bool)
        for i in range(n):
            t = cu_q[b] + i
            pos = start + i if positions is None else max(int(positions[t]), start)
            number = j - start
            inside = (number >= 0) & (number < 32 * masks.shape[1])
            word = masks[t, np.clip(number, 0, 32 * masks.shape[1] - 1) // 32].astype(np.int64)
            sees[i] = np.where(number < 0, (j > pos - window) if window > 0 else True, inside & ((word >> (np.maximum(number, 0) % 32)) & 1 == 1))
        for h in range(Hkv):
            k = ref.E4M3[kc[at, h, j % P]] * 2.0 ** (ks[at, h].astype(np.float64) - 127)[:, None]
            v = ref.E4M3[vc[at, h, j % P]] * 2.0 ** (vs[at, h].astype(np.float64) - 127)[:, None]
            for i in range(n):
                t, see = cu_q[b] + i, sees[i]
                if not see.any():
                    continue
                heads = slice(h * G, (h + 1) * G)
                x = q[t, heads].astype(np.float64) @ k[see].T * scale
                p = np.exp(x - x.max(1, keepdims=True))
                p /= p.sum(1, keepdims=True)
                p = np.where(p < 1e-300, 1e-300, p)  # a NaN that is seen is not hidden by a probability that underflows
                y[t, heads], a[t, heads] = p @ v[see], p @ np.abs(v[see])
                s[t, heads, 0] = (np.abs(q[t, heads]).astype(np.float64) @ np.abs(k[see]).T).max(1) * scale
    return y, a, s


def sample(logits, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """The token of one row of binary32 logits, every step in binary64."""
    x = np.where(np.isnan(logits), -np.inf, logits).astype(np.float64) + 0.0
    order = np.argsort(-x, kind="stable")
    top = x[order[0]]
    if top == -np.inf:
        return -1
    if not temperature > 0 or not top_p > 0 or min_p != min_p:
        return int(order[0])
    with np.errstate(invalid="ignore", over="ignore"):
        w = np.where(x == top, 1.0, np.where((x == -np.inf) | (top == np.inf), 0.0, np.exp((x - top) / np.float64(temperature))))
    kept = order[:top_k] if top_k > 0 else order
    if top_p < 1:
        mass = np.cumsum(w[kept])
        kept = kept[np.concatenate([[0.0], mass[:-1]]) < top_p * mass[-1]]
    if min_p > 0:
        kept = np.concatenate([kept[:1], kept[1:][w[kept[1:]] >= min_p]])
    kept = np.sort(kept)
    mass = np.cumsum(w[kept])
    u = 0.0 if u != u else min(max(float(u), 0.0), 1.0 - 2.0 ** -40)
    return int(kept[np.searchsorted(mass, u * mass[-1], side="right")])


def accept(parents, tokens, sampled, cu_q, kv_lens):
    path, counts, following, lens = np.full(len(parents), -1, np.int32), [], [], []
    for b in range(len(kv_lens)):
        first, n = cu_q[b], cu_q[b + 1] - cu_q[b]
        way = [0] if n else []
        while way:
            child = [i for i in range(way[-1] + 1, n) if parents[first + i] == way[-1] and tokens[first + i] == sampled[first + way[-1]]]
            if not child:
                break
            way.append(child[0])
        path[first : first + len(way)] = way
        counts.append(len(way))
        following.append(sampled[first + way[-1]] if n else -1)
        lens.append(max(kv_lens[b] - n + len(way), 0))
    return path, np.array(counts, np.int32), np.array(following, np.int32), np.array(lens, np.int32)


def compact(kc, ks, vc, vs, page_table, cu_q, kv_lens, path, counts):
    """The cache is changed in place."""
    pages, Hkv, P, D = kc.shape
    page_of = lambda b, j: page_table[b, j // P] if 0 <= j < page_table.shape[1] * P and 0 <= page_table[b, j // P] < pages else -1  # noqa: E731
    for codes, scales in ((kc, ks), (vc, vs)):
        before, scales_before = codes.copy(), scales.copy()
        for b in range(len(kv_lens)):
            first, n = cu_q[b], cu_q[b + 1] - cu_q[b]
            start, count = kv_lens[b] - n, min(max(counts[b], 0), n)
            moves = {start + i: start + path[first + i] for i in range(count) if path[first + i] != i and start + i >= 0}
            for to_page in sorted({j // P for j in moves}):
                places = [j for j in sorted(moves) if j // P == to_page and page_of(b, moves[j]) >= 0]
                to = page_of(b, to_page * P)
                if to < 0 or not places:
                    continue
                lowest = min(j for j in moves if j // P == to_page)
                for h in range(Hkv):
                    old = e = int(scales_before[to, h]) - 127
                    for j in places:
                        origin = page_of(b, moves[j])
                        if origin != to:
                            e = max(e, ref.exponent(ref.E4M3[before[origin, h, moves[j] % P]] * 2.0 ** (int(scales_before[origin, h]) - 127)))
                    if e > old:
                        for j in range(to_page * P, lowest):
                            codes[to, h, j % P] = bring(before[to, h, j % P], old - e)
                    for j in places:
                        origin = page_of(b, moves[j])
                        codes[to, h, j % P] = bring(before[origin, h, moves[j] % P], int(scales_before[origin, h]) - 127 - e)
                    scales[to, h] = e + 127


def bring(codes, by):
    return codes if by == 0 else np.where(np.isnan(ref.E4M3[codes]), codes & 0x80 | 0x7F, ref.e4m3_code(np.nan_to_num(ref.E4M3[codes]) * 2.0 ** by))
