"""Plain definitions, in NumPy, of the operators on the paged FP8 cache and of the NVFP4 product with BF16 activations.

Codes and scales are compared bit for bit: the rotation is evaluated in the binary32 steps that define it, everything behind it
is exact or one defined rounding.  Attention is evaluated in binary64."""
import math

import numpy as np

LOWEST, HIGHEST = -112, 119


def bf16(x):
    """binary32 values rounded to BF16 (nearest even), as binary32; NaN stays NaN."""
    u = np.ascontiguousarray(x, dtype=np.float32).view(np.uint32).astype(np.uint64)
    r = ((u + 0x7FFF + ((u >> 16) & 1)) & 0xFFFF0000).astype(np.uint32).view(np.float32)
    return np.where(np.isnan(x), np.float32(np.nan), r).astype(np.float32)


def e4m3_table():
    b = np.arange(256)
    sign, e, m = np.where(b & 128, -1.0, 1.0), (b >> 3) & 15, b & 7
    v = sign * np.where(e == 0, m / 8 * 2.0 ** -6, (1 + m / 8) * 2.0 ** (e - 7.0))
    v[(b & 127) == 127] = np.nan
    return v


E4M3 = e4m3_table()


def e4m3_code(x):
    """Nearest E4M3 code of binary64 values: ties to the even code, clipped to +-448, the sign kept on zero, NaN as 0x7F."""
    x = np.asarray(x, dtype=np.float64)
    grid = E4M3[:127]
    a = np.minimum(np.abs(np.nan_to_num(x, nan=0.0, posinf=1e30, neginf=-1e30)), 448.0)
    hi = np.searchsorted(grid, a)  # the first that is not below
    lo = np.maximum(hi - 1, 0)
    hi = np.minimum(hi, 126)
    down, up = a - grid[lo], grid[hi] - a
    code = np.where((down < up) | ((down == up) & (lo % 2 == 0)), lo, hi).astype(np.uint8)
    code = code | np.where(np.signbit(x), 128, 0).astype(np.uint8)
    return np.where(np.isnan(x), 0x7F, code).astype(np.uint8)


def exponent(x):
    a = np.abs(x[np.isfinite(x)]).max(initial=0.0)
    if a == 0:
        return LOWEST
    m, e = math.frexp(float(a))
    return min(max(e - 9 if m <= 0.875 else e - 8, LOWEST), HIGHEST)


def rotate(x, row, interleaved):
    """x [H, D] binary32 (of BF16 numbers) by one table row; binary32 steps, rounded to BF16."""
    R = len(row)
    x = x.astype(np.float32).copy()
    c, s = row[: R // 2], row[R // 2 :]
    a, b = (x[:, 0:R:2].copy(), x[:, 1:R:2].copy()) if interleaved else (x[:, : R // 2].copy(), x[:, R // 2 : R].copy())
    with np.errstate(all="ignore"):
        a2, b2 = bf16(a * c - b * s), bf16(b * c + a * s)
    if interleaved:
        x[:, 0:R:2], x[:, 1:R:2] = a2, b2
    else:
        x[:, : R // 2], x[:, R // 2 : R] = a2, b2
    return x


def append(q, k, v, kc, ks, vc, vs, page_table, cu_q, kv_lens, table=None, positions=None, interleaved=False):
    """All arrays in NumPy, BF16 values as binary32; the cache is changed in place.  Returns the rotated queries (NaN for tokens
    of no sequence)."""
    pages, Hkv, P, D = kc.shape
    q_out = np.full(q.shape, np.nan, np.float32)
    for b in range(len(kv_lens)):
        n, start = cu_q[b + 1] - cu_q[b], kv_lens[b] - (cu_q[b + 1] - cu_q[b])
        rotated = {}
        for i in range(n):
            t = cu_q[b] + i
            kt = k[t]
            q_out[t] = q[t]
            if table is not None:
                p = start + i if positions is None else positions[t]
                row = table[p] if 0 <= p < len(table) else np.full(table.shape[1], np.nan, np.float32)
                q_out[t], kt = rotate(q[t], row, interleaved), rotate(k[t], row, interleaved)
            rotated[start + i] = (kt, v[t])
        by_page = {}
        for place in rotated:
            if 0 <= place < page_table.shape[1] * P:
                by_page.setdefault(place // P, []).append(place)
        for page, places in by_page.items():
            at = page_table[b, page]
            if not 0 <= at < pages:
                continue
            first = min(places) % P
            for which, codes, scales in ((0, kc, ks), (1, vc, vs)):
                for h in range(Hkv):
                    new = np.stack([rotated[p][which][h] for p in places])
                    e = exponent(new)
                    if first:
                        old = int(scales[at, h]) - 127
                        e = max(e, old)
                        if e > old:
                            codes[at, h, :first] = e4m3_code(E4M3[codes[at, h, :first]] * 2.0 ** (old - e))
                    with np.errstate(over="ignore"):
                        codes[at, h, [p % P for p in places]] = e4m3_code(new.astype(np.float64) * 2.0 ** -e)
                    scales[at, h] = e + 127
    return q_out


def attention(q, kc, ks, vc, vs, page_table, cu_q, kv_lens, scale, window=0):
    """(y, a, s) in binary64: the result, sum_j p_j |v_j|, and the largest scale * sum |q| |k| of the row's visible places."""
    pages, Hkv, P, D = kc.shape
    T, Hq, _ = q.shape
    y, a, s = np.zeros(q.shape), np.zeros(q.shape), np.zeros((T, Hq, 1))
    for b in range(len(kv_lens)):
        n, start = cu_q[b + 1] - cu_q[b], kv_lens[b] - (cu_q[b + 1] - cu_q[b])
        if n <= 0:
            continue
        places = [j for j in range(min(kv_lens[b], page_table.shape[1] * P)) if 0 <= page_table[b, j // P] < pages]
        j = np.array(places, dtype=np.int64)
        at = page_table[b, j // P] if len(j) else j
        for h in range(Hkv):
            k = E4M3[kc[at, h, j % P]] * 2.0 ** (ks[at, h].astype(np.float64) - 127)[:, None]
            v = E4M3[vc[at, h, j % P]] * 2.0 ** (vs[at, h].astype(np.float64) - 127)[:, None]
            for i in range(n):
                pos, t = start + i, cu_q[b] + i
                seen = (j <= pos) & ((j > pos - window) if window > 0 else True)
                if not seen.any():
                    continue
                G = Hq // Hkv
                x = q[t, h * G : (h + 1) * G].astype(np.float64) @ k[seen].T * scale
                p = np.exp(x - x.max(1, keepdims=True))
                p /= p.sum(1, keepdims=True)
                p = np.where(p < 1e-300, 1e-300, p)  # a NaN that is seen is not hidden by a probability that underflows
                y[t, h * G : (h + 1) * G] = p @ v[seen]
                a[t, h * G : (h + 1) * G] = p @ np.abs(v[seen])
                s[t, h * G : (h + 1) * G, 0] = (np.abs(q[t, h * G : (h + 1) * G]).astype(np.float64) @ np.abs(k[seen]).T).max(1) * scale
    return y, a, s


def attention_tolerance(y, a, s, D):
    """How far a BF16 result may be off: its own rounding, that of the probabilities (each at most 2^-8 of its value), and the
    binary32 sums of D products in the scores (an error d of a score changes a probability by a factor of at most e^2d)."""
    d = (D + 4) * 2.0 ** -24 * s
    return 2.0 ** -8 * np.abs(y) + (2.0 ** -8 + 2.5 * d + 2.0 ** -20) * (1 + 2.0 ** -7) * a


FP4 = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6])


def dequantize(codes, scales):
    """[N, K] binary64 of canonical NVFP4 codes [N, K/2] and scales [N, K/16], without the tensor-level scale."""
    N, half = codes.shape
    q = np.stack([FP4[codes & 15], FP4[codes >> 4]], -1).reshape(N, 2 * half)
    return q * np.repeat(E4M3[scales], 16, 1)
