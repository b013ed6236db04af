"""Reference of the paged e4m3 cache: appending rotated keys and values, and
exact attention over the cached tokens.

Test infrastructure only (NumPy, loops over sequences, heads and tokens); the
library's code never imports it.  The rotation is defined in fp32, each
operation rounded by itself (NumPy's float32 arithmetic), so codes, scales and
rotated queries compare bit for bit; attention is float64 on the decoded cache.
"""
import numpy as np

from .sparse_attention import e4m3_encode, e4m3_table

PAGE = 64


def e4m3_decode(codes):
    return e4m3_table()[np.asarray(codes).astype(np.int64)]


def tile_places():
    """Byte in a page of (key, channel), for K and for V: two [64, 128] arrays."""
    k, v = np.empty((64, 128), dtype=np.int64), np.empty((64, 128), dtype=np.int64)
    for c in range(512):
        f, l, g = c // 64, c % 32, c // 32 % 2
        for e in range(16):
            k[32 * (f // 4) + l, 64 * (f // 2 % 2) + 32 * g + 16 * (f % 2) + e] = 16 * c + e
            v[32 * (f % 2) + 8 * (e // 4) + 4 * g + e % 4, 32 * (f // 2) + l] = 16 * c + e
    return k, v


K_PLACE, V_PLACE = tile_places()


def rotate(x, cs):
    """x float32 [heads, 128] with its first pairs turned by cs float32 [r/2, 2]."""
    x = np.array(x, dtype=np.float32)
    if cs is None:
        return x
    r = 2 * len(cs)
    a, b = x[:, 0:r:2].copy(), x[:, 1:r:2].copy()
    c, s = cs[:, 0].astype(np.float32), cs[:, 1].astype(np.float32)
    x[:, 0:r:2] = a * c - b * s
    x[:, 1:r:2] = a * s + b * c
    return x


def to_bf16_bits(x):
    """float32 -> bf16 bits, nearest even (finite)."""
    u = np.asarray(x, dtype=np.float32).view(np.uint32).astype(np.uint64)
    return ((u + 0x7FFF + ((u >> 16) & 1)) >> 16).astype(np.uint16)


def page_exponent(amax):
    """Smallest e >= -126 with amax <= 448 * 2^e."""
    e = -126
    while float(amax) > 448.0 * 2.0 ** e:
        e += 1
    return e


def append(k, v, k8, sk, v8, sv, pages, q_start, kv_len, rope=None, rope_row=None, q=None):
    """The cache (copies) after the call and the rotated queries' bf16 bits
    (None without q; zero rows where nothing is written)."""
    k8, sk, v8, sv = (a.copy() for a in (k8, sk, v8, sv))
    T, kv, _ = k.shape
    P = k8.shape[0]
    q_out = None if q is None else np.zeros(q.shape, dtype=np.uint16)
    for b in range(len(kv_len)):
        lo = min(max(int(q_start[b]), 0), T)
        n = max(min(max(int(q_start[b + 1]), 0), T) - lo, 0)
        new = {}                              # page index -> [(slot, row)]
        for i in range(n):
            pos = max(int(kv_len[b]), 0) - n + i
            if pos < 0:
                continue
            new.setdefault(pos // PAGE, []).append((pos % PAGE, lo + i, pos))
        for j, toks in new.items():
            krot = {}
            for s, t, pos in toks:
                row = pos if rope_row is None else int(rope_row[t])
                cs = rope[row] if rope is not None and 0 <= row < len(rope) else None
                krot[t] = rotate(k[t], cs)
                if q is not None:
                    q_out[t] = to_bf16_bits(rotate(q[t], cs))
            page = int(pages[b, j]) if j < pages.shape[1] else -1
            if not 0 <= page < P:
                continue
            s0 = toks[0][0]
            for h in range(kv):
                for x, code, scale, place in ((krot, k8, sk, K_PLACE), (v, v8, sv, V_PLACE)):
                    amax = max(float(np.abs(np.asarray(x[t], np.float64)[h]).max())
                               for _, t, _ in toks)
                    e = page_exponent(amax)
                    if s0 > 0:
                        old = int(np.log2(float(scale[page, h])))
                        if e > old:
                            at = place[:s0].ravel()
                            val = e4m3_decode(code[page, h, at]) * 2.0 ** (old - e)
                            code[page, h, at] = e4m3_encode(val)
                        e = max(e, old)
                    for s, t, _ in toks:
                        val = np.asarray(x[t], np.float64)[h] * 2.0 ** -e
                        code[page, h, place[s]] = e4m3_encode(val)
                    scale[page, h] = np.float32(2.0 ** e)
    return k8, sk, v8, sv, q_out


def visible(pos, keys, chunk, window):
    """Keys [lo, hi) seen from position pos."""
    if pos < 0:
        return 0, 0
    if chunk <= 0:
        return 0, keys
    c = pos // chunk
    return (max(0, c - window + 1) * chunk if window else 0), min((c + 1) * chunk, keys)


def attend(q, k8, sk, v8, sv, pages, q_start, kv_len, tau, chunk=0, window=0):
    """(o [T, H, 128], lse [T, H]) float64; NaN in rows of no sequence."""
    T, H, _ = q.shape
    P, kv, _ = k8.shape
    o, lse = np.full((T, H, 128), np.nan), np.full((T, H), np.nan)
    g = H // kv
    for b in range(len(kv_len)):
        lo_row = min(max(int(q_start[b]), 0), T)
        n = max(min(max(int(q_start[b + 1]), 0), T) - lo_row, 0)
        length = max(int(kv_len[b]), 0)
        keys = min(length, pages.shape[1] * PAGE)
        there = np.zeros(keys, dtype=bool)
        K, V = np.zeros((kv, keys, 128)), np.zeros((kv, keys, 128))
        for j in range(-(-keys // PAGE)):
            page, m = int(pages[b, j]), min(PAGE, keys - j * PAGE)
            if not 0 <= page < P:
                continue
            there[j * PAGE:j * PAGE + m] = True
            for x, code, scale, place in ((K, k8, sk, K_PLACE), (V, v8, sv, V_PLACE)):
                x[:, j * PAGE:j * PAGE + m] = e4m3_decode(code[page][:, place[:m]]) * \
                    scale[page].astype(np.float64)[:, None, None]
        for i in range(n):
            lo, hi = visible(length - n + i, keys, chunk, window)
            at = lo + np.flatnonzero(there[lo:hi])
            for h in range(H):
                if at.size == 0:
                    o[lo_row + i, h], lse[lo_row + i, h] = 0.0, -np.inf
                    continue
                x = tau * (K[h // g, at] @ np.asarray(q[lo_row + i, h], dtype=np.float64))
                m = x.max()
                p = np.exp(x - m)
                o[lo_row + i, h] = (p @ V[h // g, at]) / p.sum()
                lse[lo_row + i, h] = m + np.log(p.sum())
    return o, lse
