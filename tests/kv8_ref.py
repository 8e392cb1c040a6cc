"""Plain float64 form of the 8-bit KV cache's operators (numpy), and the
bounds that their tests hold results to (test infrastructure)."""
import numpy as np

PAGE, EXP_MIN = 16, -100
CODE = np.zeros(256)                       # value of each e4m3 code
for _c in range(256):
    _e, _m = _c >> 3 & 15, _c & 7
    CODE[_c] = (_m / 8 * 2.0 ** -6 if _e == 0 else (1 + _m / 8) * 2.0 ** (_e - 7)) * (-1 if _c >> 7 else 1)
CODE[0x7F] = CODE[0xFF] = np.nan
_POS = CODE[:127]                          # 0 .. 448, ascending


def k_at(t, d):
    return 1024 * (d // 64) + 64 * t + d % 64


def v_at(t, d):
    return 1024 * (d // 64) + 256 * (t // 4) + 16 * (d % 64 // 4) + 4 * (d % 4) + t % 4


def order(hd, value):
    """Byte of (token, dim) inside a group, [16, hd]."""
    t, d = np.meshgrid(np.arange(PAGE), np.arange(hd), indexing="ij")
    return (v_at if value else k_at)(t, d)


def encode(x):
    """Codes of the nearest e4m3 values (|x| <= 464), ties to even; NaN to NaN."""
    x = np.asarray(x, dtype=np.float64)
    a = np.abs(np.nan_to_num(x, nan=0.0))
    hi = np.clip(np.searchsorted(_POS, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    up = _POS[hi] - a < a - _POS[lo]
    tie = _POS[hi] - a == a - _POS[lo]
    c = np.where(up | (tie & (hi % 2 == 0)), hi, lo)
    c = np.where(a >= 448.0, 126, c)
    c = np.where(np.isnan(x), 127, c)
    return (c | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def storable(x):
    return np.where(np.abs(x) < 2.0 ** 127, x, np.nan)


def need(amax):
    e = EXP_MIN
    if amax > 0:
        e = max(int(np.floor(np.log2(amax))) - 10, EXP_MIN)
        while amax > 448.0 * 2.0 ** e:
            e += 1
    return e


def rotate(x, pos, sections, cos, sin):
    """x [heads, hd], pos: one position an axis."""
    half = x.shape[-1] // 2
    axis = np.repeat(np.arange(len(sections)), sections)
    at = np.clip(np.asarray(pos)[axis], 0, cos.shape[0] - 1)
    c, s = cos[at, np.arange(half)].astype(np.float64), sin[at, np.arange(half)].astype(np.float64)
    a, b = x[..., :half], x[..., half:]
    return np.concatenate([a * c - b * s, b * c + a * s], -1)


def write(codes, scales, table, k, v, row_start, pos0, max_len, sections=(), axis_pos=None, cos=None, sin=None,
          seq=None, q=None):
    """codes uint8 [nb, 2, hkv, 16 hd] and scales [nb, 2, hkv] in place; returns rotated q (NaN rows: not written).
    k, v, q: [rows, heads, hd] float64."""
    nb, _, hkv, wide = codes.shape
    hd = wide // PAGE
    rows = k.shape[0]
    q_out = None if q is None else np.full(q.shape, np.nan)
    for i in range(len(pos0)):
        tr = i if seq is None else seq[i]
        r0 = min(max(row_start[i], 0), rows)
        n = min(min(row_start[i + 1], rows) - r0, max_len)
        if not 0 <= tr < table.shape[0] or not 0 <= pos0[i] < table.shape[1] * PAGE:
            continue
        n = max(0, min(n, table.shape[1] * PAGE - pos0[i]))
        pages = {}
        for j in range(n):
            p = pos0[i] + j
            kk, vv = k[r0 + j], v[r0 + j]
            if sections:
                pos = [p] if axis_pos is None else axis_pos[r0 + j]
                kk = rotate(kk, pos, sections, cos, sin)
                if q is not None:
                    q_out[r0 + j] = rotate(q[r0 + j], pos, sections, cos, sin)
            pages.setdefault(p // PAGE, []).append((p % PAGE, kk, vv))
        for at, new in pages.items():
            pg = table[tr, at]
            if not 0 <= pg < nb:
                continue
            s0 = new[0][0]
            for w in (0, 1):
                where = order(hd, w)
                for h in range(hkv):
                    x = storable(np.stack([t[1 + w][h] for t in new]))
                    e = need(np.nanmax(np.abs(np.where(np.isnan(x), 0, x))))
                    g = codes[pg, w, h]
                    if s0:
                        was = int(np.log2(scales[pg, w, h]))
                        if e > was:
                            old = g[where[:s0]]
                            g[where[:s0]] = encode(CODE[old] * 2.0 ** (was - e))
                            # a code whose value became zero keeps its sign
                        e = max(e, was)
                    g[where[s0:s0 + len(new)]] = encode(x * 2.0 ** -e)
                    scales[pg, w, h] = 2.0 ** e
    return q_out


def gather(codes, scales, table_row, n):
    """(K, V, there) of the first n tokens: [n, hkv, hd] float64 and bool [n]; a page that is none gives zeros."""
    nb, _, hkv, wide = codes.shape
    hd = wide // PAGE
    K, V, there = np.zeros((n, hkv, hd)), np.zeros((n, hkv, hd)), np.zeros(n, bool)
    for b in range((n + PAGE - 1) // PAGE):
        pg = table_row[b]
        if not 0 <= pg < nb:
            continue
        m = min(PAGE, n - b * PAGE)
        val = CODE[codes[pg]] * scales[pg][:, :, None].astype(np.float64)
        K[b * PAGE:b * PAGE + m] = val[0][:, order(hd, 0)].transpose(1, 0, 2)[:m]
        V[b * PAGE:b * PAGE + m] = val[1][:, order(hd, 1)].transpose(1, 0, 2)[:m]
        there[b * PAGE:b * PAGE + m] = True
    return K, V, there


def attend(codes, scales, table, q, row_start, kv_len, max_q_len, max_kv_len, causal, scale, seq=None, bf16=True,
           only=None, weight_terms=1):
    """(out, bound) [rows, hq, hd] float64; rows outside every sequence are NaN in both.  `only`: the rows to work
    out; the others get an infinite bound.

    The bound, from the arithmetic: a score is a sum of hd (fp32: 3 hd) exact
    products in 32 bits, each addition off by 2^-23 of the sum of the terms'
    magnitudes at most; bf16 rows may enter it as two e4m3 terms under one
    power-of-two scale each, the largest element between 224 and 448: exact
    where the first term is normal (2^-6 and more), else off by half the
    second's least step, 2^-10 / 16, so by 2^-21 of the largest at most; the exponent's argument is rounded (2^-23 of its size
    and of the score's) and exp2 is good to 2^-22; a weight enters the second
    product rounded to bf16 (2^-8) for bf16 rows, whole for fp32; the two sums
    over keys add 2^-23 a term; the result is rounded to its type.  Where the
    sum that divides is of the weights as rounded, p (1 + d) with |d| <= 2^-8,
    the result moves by sum p d (v - o) / sum p (1 + d), so by 2^-8 of the mean
    |v - o| <= mean |v| + |o|, in place of 2^-8 of the mean |v|, to first order;
    1 / (1 - 2^-8) of it altogether.  weight_terms 2: bf16 rows' weights in two
    bf16 terms: what the first leaves of a weight from 2^k to 2^(k+1) is 2^(k-8)
    at most, and half a step of the second then 2^(k-17); the sum that divides
    is of the whole weights."""
    rows, hq, hd = q.shape
    hkv = codes.shape[2]
    out, bound = np.full(q.shape, np.nan), np.full(q.shape, np.nan)
    for i in range(len(kv_len)):
        tr = i if seq is None else seq[i]
        r0 = min(max(row_start[i], 0), rows)
        m = min(max(min(row_start[i + 1], rows) - r0, 0), max_q_len)
        known = 0 <= tr < table.shape[0]
        n = min(max(kv_len[i], 0), max_kv_len, table.shape[1] * PAGE) if known else 0
        K, V, there = gather(codes, scales, table[tr] if known else None, n)
        for j in range(m):
            if only is not None and r0 + j not in only:
                bound[r0 + j] = np.inf
                continue
            lim = max(0, min(n, n - m + j + 1)) if causal else n
            use = np.flatnonzero(there[:lim])
            for h in range(hq):
                kh = h // (hq // hkv)
                if not len(use):
                    out[r0 + j, h] = bound[r0 + j, h] = 0
                    continue
                x = q[r0 + j, h]
                with np.errstate(invalid="ignore"):
                    s = K[use, kh] @ x * scale
                    p = np.exp(s - s.max())
                    l = p.sum()
                    o = p @ V[use, kh] / l
                    mag = p @ np.abs(V[use, kh]) / l
                    terms = hd * (1 if bf16 else 3)
                    ds = terms * 2.0 ** -23 * (np.abs(K[use, kh]) @ np.abs(x)) * scale + np.abs(s) * 2.0 ** -22
                    if bf16:
                        ds = ds + 2.0 ** -21 * np.abs(x).max() * np.abs(K[use, kh]).sum(-1) * scale
                    ds = ds.max()
                    low = s[p > 0].min() if (p > 0).any() else np.nan        # NaN among the keys: no bound
                    dp = ds + (s.max() - low + 1) * 2.0 ** -22 + 2.0 ** -22
                    rel = 2 * dp + 2 * (len(use) * (1 if bf16 else 3) + 8) * 2.0 ** -23 + (2.0 ** (-8 if weight_terms == 1 else -17) if bf16 else 0)
                    out[r0 + j, h] = o
                    sums = np.abs(o) * 2.0 ** -8 + (mag + np.abs(o)) * 2.0 ** -15 if bf16 and weight_terms == 1 else 0
                    bound[r0 + j, h] = mag * rel + sums + np.abs(o) * (2.0 ** -8 if bf16 else 2.0 ** -24) + 2.0 ** -120
    return out, bound
