"""Plain float64 numpy statements of the operators around an 8-bit K/V cache and of log probabilities, for their tests."""
import numpy as np

NAN_CODE = 0x7F


def _decode_table():
    t = np.empty(256)
    for c in range(256):
        sign, e, m = (-1.0 if c & 0x80 else 1.0), (c >> 3) & 15, c & 7
        t[c] = np.nan if (c & 0x7F) == NAN_CODE else sign * (m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
    return t


TABLE = _decode_table()
_POS = TABLE[:NAN_CODE]                                   # 0 .. 448, ascending: the code is the index


def encode(x):
    """Nearest e4m3 code, halves to the even code, saturating; NaN to NaN."""
    x = np.asarray(x, dtype=np.float64)
    a = np.minimum(np.abs(np.where(np.isnan(x), 0.0, x)), 448.0)
    hi = np.clip(np.searchsorted(_POS, a), 0, NAN_CODE - 1)           # first code with value >= a
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - _POS[lo], _POS[hi] - a
    c = np.where(dl < dh, lo, np.where(dh < dl, hi, np.where(lo % 2 == 0, lo, hi)))
    c = np.where(np.signbit(x), c | 0x80, c)
    return np.where(np.isnan(x), NAN_CODE, c).astype(np.uint8)


def scale_for(a):
    s = 2.0 ** -120
    while a > 448 * s:
        s *= 2
    return s


def append(kv, which, rows, n_new, page):
    """rows [B, M, Hkv, dh] float64 into kv[which + '_pages'] (uint8 codes) and its scales, in place."""
    P, S = kv[which + "_pages"], kv[which + "_scales"]
    num_pages, hkv = P.shape[:2]
    capacity = kv["block_table"].shape[1] * page
    for b in range(rows.shape[0]):
        L, n = int(kv["seq_lens"][b]), int(n_new[b])
        for blk in range(L // page, (L + n + page - 1) // page if n else L // page):
            first, end = max(L, blk * page), min(L + n, (blk + 1) * page, capacity)
            if first >= end:
                continue
            pg = int(kv["block_table"][b, blk])
            if not 0 <= pg < num_pages:
                continue
            for h in range(hkv):
                x = rows[b, first - L:end - L, h]
                fin = np.abs(x[np.isfinite(x)])
                s = scale_for(fin.max() if fin.size else 0.0)
                at, old = blk * page, float(S[pg, h])
                if first > at:
                    if old >= s:
                        s = old
                    else:
                        kept = P[pg, h, :first - at]
                        P[pg, h, :first - at] = encode(TABLE[kept] * (old / s))
                with np.errstate(invalid="ignore"):
                    P[pg, h, first - at:end - at] = encode(x / s)
                S[pg, h] = s


def tokens(kv, which, b, n, page):
    """The first n positions of a sequence [n, Hkv, dh] as float64 values."""
    out = []
    for blk in range((n + page - 1) // page):
        pg = int(kv["block_table"][b, blk])
        out.append((TABLE[kv[which + "_pages"][pg]] * kv[which + "_scales"][pg].astype(np.float64)[:, None, None]).transpose(1, 0, 2))
    hkv, dh = kv["k_pages"].shape[1], kv["k_pages"].shape[3]
    return np.concatenate(out)[:n] if out else np.zeros((0, hkv, dh))


def attention(kv, q, n_new, page):
    """q [B, M, Hq, dh] float64 -> (out, bound): the result and how far the kernel's may be off, element by element (NaN rows
    where n_new excludes them).

    The bound: a probability enters in two e4m3 parts, each off by 2^-4 of itself at most, so by 2^-8 of the probability, or by 2^-11
    steps of the second part's smallest code (2^-9 / (256 * 32) of the chunk's largest weight); the result is rounded to bf16
    (2^-8). Scores: the products are exact, an fp8 MMA adds them with an error of 2^-20 of their magnitudes' sum (it keeps 22 bits of
    the largest), which moves a probability by as much; 2^-14 is left for the exponentials, fp32 sums and joins."""
    B, M, Hq, dh = q.shape
    hkv = kv["k_pages"].shape[1]
    g = Hq // hkv
    out = np.full(q.shape, np.nan)
    tol = np.zeros(q.shape)
    for b in range(B):
        if not n_new[b]:
            continue
        L = int(kv["seq_lens"][b])
        T = min(L + int(n_new[b]), kv["block_table"].shape[1] * page)
        K, V = tokens(kv, "k", b, T, page), tokens(kv, "v", b, T, page)
        for m in range(int(n_new[b])):
            n = min(L + m + 1, T)
            for h in range(Hq):
                k, v = K[:n, h // g], V[:n, h // g]
                s = k @ q[b, m, h] / np.sqrt(dh)
                w = np.exp(s - s.max())
                w /= w.sum()
                o = w @ v
                mass = w @ np.abs(v)
                serr = 2.0 ** -20 * (np.abs(k) @ np.abs(q[b, m, h])).max() / np.sqrt(dh)
                out[b, m, h] = o
                tol[b, m, h] = 2.0 ** -8 * (mass + np.abs(o)) + (2 * serr + 2.0 ** -14) * mass + \
                    2.0 ** -22 * min(n, 1024) * np.abs(v).max() * w.max() + 1e-30
    return out, tol


def logprobs(x, tok, top):
    """x [rows, V] float64 (NaN allowed) -> logprob, entropy, ids, logprobs of the ids."""
    x = np.where(np.isnan(x), -np.inf, x)
    R, V = x.shape
    lp, ent = np.empty(R), np.empty(R)
    ids, tops = np.empty((R, top), np.int32), np.empty((R, top))
    for r in range(R):
        m = x[r].max()
        with np.errstate(invalid="ignore"):
            d = np.where(x[r] == m, 0.0, x[r] - m)
        p = np.exp(d)
        S = p.sum()
        all_lp = d - np.log(S)
        pos = p > 0
        ent[r] = np.log(S) - (p[pos] * d[pos]).sum() / S
        if m == -np.inf:
            all_lp[:], ent[r] = -np.inf, 0.0
        order = np.lexsort((np.arange(V), -x[r]))[:top]
        lp[r] = all_lp[tok[r]]
        ids[r], tops[r] = order, all_lp[order]
    return lp, ent, ids, tops
