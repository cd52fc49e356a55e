"""The 8-bit cache and the rotary positions written out in 64 bits (numpy): test infrastructure."""
import math

import numpy as np

E_MIN, E_MAX = -32, 31


def _e4m3_table():
    """The values of the 128 non-negative codes (the last one is NaN)."""
    out = []
    for c in range(128):
        e, m = c >> 3, c & 7
        out.append(m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
    out[127] = np.nan
    return np.array(out)


TABLE = _e4m3_table()


def decode(codes):
    """Values of e4m3 codes (uint8)."""
    c = np.asarray(codes, np.uint8)
    return np.where(c & 0x80, -TABLE[c & 0x7F], TABLE[c & 0x7F])


def encode(x):
    """Nearest e4m3 codes, ties to the even code, cut at 448; NaN becomes NaN."""
    x = np.asarray(x, np.float64)
    a = np.minimum(np.abs(x), 448.0)
    hi = np.clip(np.searchsorted(TABLE[:127], np.nan_to_num(a), side="left"), 0, 126)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - TABLE[lo], TABLE[hi] - a
    c = np.where(dl < dh, lo, np.where(dl > dh, hi, np.where(lo % 2 == 0, lo, hi)))
    c = np.where(np.isnan(x), 127, c).astype(np.uint8)
    return c | (np.signbit(x).astype(np.uint8) << 7)


def exponent(amax):
    """Smallest e in range with amax <= 448 * 2^e."""
    if not amax > 0:
        return E_MIN
    if np.isinf(amax):
        return E_MAX
    m, x = math.frexp(float(amax))          # m in [0.5, 1): amax = m 2^x, 448 = 0.875 * 2^9
    return max(E_MIN, min(E_MAX, x - 9 + (1 if m > 0.875 else 0)))


def frequencies(rot, theta=10000.0, scaling="none", factor=1.0, original_context=0, low=1.0, high=32.0, magnitude=0.0, **_):
    f, m = [], 1.0
    base = theta * factor ** (rot / (rot - 2)) if scaling == "base" else theta
    if scaling == "parts":
        m = 0.1 * math.log(factor) + 1.0
        turn = lambda n: rot * math.log(original_context / (n * 2 * math.pi)) / (2 * math.log(theta))
        first, last = max(math.floor(turn(high)), 0), min(math.ceil(turn(low)), rot - 1)
    for i in range(rot // 2):
        v = base ** (-2.0 * i / rot)
        if scaling == "linear":
            v /= factor
        if scaling == "parts":
            r = min(max((i - first) / max(last - first, 1e-3), 0.0), 1.0)
            v *= 1 - r + r / factor
        if scaling == "bands":
            s = min(max((original_context * v / (2 * math.pi) - low) / (high - low), 0.0), 1.0)
            v *= s + (1 - s) / factor
        f.append(v)
    return np.array(f), magnitude or m


def rotate(x, positions, freq, magnitude, interleaved):
    """x [T, heads, dims] -> float64."""
    y = np.array(x, np.float64)
    n = len(freq)
    a = np.asarray(positions, np.float64)[:, None, None] * freq
    c, s = np.cos(a) * magnitude, np.sin(a) * magnitude
    i1, i2 = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n))
    x1, x2 = y[..., i1].copy(), y[..., i2].copy()
    y[..., i1], y[..., i2] = x1 * c - x2 * s, x2 * c + x1 * s
    return y


class Cache:
    """Codes [pages, 2, n_kv, block, dims] and exponents [pages, 2, n_kv]."""

    def __init__(self, codes, exps):
        self.codes, self.exps = codes.copy(), exps.astype(np.int32).copy()
        self.block = codes.shape[3]

    def values(self, table, n):
        """(keys, values) [n, n_kv, dims] of a row's first n tokens."""
        j = np.arange(n)
        pg, off = np.asarray(table)[j // self.block], j % self.block
        v = decode(self.codes[pg, :, :, off]) * 2.0 ** self.exps[pg][..., None]
        return v[:, 0], v[:, 1]

    def append(self, table, start, k, v):
        """k, v [n, n_kv, dims] behind the first `start` tokens of a row."""
        n = len(k)
        kv = np.stack([k, v], 1)
        for jb in range(start // self.block, (start + n - 1) // self.block + 1):
            z0, z1 = max(0, start - jb * self.block), min(self.block, start + n - jb * self.block)
            pg, t0 = table[jb], jb * self.block + z0 - start
            for kind in range(2):
                for h in range(kv.shape[2]):
                    new = kv[t0:t0 + z1 - z0, kind, h]
                    mag = np.abs(new[~np.isnan(new)])
                    e = exponent(mag.max() if mag.size else 0.0)
                    if z0 > 0:
                        old = self.exps[pg, kind, h]
                        e = max(e, old)
                        self.codes[pg, kind, h, :z0] = encode(decode(self.codes[pg, kind, h, :z0]) * 2.0 ** (old - e))
                    self.exps[pg, kind, h] = e
                    self.codes[pg, kind, h, z0:z1] = encode(new * 2.0 ** -e)

    def evict(self, table, n, mass, keep, sinks, recent):
        """One row: mass [n_kv, n ...] in place; returns the places that stayed [n_kv, keep]."""
        before, exps = self.codes.copy(), self.exps.copy()
        out = []
        for h in range(mass.shape[0]):
            middle = np.arange(sinks, n - recent)
            w = np.where(np.isnan(mass[h, middle]), -np.inf, mass[h, middle])
            pick = middle[np.argsort(-w, kind="stable")[:keep - sinks - recent]]
            src = np.sort(np.concatenate([np.arange(sinks), pick, np.arange(n - recent, n)])).astype(np.int64)
            out.append(src)
            pg, off = np.asarray(table)[src // self.block], src % self.block
            for jb in range(-(-keep // self.block)):
                j = np.arange(jb * self.block, min(keep, (jb + 1) * self.block))
                for kind in range(2):
                    es = exps[pg[j], kind, h]
                    self.exps[table[jb], kind, h] = es.max()
                    self.codes[table[jb], kind, h, :len(j)] = encode(decode(before[pg[j], kind, h, off[j]]) * 2.0 ** (es - es.max())[:, None])
            mass[h, :keep] = mass[h, src]
        return np.stack(out)


def attend(q, k, v, scale, window=0):
    """q [n, n_q, dims]: the last n of the c tokens k, v [c, n_kv, dims].  Returns (out, weights [n, n_q, c], bound [n, n_q]): bound is
    the largest sum of |q k| scale, sum of p |v| [n, n_q, dims]."""
    n, n_q, _ = q.shape
    c, n_kv, _ = k.shape
    G = n_q // n_kv
    k, v = (np.repeat(np.asarray(x, np.float64), G, 1) for x in (k, v))
    q = np.asarray(q, np.float64)
    i, j = c - n + np.arange(n)[:, None], np.arange(c)
    see = (j <= i) & ((j > i - window) if window else True)
    s = np.einsum("nhd,chd->nhc", q, k) * scale
    a = (np.einsum("nhd,chd->nhc", np.abs(q), np.abs(k)) * scale * see[:, None]).max(-1) if c else np.zeros((n, n_q))
    s = np.where(see[:, None], s, -np.inf)
    top = s.max(-1, keepdims=True)
    p = np.exp(s - np.where(np.isfinite(top), top, 0.0))
    tot = p.sum(-1, keepdims=True)
    p = np.where(tot > 0, p / np.where(tot > 0, tot, 1), 0.0)
    return np.einsum("nhc,chd->nhd", p, v), p, a, np.einsum("nhc,chd->nhd", p, np.abs(v))
