"""The paged 8-bit cache and the attention over it, plainly, in 64 bits on the CPU: what the GPU tests compare with.  Nothing here uses the package."""
import numpy as np

LEAST = -110
MOST = {"e4m3": 448.0, "int8": 127.0}


def e4m3_values():
    """The value of each of the 256 codes: sign, 4 exponent bits (bias 7), 3 mantissa bits; all ones is NaN."""
    v = np.empty(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        v[c] = (m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)) * (-1 if c & 128 else 1)
        if c & 127 == 127:
            v[c] = np.nan
    return v


E4M3 = e4m3_values()
_POSITIVE = E4M3[:127]


def encode(x, fmt):
    """Values in units of their scale -> codes (uint8): nearest, ties to even; infinities to the largest; NaN to NaN, or 0."""
    x = np.asarray(x, np.float64)
    if fmt == "int8":
        return np.clip(np.rint(np.where(np.isnan(x), 0, x)), -127, 127).astype(np.int8).view(np.uint8)
    a = np.minimum(np.abs(np.where(np.isnan(x), 0, x)), 448.0)
    hi = np.searchsorted(_POSITIVE, a)                       # least code with a value of at least a
    lo = np.maximum(hi - 1, 0)
    d_lo, d_hi = a - _POSITIVE[lo], _POSITIVE[hi] - a
    c = np.where((d_lo < d_hi) | ((d_lo == d_hi) & (lo % 2 == 0)), lo, hi)
    c = c | np.where(np.signbit(x), 128, 0)
    return np.where(np.isnan(x), 127, c).astype(np.uint8)    # (either sign of NaN: compare with same_codes)


def decode(c, fmt):
    return c.view(np.int8).astype(np.float64) if fmt == "int8" else E4M3[c]


def same_codes(a, b, fmt):
    if fmt == "int8":
        return np.array_equal(a, b)
    nan = (a & 127) == 127
    return np.array_equal(nan, (b & 127) == 127) and np.array_equal(a[~nan], b[~nan])


def exponent(x, fmt):
    """Least e >= LEAST with the largest finite |x| <= most * 2^e."""
    a = np.abs(x[np.isfinite(x)])
    top = a.max() if a.size else 0.0
    if top == 0:
        return LEAST
    e = LEAST
    while top > MOST[fmt] * 2.0 ** e:
        e += 1
    return e


class RefCache:
    """k [pages, hkv, P, D], v the same (as rows), codes as uint8; exponents of the scales."""

    def __init__(self, rng, n_pages, hkv, P, D, fmt):
        self.P, self.D, self.hkv, self.fmt, self.n_pages = P, D, hkv, fmt, n_pages
        self.k, self.v = (rng.integers(0, 256, (n_pages, hkv, P, D), dtype=np.uint8) for _ in range(2))
        for x in (self.k, self.v):
            if fmt == "int8":
                x[x == 128] = 0
            else:
                x[(x & 127) == 127] = 0
        self.k_e, self.v_e = (rng.integers(-9, -5, (n_pages, hkv)) if fmt == "e4m3" else rng.integers(-7, -4, (n_pages, hkv)) for _ in range(2))
        self.weight = np.floor(np.exp(rng.standard_normal((n_pages, hkv, P))) * 8) / 8

    def copy(self):
        c = object.__new__(RefCache)
        c.__dict__.update({n: (x.copy() if isinstance(x, np.ndarray) else x) for n, x in self.__dict__.items()})
        return c

    def append(self, k, v, cu, kv_len, pages):
        """k, v [rows, hkv, D] float64"""
        for s in range(len(kv_len)):
            r0, n, ln = cu[s], cu[s + 1] - cu[s], min(int(kv_len[s]), pages.shape[1] * self.P)
            for place in range(pages.shape[1]):
                slots = [t - place * self.P for t in range(max(ln - n, 0), ln) if t // self.P == place]
                p = int(pages[s, place])
                if not slots or not 0 <= p < self.n_pages:
                    continue
                rows = [r0 + n - ln + place * self.P + j for j in slots]
                for codes, es, x in ((self.k, self.k_e, k), (self.v, self.v_e, v)):
                    for h in range(self.hkv):
                        e = exponent(x[rows, h], self.fmt)
                        lo = slots[0]
                        if lo:
                            before = es[p, h]
                            e = max(e, before)
                            if e > before:
                                codes[p, h, :lo] = encode(decode(codes[p, h, :lo], self.fmt) * 2.0 ** (before - e), self.fmt)
                        codes[p, h, slots] = encode(x[rows, h] * 2.0 ** -float(e), self.fmt)
                        es[p, h] = e
                for j in slots:
                    self.weight[p, :, j] = 0

    def rows(self, which, pages_of, n, head):
        """[n, D] values of a sequence's tokens, and which of them exist"""
        codes, es = (self.k, self.k_e) if which == "k" else (self.v, self.v_e)
        out, there = np.zeros((n, self.D)), np.zeros(n, bool)
        for t in range(n):
            p = int(pages_of[t // self.P])
            if 0 <= p < self.n_pages:
                out[t], there[t] = decode(codes[p, head, t % self.P], self.fmt) * 2.0 ** float(es[p, head]), True
        return out, there

    def attn(self, q, cu, kv_len, pages, scale, lse_in=None):
        """O [tq, hq, D], LSE [hq, tq], added weights [pages, hkv, P], and bounds: the sum of p |v| per element, the greatest error of a score per row in units of
        2^-24 (terms of a product, each rounded, are at most D + 2 roundings of their absolute sum)."""
        tq, hq, D = q.shape
        G = hq // self.hkv
        O, LSE, W = np.zeros((tq, hq, D)), np.full((hq, tq), -np.inf), np.zeros(self.weight.shape)
        absv, units = np.zeros((tq, hq, D)), np.zeros((hq, tq))
        for s in range(len(kv_len)):
            n, ln = cu[s + 1] - cu[s], min(int(kv_len[s]), pages.shape[1] * self.P)
            for h in range(self.hkv):
                K, there = self.rows("k", pages[s], ln, h)
                V, _ = self.rows("v", pages[s], ln, h)
                for i in range(n):
                    seen = there & (np.arange(ln) <= ln - n + i)
                    if not seen.any():
                        continue
                    for g in range(G):
                        row, head = cu[s] + i, h * G + g
                        with np.errstate(invalid="ignore", over="ignore"):
                            x = scale * (K[seen] @ q[row, head])
                            m = x.max()
                            z = np.exp(x - m)
                            LSE[head, row] = m + np.log(z.sum())
                            p = z / z.sum() if lse_in is None else np.exp(x - lse_in[head, row])
                            O[row, head] = p @ V[seen]
                            absv[row, head] = p @ np.abs(V[seen])
                            units[head, row] = (D + 4) * scale * (np.abs(K[seen]) @ np.abs(q[row, head])).max()
                        for t, w in zip(np.nonzero(seen)[0], p):
                            W[pages[s][t // self.P], h, t % self.P] += w
        return O, LSE, W, absv, units

    def evict(self, pages, kv_len, new_pages, budget, first, recent):
        old = self.copy()
        kept = np.full((len(kv_len), self.hkv, budget), -1, np.int32)
        new_len = np.minimum(kv_len, budget).astype(np.int32)
        for s in range(len(kv_len)):
            n = int(kv_len[s])
            for h in range(self.hkv):
                w = np.array([old.weight[pages[s][t // self.P], h, t % self.P] for t in range(n)])
                safe = lambda t: t < first or t >= n - recent
                order = sorted(range(n), key=lambda t: (not safe(t), 0 if safe(t) else (0 if np.isnan(w[t]) else 1), 0 if safe(t) or np.isnan(w[t]) else -w[t], t))
                keep = sorted(order[:budget])
                kept[s, h, : len(keep)] = keep
                for place in range(-(-len(keep) // self.P)):
                    at, p = keep[place * self.P: (place + 1) * self.P], new_pages[s][place]
                    for which, codes, es in (("k", self.k, self.k_e), ("v", self.v, self.v_e)):
                        x = np.stack([decode(getattr(old, which)[pages[s][t // self.P], h, t % self.P], self.fmt)
                                      * 2.0 ** float(getattr(old, which + "_e")[pages[s][t // self.P], h]) for t in at])
                        e = es[p, h] = exponent(x, self.fmt)
                        codes[p, h] = 0
                        codes[p, h, : len(at)] = encode(x * 2.0 ** -float(e), self.fmt)
                    self.weight[p, h] = 0
                    self.weight[p, h, : len(at)] = w[at]
        return kept, new_len


# ---- the cache's order of values --------------------------------------------------------------------------------------------------------
def v_order(rows):
    """[..., P, D] -> [..., P / 16, D, 16]"""
    *lead, P, D = rows.shape
    return np.ascontiguousarray(np.swapaxes(rows.reshape(*lead, P // 16, 16, D), -1, -2))


def v_back(v):
    *lead, n, D, _ = v.shape
    return np.ascontiguousarray(np.swapaxes(v, -1, -2)).reshape(*lead, n * 16, D)


def to_device(ref, torch, B):
    """A Cache of the package with the reference's content."""
    dt = torch.int8 if ref.fmt == "int8" else torch.float8_e4m3fn
    mk = lambda a: torch.from_numpy(a.view(np.int8).copy()).cuda().view(dt)
    sc = lambda e: torch.from_numpy((2.0 ** e.astype(np.float64)).astype(np.float32)).cuda()
    return B.Cache(mk(ref.k), mk(v_order(ref.v)), sc(ref.k_e), sc(ref.v_e), torch.from_numpy(ref.weight.astype(np.float32)).cuda())


def from_device(cache):
    """(k codes, v codes as rows, k scales, v scales, weights) as numpy arrays"""
    import torch
    bits = lambda t: t.view(torch.int8).cpu().numpy().view(np.uint8)
    return bits(cache.k), v_back(bits(cache.v)), cache.k_scale.cpu().numpy(), cache.v_scale.cpu().numpy(), cache.weight.cpu().numpy()


def check_content(cache, ref):
    k, v, ks, vs, w = from_device(cache)
    assert same_codes(k, ref.k, ref.fmt), "key codes"
    assert same_codes(v, ref.v, ref.fmt), "value codes"
    assert np.array_equal(ks, (2.0 ** ref.k_e.astype(np.float64)).astype(np.float32)), "key scales"
    assert np.array_equal(vs, (2.0 ** ref.v_e.astype(np.float64)).astype(np.float32)), "value scales"
    return w


def tables(rng, kv_len, P, extra=0, spare=2):
    """(pages [n_seqs, max_pages] int32 with -1 past a sequence's pages, number of pages of the pool): pages of a sequence lie anywhere"""
    counts = [-(-int(n) // P) for n in kv_len]
    total = sum(counts) + spare
    order = rng.permutation(total)[: sum(counts)]
    t = np.full((len(kv_len), max(max(counts), 1) + extra), -1, np.int32)
    at = 0
    for s, c in enumerate(counts):
        t[s, :c] = order[at: at + c]
        at += c
    return t, total


def bf16(rng, *shape, scale=1.0):
    """float64 values that are bf16 numbers"""
    x = (rng.standard_normal(shape) * scale).astype(np.float32)
    u = x.view(np.uint32)
    return ((u + 0x7fff + ((u >> 16) & 1)) & np.uint32(0xffff0000)).view(np.float32).astype(np.float64)
