"""Float64 forms of the operators around the 4-bit key/value cache: norm and rotation of heads, quantiser and page layout,
attention with a query's own horizon, accumulated weights, eviction.  Plain loops over sequences and heads."""
import numpy as np

GROUP = 16


def norm_rope(x, positions, inv_freq, gamma=None, eps=None, neighbours=False, hadamard=False):
    """x [tokens][heads][dim]; eps None: no norm; inv_freq None: no rotation."""
    h = np.array(x, np.float64)
    dim = h.shape[-1]
    if eps is not None:
        h = h / np.sqrt((h * h).mean(-1, keepdims=True) + eps)
        if gamma is not None:
            h = h * np.asarray(gamma, np.float64)
    if inv_freq is not None:
        half = len(inv_freq)
        for i in range(half):
            a, b = (2 * i, 2 * i + 1) if neighbours else (i, i + half)
            t = np.asarray(positions, np.float64) * float(inv_freq[i])
            c, s = np.cos(t)[:, None], np.sin(t)[:, None]
            h[..., a], h[..., b] = h[..., a] * c - h[..., b] * s, h[..., b] * c + h[..., a] * s
    return h @ sylvester(dim) / np.sqrt(dim) if hadamard else h


def sylvester(dim):
    h = np.ones((1, 1))
    while len(h) < dim:
        h = np.block([[h, h], [h, -h]])
    return h


def bf16_below(v):
    """The largest bf16 number not above v (finite float64 within fp32's range), -0 as 0."""
    v = np.asarray(v, np.float64)
    _, e = np.frexp(v)
    step = np.ldexp(1.0, np.maximum(e, -125) - 8)
    return np.floor(v / step) * step + 0.0


def quantize(x):
    """(codes, scale, offset) of x [..., dim]; a row that is not finite has a scale of NaN."""
    x = np.asarray(x, np.float64)
    good = np.isfinite(x).all(-1, keepdims=True)
    y = np.where(good, x, 0.0)
    off = bf16_below(y.min(-1, keepdims=True))
    with np.errstate(over="ignore", divide="ignore", invalid="ignore"):
        span = (y.max(-1, keepdims=True) - off).astype(np.float32)
        scale = -bf16_below(-(span / np.float32(15)).astype(np.float64)) + 0.0
        good = good & np.isfinite(span) & (scale < 2.0 ** 128) & (off > -2.0 ** 128)
        d = (y - off).astype(np.float32)
        codes = np.where(scale > 0, np.rint(d / scale.astype(np.float32)), 0)
    codes = np.where(good, codes, 0).astype(np.uint8)
    return codes, np.where(good, scale, np.nan), np.where(good, off, np.nan)


def value(codes, scale, off):
    """What the codes stand for, as the operators form it: two fp32 operations."""
    with np.errstate(over="ignore", invalid="ignore"):
        return (off.astype(np.float32) + scale.astype(np.float32) * codes.astype(np.float32)).astype(np.float64)


def bf16_bits(v):
    """Bits of float64 values that are bf16 numbers (or NaN)."""
    with np.errstate(invalid="ignore"):
        b = (np.asarray(v, np.float32).view(np.uint32) >> 16).astype(np.uint16)
    return np.where(np.isnan(v), np.uint16(0x7fc0), b)


def group_bytes(dim):
    return GROUP * (dim + 8)


class Cache:
    """Pages [page][head][bytes], a table and lengths; the layout written out token by token."""

    def __init__(self, n_pages, heads, dim, page, table, lengths, fill=0):
        self.heads, self.dim, self.page = heads, dim, page
        self.pages = np.full((n_pages, heads, page * (dim + 8)), fill, np.uint8)
        self.table, self.lengths = np.asarray(table, np.int64), np.asarray(lengths, np.int64)

    def place(self, b, slot):
        """(page, byte of the token's group, token in the group), None where there is no page."""
        page = self.table[b, slot // self.page]
        if page < 0 or page >= len(self.pages):
            return None
        return page, slot % self.page // GROUP * group_bytes(self.dim), slot % GROUP

    def _at(self, b, h, slot, second):
        at = self.place(b, slot)
        if at is None:
            return None
        page, group, t = at
        base = group + second * GROUP * (self.dim // 2 + 4)
        codes = base + t * self.dim // 2
        params = base + GROUP * self.dim // 2 + 4 * t
        return self.pages[page, h, codes:codes + self.dim // 2], self.pages[page, h, params:params + 4]

    def write(self, b, h, slot, second, x):
        codes, scale, off = quantize(x)
        at = self._at(b, h, slot, second)
        if at is not None:
            at[0][:] = codes[0::2] | (codes[1::2] << 4)
            at[1][:] = np.concatenate((bf16_bits(scale), bf16_bits(off))).view(np.uint8)
        return value(codes, scale, off)

    def raw(self, b, h, slot, second):
        """(codes, scale, offset), None where there is no page."""
        at = self._at(b, h, slot, second)
        if at is None:
            return None
        codes = np.empty(self.dim, np.uint8)
        codes[0::2], codes[1::2] = at[0] & 15, at[0] >> 4
        p = (at[1].view(np.uint16).astype(np.uint32) << 16).view(np.float32).astype(np.float64)
        return codes, p[0], p[1]

    def exact(self, b, h, n, second):
        """Values [n][dim] with nothing rounded, magnitudes of their two terms, and which slots have a page."""
        v, m, there = np.zeros((n, self.dim)), np.zeros((n, self.dim)), np.zeros(n, bool)
        for slot in range(n):
            r = self.raw(b, h, slot, second)
            if r is not None:
                c, s, o = r
                v[slot], there[slot] = s * c + o, True
                m[slot] = np.abs(s * c) + np.abs(o)
        return v, m, there

    def length(self, b):
        return int(min(max(self.lengths[b], 0), self.table.shape[1] * self.page))


def attention(cache, b, h, q, scale):
    """q [n][group][dim] of a sequence's last n tokens: dict of out, lse, p [n][group][slots] and error magnitudes: `terms` of the
    output (sum of p times the values' terms), `logits` (the largest sum of magnitudes behind a logit that is seen) and `largest` (of the
    values' terms)."""
    n, length = q.shape[0], cache.length(b)
    k, k_terms, there = cache.exact(b, h, length, 0)
    v, v_terms, _ = cache.exact(b, h, length, 1)
    out, terms = np.zeros(q.shape), np.zeros(q.shape)
    lse, logits = np.full(q.shape[:2], -np.inf), np.zeros(q.shape[:2])
    p = np.zeros((*q.shape[:2], length))
    for i in range(n):
        seen = np.flatnonzero(there & (np.arange(length) < length - n + i + 1))
        if not len(seen):
            continue
        for g in range(q.shape[1]):
            s = k[seen] @ q[i, g] * scale
            top = s.max()
            e = np.exp(s - top)
            lse[i, g] = top + np.log(e.sum())
            p[i, g, seen] = e / e.sum()
            out[i, g], terms[i, g] = p[i, g, seen] @ v[seen], p[i, g, seen] @ v_terms[seen]
            logits[i, g] = (k_terms[seen] @ np.abs(q[i, g])).max() * abs(scale)
    return dict(out=out, lse=lse, p=p, terms=terms, logits=logits, largest=np.nanmax(v_terms, initial=0.0))


def evict(weights, positions, length, keep, recent, paged=None):
    """One head's row: (source slot of each slot that is left).  paged: which slots have a page (None: all); one that has none is no
    source for one that has, which stays as it is."""
    if length <= keep:
        return np.arange(length)
    newest = positions[:length].max()
    order = sorted(range(length), key=lambda i: (not positions[i] > newest - recent,
                                                 0 if positions[i] > newest - recent else
                                                 (1, 0) if np.isnan(weights[i]) else (0, -weights[i]), i))
    stays = set(order[:keep])
    holes = [i for i in range(keep) if i not in stays]
    source = np.arange(keep)
    source[holes] = [i for i in range(keep, length) if i in stays]
    if paged is not None:
        lost = ~np.asarray(paged, bool)[source] & np.asarray(paged, bool)[:keep]
        source[lost] = np.arange(keep)[lost]
    return source
