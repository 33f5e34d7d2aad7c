"""Plain forms in 64 bits of what stands between a decode step's products (include/tetra_kv.h, include/tetra_sample.h),
written from the headers: a cache as a dictionary of blocks, the attention row by row, the sampler by sorting."""
import numpy as np

BLOCK = 16


def byte_places(D):
    """Byte of (token, dim) in a record's keys and in its values, int [16, D]."""
    t, d = np.arange(BLOCK)[:, None], np.arange(D)[None]
    keys = d // 32 * 512 + (t % 8 * 4 + d % 32 // 8) * 16 + t // 8 * 8 + d % 8
    values = 16 * D + d // 32 * 512 + (d % 32 // 4 * 4 + t % 8 // 2) * 16 + d % 4 * 4 + t // 8 * 2 + t % 2
    return keys, values


def unpack(cache, D):
    """uint8 [..., 32 D + 16] -> (codes of keys and of values, float64 [2, ..., 16, D]; scales float32 [..., 2])."""
    cache = np.asarray(cache)
    codes = [cache[..., p.reshape(-1)].reshape(*cache.shape[:-1], BLOCK, D).astype(np.float64) - 128 for p in byte_places(D)]
    return np.stack(codes), np.ascontiguousarray(cache[..., 32 * D:32 * D + 8]).view(np.float32)


def pack(codes, scales, D):
    out = np.zeros((*codes.shape[1:-2], 32 * D + 16), np.uint8)
    for c, p in zip(codes, byte_places(D)):
        out[..., p.reshape(-1)] = (c.reshape(*c.shape[:-2], -1) + 128).astype(np.uint8)
    out[..., 32 * D:32 * D + 8] = np.ascontiguousarray(scales.astype(np.float32)).view(np.uint8)
    return out


def least_scale(amax):
    """Smallest power of two s >= 2^-126 with amax <= 127 s; 0 for 0 (and for what is below 2^-126)."""
    if amax < 2.0 ** -126:
        return 0.0
    s = 2.0 ** -126
    e = max(-126, int(np.floor(np.log2(amax))) - 8)
    s = 2.0 ** e
    while amax > 127 * s:
        s *= 2
    return s


def turned(x, weight, inv_freq, pos, eps):
    """Head norm and rotation by halves of rows [heads, D]."""
    x = np.asarray(x, np.float64)
    if weight is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * np.asarray(weight, np.float64)
    if inv_freq is not None:
        c, s = np.cos(pos * np.asarray(inv_freq, np.float64)), np.sin(pos * np.asarray(inv_freq, np.float64))
        a, b = np.split(x, 2, -1)
        x = np.concatenate([a * c - b * s, b * c + a * s], -1)
    return x


class Cache:
    """codes [2, pages, heads, blocks, 16, D] as float64, scales float32 [pages, heads, blocks, 2]."""

    def __init__(self, raw, D, page_tokens):
        self.codes, self.scales = unpack(raw, D)
        self.D, self.P = D, page_tokens

    def place(self, table, s, pos):
        """(page, block of the page, token of the block) of a position, or None."""
        if pos < 0 or pos >= table.shape[1] * self.P:
            return None
        page = int(table[s, pos // self.P])
        return None if page < 0 or page >= self.codes.shape[1] else (page, pos % self.P // BLOCK, pos % BLOCK)

    def append(self, q, k, v, table, starts, lengths, inv_freq=None, q_weight=None, k_weight=None, eps=1e-6):
        """Returns the queries, float64, NaN for rows that belong to nobody."""
        out = np.full(q.shape, np.nan)
        for s in range(len(lengths)):
            a, b = int(starts[s]), int(starts[s + 1])
            blocks = {}
            for r in range(a, b):
                pos = int(lengths[s]) + r - a
                out[r] = turned(q[r], q_weight, inv_freq, pos, eps)
                at = self.place(table, s, pos)
                if at is not None:
                    kk = turned(k[r], k_weight, inv_freq, pos, eps).astype(np.float32).astype(np.float64)
                    blocks.setdefault(at[:2], []).append((at[2], np.stack([kk, np.asarray(v[r], np.float64)])))
            for (page, block), rows in blocks.items():
                first = min(t for t, _ in rows)
                for w in range(2):
                    for h in range(self.codes.shape[2]):
                        codes = self.codes[w, page, h, block]
                        had = np.float64(self.scales[page, h, block, w]) if first > 0 else 0.0
                        new = np.stack([x[w, h] for _, x in rows])
                        if not np.isfinite(had) or not np.isfinite(new).all():
                            codes[:first] = 0
                            now = np.nan
                        else:
                            now = max(had, 0.0, least_scale(np.abs(new).max()))
                            if first > 0 and now != had:
                                codes[:first] = np.rint((codes[:first] * np.float32(max(had, 0.0) / now)).astype(np.float32))
                        for t, x in rows:
                            codes[t] = np.clip(np.rint(x[w, h] / now), -127, 127) if now > 0 else 0
                        self.scales[page, h, block, w] = now
        return out

    def tokens(self, table, s, n):
        """Keys and values float64 [2, n, heads, D] of the first n positions of a sequence, and which of them have a place."""
        out, there = np.zeros((2, max(n, 0), self.codes.shape[2], self.D)), np.zeros(max(n, 0), bool)
        for pos in range(0, n, BLOCK):
            at = self.place(table, s, pos)
            if at is None:
                continue
            m = min(BLOCK, n - pos)
            x = self.codes[:, at[0], :, at[1]] * self.scales[at[0], :, at[1]].T.astype(np.float64)[:, :, None, None]
            out[:, pos:pos + m] = x[:, :, :m].transpose(0, 2, 1, 3)
            there[pos:pos + m] = True
        return out, there

    def value_scales(self, table, s, n):
        """The scale of the values at each of the first n positions, float64 [n, heads]."""
        out = np.zeros((max(n, 0), self.codes.shape[2]))
        for pos in range(0, n, BLOCK):
            at = self.place(table, s, pos)
            if at is not None:
                out[pos:pos + BLOCK] = self.scales[at[0], :, at[1], 1]
        return out


def attend(cache, q, table, starts, lengths, scale):
    """(float64 [rows, heads, D], the bound of its error, NaN for rows that belong to nobody).

    The bound: the output is rounded once (2^-11 of it); a weight is rounded to float16 (2^-11 of it, or 2^-25 beside a
    largest of 2^7 at least), so the sum is off by 2^-11 sum p |v| at most, and by n 2^-32 of the largest p s 127; the score
    sums D products, exact ones, in float32 and is scaled, moved by the reference and raised: (D + 16) 2^-23 sum |q k| scale and
    2^-17 beside it (half a step of |score - reference| < 128), twice (numerator and denominator); outputs below float16's least step are off by half of it."""
    out, bound = np.full(q.shape, np.nan), np.full(q.shape, np.nan)
    H = cache.codes.shape[2]
    G = q.shape[1] // H
    for s in range(len(lengths)):
        a, b = int(starts[s]), int(starts[s + 1])
        n = max(0, min(int(lengths[s]) + b - a, table.shape[1] * cache.P)) if b > a else 0
        kv, there = cache.tokens(table, s, n)
        steps = cache.value_scales(table, s, n)
        for r in range(a, b):
            m = max(0, min(int(lengths[s]) + r - a + 1, n))
            use = np.flatnonzero(there[:m])
            if len(use) == 0:
                out[r] = bound[r] = 0
                continue
            k, v = kv[0, use], kv[1, use]
            qr = np.asarray(q[r], np.float64).reshape(H, G, -1)
            x = np.einsum("hgd,phd->hgp", qr, k) * scale
            size = np.einsum("hgd,phd->hgp", np.abs(qr), np.abs(k)).max(-1) * abs(scale)
            with np.errstate(invalid="ignore"):
                p = np.exp(x - x.max(-1, keepdims=True))
                p /= p.sum(-1, keepdims=True)
                o, mean = np.einsum("hgp,phd->hgd", p, v), np.einsum("hgp,phd->hgd", p, np.abs(v))
                off = 2 * ((cache.D + 16) * 2.0 ** -23 * size + 2.0 ** -17)
                most = (p * steps[use].T[:, None]).max(-1)
                e = 2.0 ** -11 * np.abs(o) + (2.0 ** -11 + off[..., None]) * mean + len(use) * 2.0 ** -32 * 127 * most[..., None] + 2.0 ** -25
            out[r], bound[r] = o.reshape(q.shape[1:]), e.reshape(q.shape[1:])
    return out, bound


def weights(x, T):
    """Weights of a row and the order of its tokens; None for a row without a token."""
    x = np.where(np.isnan(x), -np.inf, np.asarray(x, np.float64))
    order = np.argsort(-x, kind="stable")
    top = x[order[0]]
    if top == -np.inf:
        return None
    if not T > 0:
        w = np.zeros(x.size)
        w[order[0]] = 1
    elif top == np.inf:
        w = (x == np.inf) * 1.0
    else:
        with np.errstate(over="ignore", invalid="ignore"):
            w = np.where(x == -np.inf, 0.0, np.exp((x - top) / T))
    return w, order


def sample(x, u, T=1.0, k=0, p=1.0, m=0.0):
    """(token, its probability, the distance of u's aim from the nearest border in units of the largest weight)."""
    got = weights(x, T)
    if got is None:
        return -1, 0.0, 1.0
    w, order = got
    n = min(k, x.size) if k > 0 else x.size
    ws = w[order]
    if p < 1:
        n = min(n, 1 + int(np.searchsorted(np.cumsum(ws[:n]), p * ws[:n].sum())))
    if m > 0:
        n = min(n, int((ws >= m).sum()))
    kept = np.sort(order[:max(1, n)])
    c = np.cumsum(w[kept])
    aim = min(max(float(u), 0.0), 1.0) * c[-1]
    i = min(int(np.searchsorted(c, aim, side="right")), int(np.flatnonzero(w[kept])[-1]))
    lo, hi = (c[i - 1] if i else 0.0), c[i]
    return int(kept[i]), w[kept[i]] / c[-1], min(aim - lo if lo else 1.0, hi - aim if hi < c[-1] else 1.0)
