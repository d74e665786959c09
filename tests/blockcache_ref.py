"""Plain forms of the block cache's operators in 64 bits, on the CPU, and the
inputs of their tests."""
import numpy as np
import torch

F8 = torch.float8_e4m3fn


def values(b):
    """What e4m3 bytes stand for (numpy u8 -> f64)."""
    b = b.astype(np.int64)
    e, m = (b >> 3) & 15, b & 7
    x = np.where(e == 0, m / 8 * 2.0 ** -6, (1 + m / 8) * 2.0 ** (e - 7))
    x = np.where((b & 127) == 127, np.nan, x)
    return np.where(b >= 128, -x, x)


def nearest(x):
    """x (f64, within +-448 or not finite) to e4m3 bytes, nearest even."""
    with np.errstate(all="ignore"):
        a = np.abs(x)
        e = np.frexp(np.where(np.isfinite(a) & (a > 0), a, 1.0))[1] - 1
        e = np.maximum(np.where(a > 0, e, -6), -6)
        step = 2.0 ** (e - 3.0)
        q = np.rint(a / step) * step                      # may reach the next power of two
        e2 = np.maximum(np.frexp(np.where(q > 0, q, 1.0))[1] - 1, -6)
        sub = q < 2.0 ** -6
        m = np.where(sub, q / 2.0 ** -9, (q / 2.0 ** e2 - 1) * 8)
        b = np.where(sub, 0, (e2 + 7) << 3) + np.where(np.isfinite(m), m, 0).astype(np.int64)
    b = b | np.where(np.signbit(x), 128, 0)
    return np.where(np.isfinite(x), b, 0x7F).astype(np.uint8)


def scale_for(amax):
    """The smallest power of two s >= 2^-126 with amax <= 448 s."""
    if amax == 0:
        return 2.0 ** -126
    m, e = np.frexp(amax)                                 # amax = m 2^e, 448 = 0.875 2^9
    return 2.0 ** max(-126, e - 9 if m <= 0.875 else e - 8)


class Cache:
    """Host copy of a cache: k[page][head][token][dim], v the same, as bytes."""

    def __init__(self, pages, heads, dim, block, rng, std=1.0, fill=0x7F):
        self.shape = (pages, heads, dim, block)
        self.k, self.v = (np.full((pages, heads, block, dim), fill, np.uint8) for _ in range(2))
        self.ks, self.vs = (2.0 ** rng.integers(-9, -5, (pages, heads)) for _ in range(2))
        self.rng, self.std = rng, std

    def put(self, page, n):
        """Random values in the first n slots of a page."""
        p, h, d, b = self.shape
        for x in (self.k, self.v):
            t = torch.from_numpy(self.rng.standard_normal((h, n, d)) * 100 * self.std).clamp(-448, 448).float()
            x[page, :, :n] = t.to(F8).view(torch.uint8).numpy()

    def device_v(self):
        p, h, d, b = self.shape
        t = min(b, 64)
        return np.ascontiguousarray(self.v.reshape(p, h, b // t, t, d).transpose(0, 1, 2, 4, 3))

    def from_device(self, k, v):
        p, h, d, b = self.shape
        t = min(b, 64)
        self.k = k.reshape(p, h, b, d)
        self.v = np.ascontiguousarray(v.reshape(p, h, b // t, d, t).transpose(0, 1, 2, 4, 3)).reshape(p, h, b, d)

    def held(self, pages, n, h, which):
        """Values [n][dim] in 64 bits of a sequence's first n tokens."""
        b = self.shape[3]
        x, s = (self.k, self.ks) if which == "k" else (self.v, self.vs)
        pg = np.asarray(pages[:-(-n // b)], np.int64)
        return (values(x[pg, h]) * s[pg, h][:, None, None]).reshape(-1, x.shape[-1])[:n]


def tables(rng, ctx, block, spare=2, shared=0):
    """Page tables in random order, the first `shared` blocks common to all."""
    nb = [-(-c // block) for c in ctx]
    total = shared + sum(max(0, n - shared) for n in nb) + spare
    order = rng.permutation(total)
    width = max(1, max(nb))
    t = np.zeros((len(ctx), width), np.int64)
    at = shared
    for s, n in enumerate(nb):
        k = min(n, shared)
        t[s, :k] = order[:k]
        t[s, k:n] = order[at:at + n - k]
        at += n - k
    return t, total


def attend(cache, table, ctx, n_new, q, heads, scale):
    """(out, block weights, bound on |out error| before its own rounding,
    bound on the weights' error), each in 64 bits.

    The bounds, for exact products summed in fp32 over D terms: a score is off
    by at most D 2^-24 sum |q k| scale, a weight relatively by that plus the
    exponential's and the sum's few 2^-23 (delta); the weights are rounded to
    11 bits, 2^-11 each (their steps are 2^-10 of their power of two, and half
    a step of a weight just above it is 2^-11 of it), or by 2^-25 of the largest
    (weight times value scale) below 2^-14 of it, with |value| <= 448."""
    p, hk, D, b = cache.shape
    g = heads // hk
    out = np.zeros(q.shape)
    tol = np.zeros(q.shape)
    w = np.zeros(table.shape)
    wtol = np.zeros(table.shape)
    row = 0
    with np.errstate(all="ignore"):
        for s, (n, c) in enumerate(zip(n_new, ctx)):
            for h in range(hk):
                k, v = cache.held(table[s], c, h, "k"), cache.held(table[s], c, h, "v")
                sv = np.repeat(cache.vs[table[s, :-(-c // b)], h], b)[:c]
                for t in range(n):
                    seen = c - n + t + 1
                    if seen <= 0:
                        continue
                    x = q[row + t, h * g:(h + 1) * g]                     # [g][D]
                    z = x @ k[:seen].T * scale
                    size = np.abs(x) @ np.abs(k[:seen]).T * abs(scale)
                    delta = (D * 2.0 ** -24 * size).max(1) + (8 + seen ** 0.5) * 2.0 ** -23 + np.abs(z).max(1) * 2.0 ** -22
                    e = np.exp(z - z.max(1, keepdims=True))
                    pr = e / e.sum(1, keepdims=True)
                    a = np.abs(v[:seen])
                    out[row + t, h * g:(h + 1) * g] = pr @ v[:seen]
                    tol[row + t, h * g:(h + 1) * g] = ((2.0 ** -11 + 2 * delta)[:, None] * (pr @ a)
                                                      + seen * 2.0 ** -25 * 448 * (pr * sv[:seen]).max(1)[:, None])
                    blocks = np.arange(seen) // b
                    for j in range(g):
                        w[s] += np.bincount(blocks, pr[j], len(w[s]))
                        wtol[s] += np.bincount(blocks, pr[j], len(w[s])) * 2 * delta[j]
            row += n
    wtol += w * (heads * max(1, max(n_new))) ** 0.5 * 2.0 ** -22 + 2.0 ** -40
    return out, w, tol, wtol


def evict(off, weight, hashes, keep, newest):
    out_off, pos, hs = [0], [], []
    for i in range(len(off) - 1):
        a, b = int(off[i]), int(off[i + 1])
        n = b - a
        k = min(int(keep[i]), n)
        w = [int(x) for x in weight[a:b]]
        for j in range(n - min(newest, k), n):
            w[j] = 1 << 64
        stay = sorted(sorted(range(n), key=lambda j: (-w[j], j))[:k])
        pos += stay
        hs += [int(hashes[a + j]) for j in stay]
        out_off.append(out_off[-1] + k)
    return np.array(out_off, np.uint64), np.array(pos, np.uint32), np.array(hs, np.uint64)
