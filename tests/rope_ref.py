"""Rotary positions in 64 bits, on the CPU, and the inputs of their tests."""
import numpy as np


def table(n_pos, rot, rng, scale=1.0):
    """Cosines and sines in fp32 of angles as a model has them."""
    f = 10000.0 ** (-np.arange(rot // 2) * 2 / rot)
    a = (np.arange(n_pos) + rng.integers(0, 3))[:, None] * f
    return (np.concatenate([np.cos(a), np.sin(a)], 1) * scale).astype(np.float32)


def axes(rot, n_axes, mixed):
    i = np.arange(rot // 2)
    return (i % n_axes if mixed else i * n_axes // len(i)).tolist()


def rotate(x, tab, pos, axis, interleaved, transpose=False):
    """x [n][heads][dim] (f64) by pos [axes][n]; the products of 16-bit elements
    and 32-bit cosines are exact, their sum is rounded once."""
    pairs = len(axis)
    with np.errstate(all="ignore"):
        c, s = (np.full((x.shape[0], pairs), np.nan) for _ in range(2))
        for i, a in enumerate(axis):
            p = np.asarray(pos[a], np.int64)
            ok = p < tab.shape[0]
            c[ok, i], s[ok, i] = tab[p[ok], i], tab[p[ok], i + pairs]
        c, s = c[:, None], s[:, None] * (-1 if transpose else 1)
        out = np.array(x, np.float64)
        at, bt = (slice(0, 2 * pairs, 2), slice(1, 2 * pairs, 2)) if interleaved else (slice(0, pairs), slice(pairs, 2 * pairs))
        a, b = x[..., at], x[..., bt]
        out[..., at], out[..., bt] = a * c - b * s, b * c + a * s
    return out


def limit(want, eps, tiny, size):
    """What a rotated element in 16 bits may be off: half a step, and of fp32 the
    1.5 last places of a sum whose first product's loss comes back (2^-23 of it),
    and what underflows of that loss (2^-149 of products near 2^-126: `size`
    their sum's magnitude times 2^-46 bounds it above that)."""
    return np.abs(want) * (eps / 2 + 2.0 ** -23 * (1 + eps)) + size * 2.0 ** -46 + tiny / 2
