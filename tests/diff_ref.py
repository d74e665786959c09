"""Differential attention over the block cache in 64 bits, on the CPU, with a
bound on what the kernels may be off."""
import numpy as np


def attend(cache, table, ctx, n_new, q, scale, lam, norm=None, eps=1e-5, gain=1.0):
    """(out, bound on |out error| before its own rounding), in 64 bits.

    Each map's bound is that of plain attention (see blockcache_ref.attend) with
    the pair's values, whose weights are rounded with the larger value scale S in
    them: 2^-11 of a weight, or 2^-25 of the largest times S, with |value| <= 448.
    The other head's values are rounded to 11 bits twice where the ratio of the
    scales is no power of two (2^-11 for the ratio and 2^-11 for the value), and
    to 2^-25 S each below fp16's smallest steps.  The difference adds one fp32
    rounding of each term; a row's norm moves by at most the root of the mean
    square of its elements' errors, and the norm's own arithmetic is few 2^-23."""
    p, hk, D, b = cache.shape
    g = q.shape[1] // hk
    out = np.zeros((q.shape[0], q.shape[1] // 2, 2 * D))
    tol = np.zeros(out.shape)
    row = 0
    with np.errstate(all="ignore"):
        for s, (n, c) in enumerate(zip(n_new, ctx)):
            for pr in range(hk // 2):
                ks = [cache.held(table[s], c, 2 * pr + m, "k") for m in range(2)]
                vh = [cache.held(table[s], c, 2 * pr + m, "v") for m in range(2)]
                v = np.concatenate(vh, 1)
                sv = [np.repeat(cache.vs[table[s, :-(-c // b)], 2 * pr + m], b)[:c] for m in range(2)]
                S = np.maximum(*sv)
                ratio = [x / np.where(S > 0, S, 1) for x in sv]
                exact = [np.frexp(r)[0] == 0.5 for r in ratio]
                # per value: relative roundings where the ratio is no power of two, absolute 2^-25 S below fp16's steps
                rel = np.concatenate([np.where(e, 0.0, 2.0 ** -10)[:, None].repeat(D, 1) for e in exact], 1)
                step = np.concatenate([np.where(e & (r >= 2.0 ** -15), 0.0, 2.0 ** -24 * S)[:, None].repeat(D, 1)
                                       for e, r in zip(exact, ratio)], 1)
                for t in range(n):
                    seen = c - n + t + 1
                    if seen <= 0:
                        continue
                    for i in range(g):
                        j = pr * g + i
                        o, e = [], []
                        for m in range(2):
                            x = q[row + t, 2 * j + m]
                            z = ks[m][:seen] @ x * scale
                            size = np.abs(ks[m][:seen]) @ np.abs(x) * abs(scale)
                            delta = (D * 2.0 ** -24 * size).max() + (8 + seen ** 0.5) * 2.0 ** -23 + np.abs(z).max() * 2.0 ** -22
                            w = np.exp(z - z.max())
                            w /= w.sum()
                            a = np.abs(v[:seen])
                            o.append(w @ v[:seen])
                            e.append((2.0 ** -11 + 2 * delta) * (w @ a) + w @ (a * rel[:seen]) + w @ step[:seen]
                                     + seen * 2.0 ** -25 * 448 * (w * S[:seen]).max())
                        d = o[0] - lam[j] * o[1]
                        err = e[0] + abs(lam[j]) * e[1] + 2.0 ** -23 * (np.abs(o[0]) + 2 * np.abs(lam[j] * o[1]))
                        if norm is not None:
                            rms = np.sqrt((d * d).mean() + eps)
                            move = np.sqrt((err * err).mean())
                            low = max(rms - move, np.sqrt(eps))
                            err = abs(gain) * np.abs(norm) * (err + np.abs(d) / rms * move) / low
                            d = gain * norm * d / rms
                        else:
                            err, d = abs(gain) * err, gain * d
                        out[row + t, j] = d
                        tol[row + t, j] = err + 2.0 ** -20 * np.abs(d)
            row += n
    return out, tol
