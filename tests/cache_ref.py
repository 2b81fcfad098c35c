"""The calls on a paged cache in float64, from their definitions, on the CPU, and what their results
may be off by.

Half a step of the result's type, u, counts once for the result and, in attention, once for every
numerator (they are rounded for the matrix product; the sum that they are divided by is not).  A
score is a sum of D products of 16-bit numbers, exact each, in 32 bits: off by D 2^-24 of the sum of
their magnitudes at most, which is the relative error of a numerator, with 2^-22 for the hardware
exponential and 2^-23 of the exponent's size for its argument.  Sums over L slots in 32 bits: L 2^-24.
A float16 numerator below 2^-28 of its row's largest is off by 2^-39 of that."""
import numpy as np

HALF_STEP = {"bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}


def slots(cache, pages, S, b, n):
    """[n, H, D] of a sequence's first n slots of cache [P, S, H, D]; zeros where a page is not there."""
    out = np.zeros((n, *cache.shape[2:]))
    for j in range(n):
        page = pages[b, j // S]
        if 0 <= page < cache.shape[0]:
            out[j] = cache[page, j % S]
    return out


def sees(i, start, n, parents):
    """The slots that draft i sees."""
    to = list(range(start))
    while 0 <= i < n:
        to.append(start + i)
        up = i - 1 if parents is None else int(parents[i])
        i = up if 0 <= up < i else -1
    return sorted(to)


def attend(q, k_cache, v_cache, pages, starts, lengths, parents, scale, dtype):
    """(out, lse, bounds of their errors), q [B, N, Hq, D] and caches in float64."""
    u = HALF_STEP[dtype]
    B, N, Hq, D = q.shape
    S, Hk = k_cache.shape[1:3]
    G = Hq // Hk
    most = pages.shape[1] * S
    out, lse = np.zeros(q.shape), np.full(q.shape[:3], -np.inf)
    off, loff = np.zeros(q.shape), np.zeros(q.shape[:3])
    for b in range(B):
        n, start = min(max(lengths[b], 0), N), min(max(starts[b], 0), most)
        end = min(start + n, most)
        k, v = slots(k_cache, pages, S, b, end), slots(v_cache, pages, S, b, end)
        for i in range(n):
            to = [j for j in sees(i, start, n, None if parents is None else parents[b]) if j < end]
            if not to:
                continue
            for h in range(Hq):
                kk, vv = k[to, h // G], v[to, h // G]
                s = scale * (kk @ q[b, i, h])
                m = s.max()
                p = np.exp(s - m)
                l = p.sum()
                p /= l
                out[b, i, h] = p @ vv
                lse[b, i, h] = m + np.log(l)
                size = np.abs(s).max() * 1.5
                e = D * 2.0 ** -24 * scale * (np.abs(kk) @ np.abs(q[b, i, h])).max() + \
                    2.0 ** -22 + 2.0 ** -23 * size + len(to) * 2.0 ** -24
                mean = p @ np.abs(vv)
                tiny = len(to) * 2.0 ** -39 * np.abs(vv).max(0) if dtype == "float16" else 0.0
                off[b, i, h] = u * np.abs(out[b, i, h]) + (u + 2 * e) * mean + tiny + 2.0 ** -24
                loff[b, i, h] = 2 * e + 2.0 ** -23 * abs(lse[b, i, h])
    return out, lse, off, loff


def rotate(x, positions, freqs, neighbours, dtype):
    """(x [..., H, D] with its first 2 len(freqs) elements turned, bounds), positions [...]."""
    h = len(freqs)
    y, size = x.copy(), np.abs(x)
    if h:
        angle = positions[..., None, None].astype(np.float64) * freqs.astype(np.float64)
        c, s = np.cos(angle), np.sin(angle)
        one = np.arange(h) * 2 if neighbours else np.arange(h)
        two = one + 1 if neighbours else one + h
        y[..., one] = x[..., one] * c - x[..., two] * s
        y[..., two] = x[..., two] * c + x[..., one] * s
        size[..., one] = size[..., two] = np.abs(x[..., one]) + np.abs(x[..., two])
    # sine and cosine are off by 2^-22 (2^-24 of a turn in their argument, and their own), and so
    # are two products and their sum
    turned = np.arange(x.shape[-1]) < 2 * h
    return y, np.where(turned, HALF_STEP[dtype] * np.abs(y) + 2.0 ** -21 * size + 2.0 ** -25, 0.0)
