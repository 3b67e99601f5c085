"""Plain definitions of the paged operators in 64 bits (numpy, loops), and the tolerances that follow from the types."""
import math

import numpy as np

STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}      # a rounding to the type is off by at most this, relative


def plan(lens, new, table, free, n_free, page, max_pages, max_tokens):
    """locret_paged_plan on Python lists: dict of its outputs."""
    lens, table, free = [min(max(x, 0), max_pages * page) for x in lens], [list(r) for r in table], list(free)
    up = lambda n: -(-n // page)
    for r, n in enumerate(new):
        if n < 0:
            for p in range(up(lens[r])):
                free[n_free] = table[r][p]
                n_free += 1
            lens[r] = 0
    cu, slots, pos, stop = [0], [], [], False
    for r, n in enumerate(new):
        n = max(n, 0)
        if lens[r] + n > max_pages * page:
            n = 0
        if n > 0:
            want = up(lens[r] + n) - up(lens[r])
            if stop or want > n_free or len(slots) + n > max_tokens:
                stop, n = True, 0
        if n > 0:
            for i in range(want):
                n_free -= 1
                table[r][up(lens[r]) + i] = free[n_free]
            for u in range(lens[r], lens[r] + n):
                slots.append(table[r][u // page] * page + u % page)
                pos.append(u)
            lens[r] += n
        cu.append(cu[-1] + n)
    tail = max_tokens - len(slots)
    return dict(lens=lens, table=table, free=free, n_free=n_free, cu=cu, slots=slots + [-1] * tail, positions=pos + [0] * tail)


def rows(x, weight, eps, positions, freq, rot, interleaved, amplitude):
    """x [T][heads][d] float64 -> (values, the size of what was added for each)."""
    x = np.array(x, dtype=np.float64)
    if weight is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * np.asarray(weight, dtype=np.float64)
    y, size = x.copy(), np.abs(x)
    for t in range(x.shape[0]):
        for i in range(rot // 2):
            a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
            z = (x[t, :, a] + 1j * x[t, :, b]) * amplitude * np.exp(1j * float(positions[t]) * freq[i])
            y[t, :, a], y[t, :, b] = z.real, z.imag
            size[t, :, a] = size[t, :, b] = amplitude * (np.abs(x[t, :, a]) + np.abs(x[t, :, b]))
    return y, size


def visible(pos, n_units, window, sink):
    j = np.arange(n_units)
    see = j <= pos
    if window:
        see &= (pos - j < window) | (j < sink)
    return see


def attend(q, K, V, see, scale, dtype, factor=None):
    """One query q [d] over K, V [n][d] -> (out [d], lse, tolerance of out [d], tolerance of lse).

    Tolerance: a logit is a sum of d exact products in 32 bits, off by at most d 2^-24 of the sum of their sizes, then scaled and subtracted
    (2^-22 of its size in all); an exponential and the sums add some 2^-22.  So a probability is off by a relative `rel`,
    twice with its normalisation, and where it becomes a 16-bit factor by STEP more (`factor` instead, if given); the output is rounded once."""
    see = see.copy()
    if not see.any():
        return np.zeros(q.shape[0]), -math.inf, np.zeros(q.shape[0]), 0.0
    K, V = K[see], V[see]
    with np.errstate(all="ignore"):
        s = scale * (K @ q)
        top = s.max()
        p = np.exp(s - top)
        total = p.sum()
        p /= total
        out = p @ V
        size = p @ np.abs(V)
        rel = 2 * (q.shape[0] * 2.0 ** -24 * scale * (np.abs(K) @ np.abs(q)).max() + 2.0 ** -22 * np.abs(s).max() + 2.0 ** -20)
        half = 0.0 if dtype == "f32" else STEP["bf16"] if factor is None else factor
        tol = size * (rel + half) + np.abs(out) * STEP[dtype] + 1e-30
    lse = top + math.log(total)
    return out, lse, tol, rel + 2.0 ** -22 * abs(lse)
