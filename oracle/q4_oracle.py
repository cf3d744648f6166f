"""The 4-bit cache and eviction by accumulated weight in NumPy, 64 bits: what the kernels are checked against.

Written from the definitions in include/packcache.h, one row or group at a time where that is clearer; shares nothing
with the library or with perf/.
"""
import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def q4_scale_exponent(top: float) -> int:
    """The least e with top <= 7 * 2^e, kept from -120 to 125."""
    e = -120
    while e < 125 and float(top) > 7.0 * 2.0 ** e:
        e += 1
    return e


def q4_nearest(v: float) -> int:
    """Code (without sign) of the grid value nearest to |v|; between two the even code; 6 is the largest."""
    d = np.abs(GRID - abs(v))
    best = np.flatnonzero(d == d.min())
    return int(best[0] if len(best) == 1 or best[0] % 2 == 0 else best[1])


def q4_store(x):
    """x [..][D] -> (codes uint8 [..][D/2], scale bytes uint8 [..][D/32])."""
    x = np.asarray(x, np.float64)
    groups = x.reshape(-1, 32)
    bad = ~np.all(np.isfinite(groups), -1)
    v = np.where(bad[:, None], 0.0, groups)
    largest = 7.0 * 2.0 ** np.arange(-120.0, 126.0)                 # that a group may hold, by its exponent
    e = np.minimum(np.searchsorted(largest, np.max(np.abs(v), -1), "left"), 245) - 120
    borders = (GRID[1:] + GRID[:-1]) / 2
    a = np.abs(v) / 2.0 ** e[:, None].astype(np.float64)
    low, high = np.searchsorted(borders, a, "left"), np.searchsorted(borders, a, "right")
    codes = np.where(low % 2 == 0, low, high) + 8 * np.signbit(v)   # low < high only on a border
    codes = np.where(bad[:, None], 0, codes).astype(np.uint8).reshape(x.shape)
    scales = np.where(bad, 255, e + 127).astype(np.uint8).reshape(x.shape[:-1] + (-1,))
    return codes[..., 0::2] | (codes[..., 1::2] << 4), scales


def q4_load(codes, scales):
    """The values, float64 [..][D]."""
    nib = np.stack([codes & 15, codes >> 4], -1).reshape(codes.shape[:-1] + (-1,))
    v = GRID[nib & 7] * np.where(nib & 8, -1.0, 1.0)
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return v * np.repeat(s, 32, -1)


def attn(Q, K, V, scale):
    """Softmax attention with probabilities: O [Hq][Nq][D], lse [Hq][Nq], mass [Hkv][Nk] (probabilities summed over rows
    and heads)."""
    Hq, Nq, _ = Q.shape
    Hkv, Nk, _ = K.shape
    rep = Hq // Hkv
    O, lse, mass = np.zeros(Q.shape), np.zeros((Hq, Nq)), np.zeros((Hkv, Nk))
    with np.errstate(invalid="ignore", over="ignore"):
        for h in range(Hq):
            s = Q[h] @ K[h // rep].T * scale
            m = s.max(-1, keepdims=True)
            p = np.exp(s - m)
            l = p.sum(-1, keepdims=True)
            O[h] = p @ V[h // rep] / l
            lse[h] = (m + np.log(l))[:, 0]
            mass[h // rep] += (p / l).sum(0)
    return O, lse, mass


def evict_rows(weights, t, Nk, n_keep, n_anchor=0, recent_t=0):
    """Of one selection head: which row each of rows 0 .. n_keep - 1 holds afterwards.  t [Nk] or None."""
    if n_keep >= Nk:
        return np.arange(Nk)

    def order(j):
        safe = j < n_anchor or (recent_t > 0 and int(t[j]) > int(t[Nk - 1]) - recent_t)
        w = float(weights[j])
        return (0, 0.0, j) if safe else (1, -w, j) if not np.isnan(w) else (2, 0.0, j)

    kept = set(sorted(range(Nk), key=order)[:n_keep])
    movers = iter(sorted(j for j in kept if j >= n_keep))
    return np.array([j if j in kept else next(movers) for j in range(n_keep)])
