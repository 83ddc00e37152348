"""Plain 64-bit paged key-value cache and attention: the oracle of sae_kv_* and sae_attn_*.

A cache is held as its values, [block][head][token][dim] float64; pack() lays them out as the library does,
element by element from the formula of include/sae.h.
"""
import numpy as np

BLOCK = 16
BF16, F16, FP8 = 0, 1, 2
# unit roundoff of the 16-bit types: half a unit in the last place, relative
ROUNDOFF = {BF16: 2.0 ** -8, F16: 2.0 ** -11}


def e4m3_table():
    """The value of every float8 e4m3 byte (1 sign, 4 exponent bits of bias 7, 3 fraction bits; S.1111.111 is NaN)."""
    b = np.arange(256)
    e, f = (b >> 3) & 15, b & 7
    v = np.where(e == 0, f * 2.0 ** -9, (8 + f) * 2.0 ** (e - 10.0))
    v = np.where((b & 127) == 127, np.nan, v)
    return np.where(b >= 128, -v, v)


def to_e4m3(x):
    """Bytes of the nearest e4m3 values, ties to the even byte; |x| <= 448 or not finite (NaN)."""
    t = e4m3_table()[:127]
    a = np.abs(np.where(np.isfinite(x), x, 0.0))
    hi = np.clip(np.searchsorted(t, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - t[lo], t[hi] - a
    b = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    b = np.where(np.isfinite(x), b, 127)
    return (b | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def quantise(x):
    """x [..., dim]: (e4m3 bytes, scale bytes [...]) as sae_kv_write stores them."""
    top = np.where(np.isfinite(x), np.abs(x), 0.0).max(-1)
    e = np.full(top.shape, -126, np.int64)
    while True:  # the smallest e >= -126 with top <= 448 * 2^e
        up = top > 448.0 * 2.0 ** e
        if not up.any():
            break
        e += up
    e = np.where(top == 0, 0, e)
    with np.errstate(invalid="ignore"):
        return to_e4m3(x * 2.0 ** -e[..., None].astype(np.float64)), (e + 127).astype(np.uint8)


def dequantise(b, scale):
    return e4m3_table()[b] * 2.0 ** (scale.astype(np.float64) - 127)[..., None]


def places(dim, size):
    """Index in a page of (token, dimension), for keys and for values: two arrays [16][dim]."""
    c = 16 // size
    k, v = np.zeros((BLOCK, dim), np.int64), np.zeros((BLOCK, dim), np.int64)
    for t in range(BLOCK):
        for d in range(dim):
            k[t, d] = (d // c * BLOCK + t) * c + d % c
            i = d // (2 * c)
            for width, at in ((16, d % 16), (2, t // 4 % 2), (c // 8, d // 16 % (c // 8)), (2, t // 8), (4, t % 4)):
                i = i * width + at
            v[t, d] = i
    return k, v


def pack(x, size, which):
    """x [..., 16][dim] (any dtype of `size` bytes) as pages [..., 16 dim]; which: 0 keys, 1 values."""
    at = places(x.shape[-1], size)[which].reshape(-1)
    out = np.empty(x.shape[:-2] + (at.size,), x.dtype)
    out[..., at] = x.reshape(x.shape[:-2] + (-1,))
    return out


def unpack(pages, dim, size, which):
    at = places(dim, size)[which].reshape(-1)
    return pages[..., at].reshape(pages.shape[:-1] + (BLOCK, dim))


def rows_of(ids, n, cache):
    """Positions 0 .. n - 1 of a sequence with block table ids: values [n][head][dim] and which positions there are."""
    pos = np.arange(n)
    b = ids[pos // BLOCK]
    there = (b >= 0) & (b < cache.shape[0])
    return cache[np.where(there, b, 0), :, pos % BLOCK], there


def attention(q, at, k, v, there, scale, window):
    """Queries q [n][heads][dim] at positions at[n] over keys and values [len][kv_heads][dim].

    Returns out, lse and, for error bounds, per row: the mean magnitude sum w |v| / sum w of every output and the
    largest scale * sum |q| |k| among the keys it sees."""
    n, heads, dim = q.shape
    kvh = k.shape[1]
    out, mag = np.zeros((n, heads, dim)), np.zeros((n, heads, dim))
    lse, big = np.full((n, heads), -np.inf), np.zeros((n, heads))
    pos = np.arange(k.shape[0])
    for i in range(n):
        seen = there & (pos <= at[i])
        if window:
            seen &= pos > at[i] - window
        if not seen.any():
            continue
        for h in range(kvh):
            g = slice(h * (heads // kvh), (h + 1) * (heads // kvh))
            kk, vv = k[seen, h], v[seen, h]
            s = scale * (q[i, g] @ kk.T)
            top = s.max(1, keepdims=True)
            dead = top[:, 0] == -np.inf
            top[dead] = 0
            w = np.exp(s - top)
            z = w.sum(1, keepdims=True)
            z1 = np.where(z == 0, 1, z)
            out[i, g], mag[i, g] = (w @ vv) / z1, (w @ np.abs(vv)) / z1
            with np.errstate(divide="ignore"):
                lse[i, g] = (top + np.log(z))[:, 0]
            big[i, g] = (abs(scale) * (np.abs(q[i, g]) @ np.abs(kk).T)).max(1)
    return out, lse, mag, big


def bounds(out, lse, mag, big, dim, dtype, weight=None, floor=0.0):
    """How far outputs of `dtype` and log-sum-exps may be off.

    Scores are sums of dim exact products in fp32: off by at most (dim + 4) 2^-24 of the sum of their magnitudes
    (the scale and the base of the exponential included), and the exponential by a few 2^-23: a weight's relative error
    is rel.  Weights are rounded for the product with the values, by at most `weight` relative (the 16-bit type's
    roundoff where none is given; its square where a weight is taken as two such numbers); the normaliser is not.  Sums
    of non-negative weights in fp32 add less than 2^-20.  Then one rounding of the result.

    floor: what the weights' rounding may add to an output in all beside that, where the 16-bit type ends below them
    (f16): the largest |value| times the number of keys times the type's half step, in units of a row's largest weight
    (the normaliser is at least one such)."""
    u = ROUNDOFF[dtype]
    rel = (dim + 4) * 2.0 ** -24 * big + 2.0 ** -20
    tiny = 2.0 ** -25 if dtype == F16 else 2.0 ** -134  # half the smallest subnormal
    return (u * np.abs(out) + ((u if weight is None else weight) + 2 * rel)[..., None] * mag * (1 + u) + tiny + floor,
            rel + 2.0 ** -22 * np.abs(np.where(np.isfinite(lse), lse, 0)))


def tree_seen(parent, total, there, window):
    """seen [n][total]: which places each node of a tree sees, by walking up from it.  parent [n] (-1: the prefix)."""
    n = len(parent)
    base = total - n
    seen = np.zeros((n, total), bool)
    for j in range(n):
        if base + j < 0:
            continue  # no place
        way = [j]
        while parent[way[-1]] >= 0:
            way.append(parent[way[-1]])
        pos = base + len(way) - 1
        for up, i in enumerate(way):
            if base + i >= 0 and (not window or pos - up > pos - window):
                seen[j, base + i] = True
        prefix = np.arange(max(base, 0))
        seen[j, prefix] = True if not window else prefix > pos - window
    return seen & there[None, :]


def tree_attention(q, parent, k, v, there, scale, window):
    """Queries q [n][heads][dim] of a tree's nodes, the last n places of keys and values [len][kv_heads][dim]; returns as
    attention() does."""
    n, heads, dim = q.shape
    kvh = k.shape[1]
    out, mag = np.zeros((n, heads, dim)), np.zeros((n, heads, dim))
    lse, big = np.full((n, heads), -np.inf), np.zeros((n, heads))
    seen = tree_seen(parent, k.shape[0], there, window)
    for i in range(n):
        at = np.nonzero(seen[i])[0]
        if not len(at):
            continue
        for h in range(kvh):
            kk, vv = k[at, h], v[at, h]
            ka, va = np.abs(kk), np.abs(vv)
            for u in range(h * (heads // kvh), (h + 1) * (heads // kvh)):
                s = scale * (kk @ q[i, u])
                w = np.exp(s - s.max())
                out[i, u], mag[i, u] = (w @ vv) / w.sum(), (w @ va) / w.sum()
                lse[i, u] = s.max() + np.log(w.sum())
                big[i, u] = abs(scale) * (ka @ np.abs(q[i, u])).max()
    return out, lse, mag, big


def turn(x, pos, inv_freq, interleaved=False, factor=1.0):
    """Rows x [n][heads][dim] at positions pos [n] turned pair by pair (see sae_rope in include/sae.h)."""
    half = len(inv_freq)
    y = np.array(x, np.float64)
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        angle = np.asarray(pos, np.float64) * float(inv_freq[i])
        c, s = factor * np.cos(angle)[:, None], factor * np.sin(angle)[:, None]
        y[:, :, a], y[:, :, b] = x[:, :, a] * c - x[:, :, b] * s, x[:, :, a] * s + x[:, :, b] * c
    return y
