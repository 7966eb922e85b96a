"""Plain fp64 forms of the operators around the attention (numpy), for their tests."""
import numpy as np


def rotate(x, cos, sin, interleaved, back=False):
    """x [..., d]; cos, sin broadcast against [..., r / 2]."""
    half = cos.shape[-1]
    i = np.arange(half)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    s = -sin if back else sin
    y = x.copy()
    y[..., a] = x[..., a] * cos - x[..., b] * s
    y[..., b] = x[..., b] * cos + x[..., a] * s
    return y


def pair_sum(x, half, interleaved):
    """|x| of both channels of a pair added, for every rotated channel (others: |x|): what bounds a rotation's rounding."""
    m = np.abs(x).copy()
    i = np.arange(half)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    m[..., a] = m[..., b] = np.abs(x[..., a]) + np.abs(x[..., b])
    return m


def norm_rotate(x, w, cos, sin, eps, interleaved):
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    n = x * r * w
    return (n if cos is None else rotate(n, cos, sin, interleaved)), n


def norm_rotate_bwd(x, w, cos, sin, eps, interleaved, dy):
    """dx, dw summed over all rows, and magnitudes that bound the roundings of both."""
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    hat = x * r
    dn, size = dy, np.abs(dy)
    if cos is not None:
        dn, size = rotate(dy, cos, sin, interleaved, back=True), pair_sum(dy, cos.shape[-1], interleaved)
    g, gsize = dn * w, size * np.abs(w)
    rows = tuple(range(x.ndim - 1))
    dx = r * (g - hat * (g * hat).mean(-1, keepdims=True))
    dx_size = r * (gsize + np.abs(hat) * (gsize * np.abs(hat)).mean(-1, keepdims=True))
    return dx, (dn * hat).sum(rows), dx_size, (size * np.abs(hat)).sum(rows)


# ------------------------------------------------------------------ the generator, in 64-bit unsigned numbers
def philox(counter, key, rounds=10):
    """counter: four, key: two arrays (or numbers) of 32 bits."""
    c = [np.asarray(x, dtype=np.uint64) for x in counter]
    k = [int(x) for x in key]
    low, shift = np.uint64(0xFFFFFFFF), np.uint64(32)
    for _ in range(rounds):
        p0, p1 = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(p1 >> shift) ^ c[1] ^ np.uint64(k[0]), p1 & low, (p0 >> shift) ^ c[3] ^ np.uint64(k[1]), p0 & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def keep_mask(n, p, seed, offset):
    at = np.arange((n + 7) // 8, dtype=np.uint64)
    seed, offset = seed % 2 ** 64, offset % 2 ** 64
    full = np.zeros_like(at)
    words = philox((at & np.uint64(0xFFFFFFFF), at >> np.uint64(32), full + np.uint64(offset & 0xFFFFFFFF),
                    full + np.uint64(offset >> 32)), (seed & 0xFFFFFFFF, seed >> 32))
    bits = np.stack([h for w in words for h in (w & np.uint64(0xFFFF), w >> np.uint64(16))], -1).reshape(-1)[:n]
    cut = int(np.floor(p * 65536 + 0.5))
    return bits >= np.uint64(cut), 65536.0 / (65536 - cut) if cut < 65536 else 0.0
