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


# ------------------------------------------------------------------ attention to another sequence
U = 2.0 ** -8           # half a step of bf16, relative


def cross(q, k, v, lengths, scale, do=None):
    """One batch of fp64 arrays [B, H, N, d].  Returns {name: (value, bound)}; the bounds count what the kernels round.

    Forward: probabilities are rounded to bf16 and divided by the sum of the rounded ones, so that the weights are off by U
    of each against their mean: U sum p |v - o| <= U (sum p |v| + |o|); the result is rounded, U |o|.  Scores, exponentials
    and sums in fp32: 2^-13 of sum p |v| is far more than they lose.
    Backward: p from a log-sum-exp that holds the mean rounding of a row, and rounded itself, 2 U; dS = p (dP - D) with a D that
    holds the weights' error of o (o is there to 16 bits), and rounded, U; every result is rounded, U."""
    B, Hq, Nq, d = q.shape
    Hk, Nk = k.shape[1:3]
    out = {n: (np.zeros(s), np.zeros(s)) for n, s in (("o", q.shape), ("dq", q.shape), ("dk", k.shape), ("dv", k.shape))}
    lse = np.full((B, Hq, Nq), -np.inf)
    small = 2.0 ** -13
    for b in range(B):
        n = Nk if lengths is None else int(min(max(lengths[b], 0), Nk))
        if n == 0:
            continue
        for h in range(Hq):
            g = h // (Hq // Hk)
            kk, vv = k[b, g, :n], v[b, g, :n]
            s = scale * q[b, h] @ kk.T
            top = s.max(-1, keepdims=True)
            e = np.exp(s - top)
            p = e / e.sum(-1, keepdims=True)
            lse[b, h] = top[:, 0] + np.log(e.sum(-1))
            o, pv = p @ vv, p @ np.abs(vv)
            weights = U * (pv + np.abs(o)) + small * pv
            out["o"][0][b, h], out["o"][1][b, h] = o, weights + U * np.abs(o)
            if do is None:
                continue
            up = do[b, h]
            dp = up @ vv.T
            D = (up * o).sum(-1, keepdims=True)
            ds = p * (dp - D)
            ds_bound = p * (np.abs(up) * (weights + 2.0 ** -15 * np.abs(o))).sum(-1, keepdims=True) + 3 * U * np.abs(ds) \
                + small * p * (np.abs(up) @ np.abs(vv).T + np.abs(D))
            out["dq"][0][b, h], out["dq"][1][b, h] = scale * ds @ kk, scale * ds_bound @ np.abs(kk)
            out["dk"][0][b, g, :n] += scale * ds.T @ q[b, h]
            out["dk"][1][b, g, :n] += scale * ds_bound.T @ np.abs(q[b, h])
            out["dv"][0][b, g, :n] += p.T @ up
            out["dv"][1][b, g, :n] += (2 * U + small) * p.T @ np.abs(up)
    for n in ("dq", "dk", "dv"):
        out[n] = (out[n][0], out[n][1] + U * np.abs(out[n][0]))
    return out, lse
