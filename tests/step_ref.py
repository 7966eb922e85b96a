"""Plain fp64 forms of the operators of a training step around the attention (numpy), for their tests, with bounds of what the kernels'
roundings may change."""
import numpy as np

HALF = {"bfloat16": 2.0 ** -8, "float32": 2.0 ** -24}          # half a step, relative
# What sums and products in fp32 lose, relative to the sum of the magnitudes that enter: a thread adds up to 32 channels (or the
# tokens of its workgroup, a few dozen here) one by one and then over lanes and waves, 2^-24 a step, and a handful of products: far
# less than 128 steps.
SMALL = 2.0 ** -17


def gate_sum(x, branch, gate, post, eps):
    """y before it is rounded, the normed branch, 1 / its size, and what y's rounding in fp32 is bounded by.  gate and post: 1 or
    arrays that fit."""
    rb = 1.0 / np.sqrt((branch * branch).mean(-1, keepdims=True) + eps) if post is not None else np.ones_like(branch[..., :1])
    u = branch * rb
    added = gate * u * (1.0 if post is None else post)
    return x + added, u, rb, SMALL * (np.abs(x) + np.abs(added))


def gate_norm(y, kind, weight, bias, scale, shift, eps):
    """n, the normed rows, 1 / deviation, and bounds of the last two's roundings in fp32 (of h, of n)."""
    mean = y.mean(-1, keepdims=True) if kind == "layer" else 0.0
    r = 1.0 / np.sqrt(((y - mean) ** 2).mean(-1, keepdims=True) + eps)
    h = (y - mean) * r
    h_off = SMALL * (r * (np.abs(y) + np.abs(y).mean(-1, keepdims=True)) + np.abs(h)) if kind == "layer" else SMALL * np.abs(h)
    n = (h * weight + bias) * (1 + scale) + shift
    n_off = (h_off + SMALL * np.abs(h)) * np.abs(weight * (1 + scale)) + SMALL * (np.abs(bias * (1 + scale)) + np.abs(shift))
    return n, h, r, h_off, n_off


def gate_bwd(y, branch, gate, post, kind, weight, bias, scale, shift, eps, dy, dn):
    """All arrays [samples, tokens, width], or what broadcasts to it; dy or dn may be None.  {name: (value, bound in fp32)}, sums of
    parameters over the tokens of each sample."""
    zero = np.zeros_like(y)
    D, D_off = (zero, zero) if dy is None else (dy, SMALL * np.abs(dy))
    out = {}
    total = lambda t: t.sum(1)
    if dn is not None:
        _, h, r, h_off, _ = gate_norm(y, kind, weight, bias, scale, shift, eps)
        a = weight * (1 + scale)
        g, mean = dn * a, lambda t: t.mean(-1, keepdims=True)
        inner = g - h * mean(g * h) - (mean(g) if kind == "layer" else 0.0)
        size = np.abs(g) + np.abs(h) * mean(np.abs(g * h)) + (mean(np.abs(g)) if kind == "layer" else 0.0)
        D_off = D_off + r * (SMALL * size + h_off * mean(np.abs(g * h)) + np.abs(h) * mean(np.abs(g) * h_off))
        # (r is off by what the deviation is: that of h, relative)
        D_off = D_off + SMALL * r * size + r * np.abs(inner) * SMALL
        D = D + r * inner
        off = SMALL * np.abs(dn * h) + np.abs(dn) * h_off
        out["weight"] = total(dn * h * (1 + scale)), total(off * np.abs(1 + scale))
        out["bias"] = total(dn * (1 + scale)), SMALL * total(np.abs(dn * (1 + scale)))
        out["scale"] = total(dn * (h * weight + bias)), total(off * np.abs(weight) + SMALL * np.abs(dn * bias))
        out["shift"] = total(dn + zero), SMALL * total(np.abs(dn) + zero)
    out["x"] = D, D_off
    if branch is not None:
        _, u, rb, _ = gate_sum(zero, branch, gate, post, eps)
        w = 1.0 if post is None else post
        out["gate"] = total(D * u * w), total((SMALL * np.abs(D) + D_off) * np.abs(u * w))
        du, du_off = D * gate * w, (D_off + SMALL * np.abs(D)) * np.abs(gate * w)
        if post is None:
            out["branch"] = du, du_off
        else:
            out["branch_weight"] = total(D * u * gate), total((SMALL * np.abs(D) + D_off) * np.abs(u * gate))
            c = (du * u).mean(-1, keepdims=True)
            c_off = ((du_off + SMALL * np.abs(du)) * np.abs(u)).mean(-1, keepdims=True)
            out["branch"] = rb * (du - u * c), rb * (du_off + SMALL * (np.abs(du) + np.abs(u * c)) + np.abs(u) * c_off)
    return out


def clip_factor(arrays, max_norm, eps):
    norm = np.sqrt(sum((a.astype(np.float64) ** 2).sum() for a in arrays))
    if np.isinf(max_norm):
        return norm, 1.0
    f = max_norm / (norm + eps) if norm + eps != 0 else 1.0
    return norm, 1.0 if f >= 1 else f


# ------------------------------------------------------------------ attention over a window
def window_mask(Nq, Nk, length, start, left, right, sinks):
    """[Nq, Nk]: which pairs see each other (left, right: None for no limit)."""
    p, j = start + np.arange(Nq)[:, None], np.arange(Nk)[None]
    m = np.broadcast_to(j < length, (Nq, Nk)).copy()
    if right is not None:
        m &= j <= p + right
    if left is not None:
        m &= (j >= p - left) | (j < sinks)
    return m


def window(q, k, v, lengths, starts, left, right, sinks, scale, do=None):
    """fp64 arrays [B, H, N, d]; {name: (value, bound)}, and the log-sum-exp.  The bounds count what the kernels round, as
    block_ref.cross does: weights rounded to bf16 and divided by the sum of the rounded ones, U of each against their mean; dS
    rounded, and off by what P's log-sum-exp and D hold of the weights' rounding; results rounded; 2^-13 for what is fp32."""
    U, small = 2.0 ** -8, 2.0 ** -13
    B, Hq, Nq, d = q.shape
    Hk, Nk = k.shape[1:3]
    out = {n: (np.zeros(s), np.zeros(s)) for n, s in (("o", q.shape), ("dq", q.shape), ("dk", k.shape), ("dv", k.shape))}
    lse = np.full((B, Hq, Nq), -np.inf)
    for b in range(B):
        n = Nk if lengths is None else int(min(max(lengths[b], 0), Nk))
        seen = window_mask(Nq, Nk, n, Nk - Nq if starts is None else int(starts[b]), left, right, sinks)
        rows, keys = seen.any(1), seen.any(0)
        if not rows.any():
            continue
        m = seen[np.ix_(rows, keys)]
        for h in range(Hq):
            g = h // (Hq // Hk)
            qq, kk, vv = q[b, h][rows], k[b, g][keys], v[b, g][keys]
            s = np.where(m, scale * qq @ kk.T, -np.inf)
            top = s.max(-1, keepdims=True)
            e = np.exp(s - top)
            p = e / e.sum(-1, keepdims=True)
            lse[b, h, rows] = top[:, 0] + np.log(e.sum(-1))
            o, pv = p @ vv, p @ np.abs(vv)
            weights = U * (pv + np.abs(o)) + small * pv
            out["o"][0][b, h, rows], out["o"][1][b, h, rows] = o, weights + U * np.abs(o)
            if do is None:
                continue
            up = do[b, h][rows]
            dp = np.where(m, up @ vv.T, 0.0)
            D = (up * o).sum(-1, keepdims=True)
            ds = p * (dp - D)
            ds_bound = p * (np.abs(up) * (weights + 2.0 ** -15 * np.abs(o))).sum(-1, keepdims=True) + 3 * U * np.abs(ds) \
                + small * p * (np.abs(up) @ np.abs(vv).T + np.abs(D))
            out["dq"][0][b, h, rows], out["dq"][1][b, h, rows] = scale * ds @ kk, scale * ds_bound @ np.abs(kk)
            for name, value, bound in (("dk", scale * ds.T @ qq, scale * ds_bound.T @ np.abs(qq)),
                                       ("dv", p.T @ up, (2 * U + small) * p.T @ np.abs(up))):
                out[name][0][b, g, keys] += value
                out[name][1][b, g, keys] += bound
    for n in ("dq", "dk", "dv"):
        out[n] = (out[n][0], out[n][1] + U * np.abs(out[n][0]))
    return out, lse
