"""The operators around the block-sparse attention of a transformer block, as cases that can be timed and compared.

* ``norm``   ``qk_norm_rotate``: the norm of every head of q and k and the rotation by position, in front of the attention;
* ``attn``   ``cross_attention``: attention to another sequence (or to a cache) whose samples have lengths of their own;
* ``drop``   ``dropout_add``: dropout of a branch and the sum with the residual stream, behind the attention.

A case with ``train`` is a forward and a backward pass with the upstream gradients given, otherwise a forward pass that
keeps nothing.  With ``own`` false ``run`` evaluates the formulas with elementary torch operations in 32 bits (64 for the
sums over all tokens), rounded once at the end; with ``own`` true it calls the library's operators.
"""
from __future__ import annotations

import math

import torch

own = False
DEVICE = "cuda"


def _norm(name, train, B, N, Hq, Hk, d, rot, interleaved, dtype, positions, table):
    """positions: "none" (token n uses row n of the table), "sample" (every sample starts at a place of its own).
    table: rows of the tables of cosines and sines."""
    return {"name": name, "op": "norm", "train": train, "B": B, "N": N, "Hq": Hq, "Hk": Hk, "d": d, "rot": rot,
            "interleaved": interleaved, "dtype": dtype, "positions": positions, "table": table}


def _attn(name, train, B, Hq, Hk, Nq, Nk, d, lengths):
    """lengths: "full", or "ragged" (samples of unlike length, one of them empty if there are four or more)."""
    return {"name": name, "op": "attn", "train": train, "B": B, "Hq": Hq, "Hk": Hk, "Nq": Nq, "Nk": Nk, "d": d,
            "lengths": lengths}


def _drop(name, train, rows, width, x_dtype, r_dtype, p):
    """r_dtype: type of the residual stream, or "none"."""
    return {"name": name, "op": "drop", "train": train, "rows": rows, "width": width, "x_dtype": x_dtype,
            "r_dtype": r_dtype, "p": p}


def listed():
    return [
        # one new token of sixteen sequences, at places of their own in a long table: latency
        _norm("norm-token", False, 16, 1, 40, 8, 128, 128, False, "bfloat16", "sample", 32760),
        # a batch of short sequences that end just past a block, shared key heads, half the channels rotated
        _norm("norm-train-ragged", True, 4, 1281, 6, 2, 64, 32, False, "bfloat16", "sample", 4096),
        # the layer of a 480p video in training, from the fp32 output of the projection
        _norm("norm-train-480p", True, 1, 32760, 12, 12, 128, 128, True, "float32", "none", 32760),
        # the layer of a 720p video in sampling
        _norm("norm-720p", False, 1, 75600, 40, 40, 128, 128, True, "bfloat16", "none", 75600),
        # one new token against long caches of unlike length, key heads shared by five query heads
        _attn("attn-token", False, 8, 40, 8, 1, 32760, 128, "ragged"),
        # a batch of short sequences against short prompts, one of them empty
        _attn("attn-train-ragged", True, 4, 6, 2, 1281, 77, 64, "ragged"),
        # a 480p video's tokens against a prompt, training
        _attn("attn-train-480p", True, 1, 12, 12, 32760, 512, 128, "full"),
        # a 720p video's tokens against a prompt, sampling
        _attn("attn-720p", False, 1, 40, 40, 75600, 512, 128, "full"),
        # a branch of a small block: a thousand tokens, latency
        _drop("drop-short", False, 1000, 256, "bfloat16", "bfloat16", 0.1),
        # an odd number of elements, no residual
        _drop("drop-train-odd", True, 5123, 1281, "bfloat16", "none", 0.25),
        # 480p video: bf16 branch into an fp32 residual stream
        _drop("drop-train-480p", True, 32760, 1536, "bfloat16", "float32", 0.1),
        # 720p video, bf16 throughout
        _drop("drop-train-720p", True, 75600, 5120, "bfloat16", "bfloat16", 0.1),
    ]


def _log(rng, low, high):
    return int(round(2.0 ** rng.uniform(math.log2(low), math.log2(high))))


def draw(rng):
    case = _drawn(rng)
    del case["name"]
    return case


def _drawn(rng):
    op = rng.choice(["norm", "attn", "drop"])
    train = rng.random() < 0.5
    if op == "drop":
        rows, width = _log(rng, 1, 37800), _log(rng, 63, 5120)
        x_dtype = rng.choice(["bfloat16", "bfloat16", "float32"])
        r_dtype = rng.choice(["none", "float32"] if x_dtype == "float32" else ["none", "bfloat16", "float32"])
        return _drop("", train, rows, width, x_dtype, r_dtype, rng.choice([0.0, 0.05, 0.1, 0.3, 0.5]))
    Hk, group = rng.choice([1, 2, 3, 6, 8, 12]), rng.choice([1, 1, 2, 3, 5])
    B, d = rng.choice([1, 1, 2, 3, 4, 16]), rng.choice([64, 128])
    if op == "norm":
        N = max(1, min(_log(rng, 1, 75600), 75600 * 40 * 64 // (B * Hk * (group + 1) * d)))
        rot = rng.choice([d, d, d // 2, 0])
        positions = rng.choice(["none", "sample"])
        return _norm("", train, B, N, Hk * group, Hk, d, rot, rng.random() < 0.5,
                     rng.choice(["bfloat16", "bfloat16", "float32"]), positions, N + 4096)
    Nq = rng.choice([1, _log(rng, 1, 75600)])
    Nk = _log(rng, 1, 65536)
    limit = 0.4 * 40.0 * 75600 * 512 * 128 / (3.5 if train else 1.0)
    Nq = max(1, min(Nq, int(limit / (B * Hk * group * Nk * d))))
    return _attn("", train, B, Hk * group, Hk, Nq, Nk, d, rng.choice(["full", "ragged"]))


# ------------------------------------------------------------------ inputs
def _dtype(name):
    return None if name == "none" else getattr(torch, name)


def _lengths(case, g=None):
    """Lengths of the samples: all of the keys, or a fixed set of shares of them, dealt to the samples by the seed."""
    B, Nk = case["B"], case["Nk"]
    if case["lengths"] == "full":
        return None
    set_ = [max(1, Nk - (Nk * b) // B - (b & 1)) for b in range(B)]
    if B >= 4:
        set_[-1] = 0
    if g is None:
        return set_
    order = torch.randperm(B, generator=g, device=DEVICE)
    return torch.tensor(set_, dtype=torch.int32, device=DEVICE)[order]


def _tables(case):
    """Cosines and sines of position times frequency, taken in 64 bits."""
    if not case["rot"]:
        return None, None
    freq = 10000.0 ** (-torch.arange(0, case["rot"], 2, dtype=torch.float64, device=DEVICE) / case["rot"])
    angle = torch.arange(case["table"], dtype=torch.float64, device=DEVICE)[:, None] * freq
    return angle.cos().float(), angle.sin().float()


def _inputs(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)

    def randn(*shape):
        return torch.randn(shape, generator=g, device=DEVICE)

    s = {"case": case}
    if case["op"] == "norm":
        B, N, Hq, Hk, d = (case[x] for x in ("B", "N", "Hq", "Hk", "d"))
        dtype = _dtype(case["dtype"])
        # one projection's output: query, key and value heads of a token next to each other
        qkv = (randn(B, N, Hq + 2 * Hk, d) * (0.5 + 2 * torch.rand((B, N, 1, 1), generator=g, device=DEVICE))).to(dtype)
        s["q"], s["k"] = qkv[:, :, :Hq].permute(0, 2, 1, 3), qkv[:, :, Hq:Hq + Hk].permute(0, 2, 1, 3)
        s["wq"], s["wk"] = 1.0 + 0.2 * randn(d), 1.0 + 0.2 * randn(d)
        s["cos"], s["sin"] = _tables(case)
        s["positions"] = None
        if case["rot"] and case["positions"] == "sample":
            start = torch.randint(0, case["table"] - N + 1, (B, 1), generator=g, device=DEVICE)
            s["positions"] = (start + torch.arange(N, device=DEVICE)).to(torch.int32)
        leaves = ("q", "k", "wq", "wk")
        if case["train"]:
            s["dq"] = randn(B, N, Hq, d).to(torch.bfloat16).permute(0, 2, 1, 3)
            s["dk"] = randn(B, N, Hk, d).to(torch.bfloat16).permute(0, 2, 1, 3)
    elif case["op"] == "attn":
        B, Hq, Hk, Nq, Nk, d = (case[x] for x in ("B", "Hq", "Hk", "Nq", "Nk", "d"))
        s["q"] = (1.5 * randn(B, Nq, Hq, d)).to(torch.bfloat16).permute(0, 2, 1, 3)
        kv = randn(B, Nk, 2 * Hk, d).to(torch.bfloat16)
        s["k"], s["v"] = kv[:, :, :Hk].permute(0, 2, 1, 3), kv[:, :, Hk:].permute(0, 2, 1, 3)
        s["lengths"] = _lengths(case, g)
        leaves = ("q", "k", "v")
        if case["train"]:
            s["do"] = randn(B, Nq, Hq, d).to(torch.bfloat16).permute(0, 2, 1, 3)
    else:
        shape = (case["rows"], case["width"])
        s["x"] = randn(*shape).to(_dtype(case["x_dtype"]))
        r_dtype = _dtype(case["r_dtype"])
        s["r"] = None if r_dtype is None else (2 * randn(*shape)).to(r_dtype)
        s["seed"], s["offset"] = (seed * 0x9E3779B97F4A7C15 + 12345) % 2 ** 63, seed % 1000 + 2 ** 33
        leaves = ("x",) if s["r"] is None else ("x", "r")
        if case["train"]:
            s["dy"] = randn(*shape).to(r_dtype or _dtype(case["x_dtype"]))
    s["leaves"] = leaves
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        import paper_2602_13515_amd as spa2
        s["spa2"] = spa2
        if case["train"]:
            for name in s["leaves"]:
                s[name] = s[name].detach().requires_grad_(True)
    return s


# ------------------------------------------------------------------ the plain forms
def _rotate(x, cos, sin, interleaved, back=False):
    """Pairs of the first channels turned by their angle (by minus the angle: the transposed matrix)."""
    rot = 2 * cos.shape[-1]
    if back:
        sin = -sin
    if interleaved:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack((a * cos - b * sin, b * cos + a * sin), dim=-1).flatten(-2)
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        turned = torch.cat((a * cos - b * sin, b * cos + a * sin), dim=-1)
    return torch.cat((turned, x[..., rot:]), dim=-1)


def _plain_norm(s):
    case, eps = s["case"], 1e-6
    cos = sin = None
    if s["cos"] is not None:
        cos, sin = s["cos"][:case["N"]], s["sin"][:case["N"]]
        if s["positions"] is not None:
            cos, sin = s["cos"][s["positions"].long()][:, None], s["sin"][s["positions"].long()][:, None]
    outs, grads, weight_grads = [], [], []
    for x, w, up in (("q", "wq", "dq"), ("k", "wk", "dk")):
        xf, weight = s[x].float(), s[w]
        r = (xf.square().mean(-1, keepdim=True) + eps).rsqrt()
        n = xf * r
        y = n * weight
        outs.append((y if cos is None else _rotate(y, cos, sin, case["interleaved"])).to(torch.bfloat16))
        if case["train"]:
            dn = s[up].float()
            if cos is not None:
                dn = _rotate(dn, cos, sin, case["interleaved"], back=True)
            weight_grads.append((dn * n).sum((0, 1, 2), dtype=torch.float64).float())
            gr = dn * weight
            grads.append((r * (gr - n * (gr * n).mean(-1, keepdim=True))).to(s[x].dtype))
    return outs + grads + weight_grads


def _plain_attn(s):
    case = s["case"]
    B, Hq, Hk, Nq, Nk, d = (case[x] for x in ("B", "Hq", "Hk", "Nq", "Nk", "d"))
    scale, group = 1.0 / math.sqrt(d), Hq // Hk
    outs = [torch.empty_like(s["q"])]
    if case["train"]:
        outs += [torch.empty_like(s["q"]), torch.empty((B, Hk, Nk, d), dtype=torch.bfloat16, device=DEVICE),
                 torch.empty((B, Hk, Nk, d), dtype=torch.bfloat16, device=DEVICE)]
    seen = torch.arange(Nk, device=DEVICE)
    for b in range(B):
        # [Hk, group * Nq, d]: the query heads of a key head as further rows
        q = s["q"][b].float().reshape(Hk, group * Nq, d)
        k, v = s["k"][b].float().contiguous(), s["v"][b].float().contiguous()
        score = scale * torch.matmul(q, k.transpose(1, 2).contiguous())
        if s["lengths"] is not None:
            score = torch.where(seen < s["lengths"][b], score, -math.inf)
        top = score.amax(-1, keepdim=True)
        top = torch.where(top == -math.inf, 0.0, top)
        p = score.sub_(top).exp_()
        total = p.sum(-1, keepdim=True)
        p.div_(torch.where(total == 0, 1.0, total))
        o = torch.matmul(p, v)
        outs[0][b] = o.reshape(Hq, Nq, d).to(torch.bfloat16)
        if case["train"]:
            do = s["do"][b].float().reshape(Hk, group * Nq, d)
            outs[3][b] = torch.matmul(p.transpose(1, 2).contiguous(), do).to(torch.bfloat16)
            ds = torch.matmul(do, v.transpose(1, 2).contiguous())
            ds = ds.sub_((do * o).sum(-1, keepdim=True)).mul_(p)
            outs[1][b] = (scale * torch.matmul(ds, k)).reshape(Hq, Nq, d).to(torch.bfloat16)
            outs[2][b] = (scale * torch.matmul(ds.transpose(1, 2).contiguous(), q)).to(torch.bfloat16)
    return outs


def _philox(counters, offset, seed):
    """Philox4x32-10 (Salmon et al., 2011): key = seed, counter = (counters, offset), both of 64 bits; four words of 32
    bits for each counter, as 64-bit integers."""
    low = 0xFFFFFFFF
    c = [counters & low, counters >> 32, torch.full_like(counters, offset & low), torch.full_like(counters, offset >> 32)]
    k0, k1 = seed & low, (seed >> 32) & low
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [((b >> 32) & low) ^ c[1] ^ k0, b & low, ((a >> 32) & low) ^ c[3] ^ k1, a & low]
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return c


def _threshold(p):
    return int(math.floor(p * 65536.0 + 0.5))


def _plain_drop(s):
    """Element e is kept where its 16 random bits, half e % 2 of word (e % 8) / 2 of counter e / 8, reach the threshold."""
    case, x = s["case"], s["x"]
    n, cut = x.numel(), _threshold(case["p"])
    words = _philox(torch.arange((n + 7) // 8, device=DEVICE), s["offset"], s["seed"])
    bits = torch.stack([h for w in words for h in (w & 0xFFFF, w >> 16)], dim=-1).flatten()[:n]
    keep = (bits >= cut).reshape(x.shape)
    factor = 65536.0 / (65536 - cut)
    y = torch.where(keep, x.float() * factor, 0.0)
    if s["r"] is not None:
        y = s["r"].float() + y
    outs = [y.to(x.dtype if s["r"] is None else s["r"].dtype)]
    if case["train"]:
        outs.append(torch.where(keep, s["dy"].float() * factor, 0.0).to(x.dtype))
        if s["r"] is not None:
            outs.append(s["dy"])
    return outs


def run(state):
    s, case = state, state["case"]
    if not own:
        return {"norm": _plain_norm, "attn": _plain_attn, "drop": _plain_drop}[case["op"]](s)
    spa2, train = s["spa2"], case["train"]
    with torch.set_grad_enabled(train):
        if case["op"] == "norm":
            outs = spa2.qk_norm_rotate(s["q"], s["k"], s["wq"], s["wk"], s["cos"], s["sin"], positions=s["positions"],
                                       interleaved=case["interleaved"])
            ups = (s["dq"], s["dk"]) if train else None
        elif case["op"] == "attn":
            outs = (spa2.cross_attention(s["q"], s["k"], s["v"], lengths=s["lengths"]),)
            ups = (s["do"],) if train else None
        else:
            outs = (spa2.dropout_add(s["x"], s["r"], case["p"], s["seed"], s["offset"]),)
            ups = (s["dy"],) if train else None
    if not train:
        return list(outs)
    grads = torch.autograd.grad(outs, [s[name] for name in s["leaves"]], ups)
    return [o.detach() for o in outs] + list(grads)


# ------------------------------------------------------------------ in 64 bits, from the definitions
def _exact_norm(s):
    case = s["case"]
    N, d, rot = case["N"], case["d"], case["rot"]
    rows = (torch.arange(N, device=DEVICE)[None].expand(case["B"], N) if s["positions"] is None
            else s["positions"].long())
    first = second = None
    if rot:
        half = torch.arange(rot // 2, device=DEVICE)
        first, second = (2 * half, 2 * half + 1) if case["interleaved"] else (half, half + rot // 2)
        c, t = s["cos"].double()[rows][:, None], s["sin"].double()[rows][:, None]
    outs, grads, weight_grads = [], [], []
    for x, w, up in (("q", "wq", "dq"), ("k", "wk", "dk")):
        xd, wd = s[x].double(), s[w].double()
        root = torch.sqrt((xd * xd).sum(-1, keepdim=True) / d + 1e-6)
        unit = xd / root
        y = unit * wd
        if rot:
            z = y.clone()
            z[..., first] = c * y[..., first] - t * y[..., second]
            z[..., second] = t * y[..., first] + c * y[..., second]
            y = z
        outs.append(y)
        if case["train"]:
            up_d = s[up].double()
            dy = up_d.clone()
            if rot:
                dy[..., first] = c * up_d[..., first] + t * up_d[..., second]
                dy[..., second] = c * up_d[..., second] - t * up_d[..., first]
            weight_grads.append((dy * unit).sum((0, 1, 2)))
            inner = (dy * wd * xd).sum(-1, keepdim=True)
            grads.append(dy * wd / root - xd * inner / (d * root ** 3))
    return outs + grads + weight_grads


def _exact_attn(s):
    case = s["case"]
    B, Hq, Hk, Nq, Nk, d = (case[x] for x in ("B", "Hq", "Hk", "Nq", "Nk", "d"))
    o = torch.zeros((B, Hq, Nq, d), dtype=torch.float64, device=DEVICE)
    dq, dk = torch.zeros_like(o), torch.zeros((B, Hk, Nk, d), dtype=torch.float64, device=DEVICE)
    dv = torch.zeros_like(dk)
    for b in range(B):
        n = Nk if s["lengths"] is None else int(s["lengths"][b])
        if n == 0:
            continue
        for h in range(Hq):
            q, k, v = s["q"][b, h].double(), s["k"][b, h // (Hq // Hk), :n].double(), s["v"][b, h // (Hq // Hk), :n].double()
            p = torch.softmax(q @ k.T / math.sqrt(d), dim=-1)
            o[b, h] = p @ v
            if case["train"]:
                do = s["do"][b, h].double()
                dp = do @ v.T
                ds = p * (dp - (dp * p).sum(-1, keepdim=True)) / math.sqrt(d)
                dq[b, h] = ds @ k
                dk[b, h // (Hq // Hk), :n] += ds.T @ q
                dv[b, h // (Hq // Hk), :n] += p.T @ do
    return [o, dq, dk, dv] if case["train"] else [o]


def _exact_drop(s):
    case, x = s["case"], s["x"]
    n, cut, low = x.numel(), _threshold(case["p"]), 0xFFFFFFFF

    def product(a, m):
        """Low and high 32 bits of a * m, by halves of 16 bits."""
        a0, a1, m0, m1 = a & 0xFFFF, a >> 16, m & 0xFFFF, m >> 16
        middle = a1 * m0 + ((a0 * m0) >> 16)
        crossed = a0 * m1 + (middle & 0xFFFF)
        return ((crossed << 16) & low) | ((a0 * m0) & 0xFFFF), a1 * m1 + (middle >> 16) + (crossed >> 16)

    at = torch.arange((n + 7) // 8, device=DEVICE)
    c0, c1 = at & low, at >> 32
    c2, c3 = torch.full_like(at, s["offset"] & low), torch.full_like(at, s["offset"] >> 32)
    for r in range(10):
        k0, k1 = ((s["seed"] & low) + r * 0x9E3779B9) & low, ((s["seed"] >> 32) + r * 0xBB67AE85) & low
        lo0, hi0 = product(c0, 0xD2511F53)
        lo1, hi1 = product(c2, 0xCD9E8D57)
        c0, c1, c2, c3 = hi1 ^ c1 ^ k0, lo1, hi0 ^ c3 ^ k1, lo0
    kept = torch.empty((at.numel(), 8), dtype=torch.bool, device=DEVICE)
    for i, word in enumerate((c0, c1, c2, c3)):
        kept[:, 2 * i], kept[:, 2 * i + 1] = (word & 0xFFFF) >= cut, (word >> 16) >= cut
    kept = kept.reshape(-1)[:n].reshape(x.shape).double()
    y = x.double() * kept / (1.0 - cut / 65536.0)
    outs = [y if s["r"] is None else s["r"].double() + y]
    if case["train"]:
        outs.append(s["dy"].double() * kept / (1.0 - cut / 65536.0))
        if s["r"] is not None:
            outs.append(s["dy"].double())
    return outs


def exact(case, seed):
    s = _inputs(case, seed)
    return {"norm": _exact_norm, "attn": _exact_attn, "drop": _exact_drop}[case["op"]](s)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    train = case["train"]
    if case["op"] == "norm":
        x = float(case["B"] * case["N"] * (case["Hq"] + case["Hk"]) * case["d"])
        size = 2 if case["dtype"] == "bfloat16" else 4
        tables = 8.0 * (case["rot"] // 2) * min(case["table"], case["B"] * case["N"])
        if train:        # x, dy in; y, dx out (x serves both passes)
            return {"bytes": x * (2 * size + 4) + tables, "flops": 20.0 * x}
        return {"bytes": x * (size + 2) + tables, "flops": 6.0 * x}
    if case["op"] == "attn":
        lengths = _lengths(case) or [case["Nk"]] * case["B"]
        rows, keys = float(case["B"] * case["Hq"] * case["Nq"]), float(sum(lengths) * case["Hk"])
        pairs = float(sum(lengths)) * case["Hq"] * case["Nq"]
        d = case["d"]
        if train:        # q, do, k, v in; o, dq, dk, dv out
            return {"bytes": 2.0 * d * (4 * rows + 2 * keys + 2.0 * case["B"] * case["Hk"] * case["Nk"]),
                    "flops": 14.0 * pairs * d}
        return {"bytes": 2.0 * d * (2 * rows + 2 * keys), "flops": 4.0 * pairs * d}
    n = float(case["rows"] * case["width"])
    x = 2 if case["x_dtype"] == "bfloat16" else 4
    r = {"none": 0, "bfloat16": 2, "float32": 4}[case["r_dtype"]]
    out = r or x
    if train:            # x, residual, dy in; y, dx out
        return {"bytes": n * (x + r + out + out + x), "flops": 4.0 * n}
    return {"bytes": n * (x + r + out), "flops": 2.0 * n}
