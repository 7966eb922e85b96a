"""Norm of the heads of q and k with the rotation by position, and its gradients, against the fp64 formulas.

Roundings counted in the bars (u = 2^-24 for one fp32 operation): the squares of a head are added by 16 products a lane and 3
exchanges, at most 19 u of their sum, half of it after the root; root, quotient and two products 4 u; a rotation adds two
products of the pair, 3 u of |a| + |b|.  That is below 2^-19 of |a| + |b|; the backward pass has two such sums, 2^-18 of the
magnitudes that the reference adds up.  Results in bf16 are then rounded once, 2^-8 of the result."""
import numpy as np
import pytest
import torch

import block_ref as ref
import paper_2602_13515_amd as spa2
from gpu_util import dev

pytestmark = pytest.mark.gpu
EPS = 1e-6


def f64(t):
    return t.detach().double().cpu().numpy()


def _heads(rng, B, H, N, d, dtype, layout):
    """[B, H, N, d] in memory: "bnhd" tokens outside, "bhnd" heads outside, "fused" a slice of wider rows, "shared" one head
    repeated."""
    x = torch.from_numpy(rng.standard_normal((B, N, H, d)) * np.exp(rng.uniform(-3, 3, (B, N, H, 1)))).to(dtype).to(dev())
    if layout == "bnhd":
        return x.permute(0, 2, 1, 3)
    if layout == "bhnd":
        return x.permute(0, 2, 1, 3).contiguous()
    if layout == "fused":
        wide = torch.full((B, N, H + 3, d), float("nan"), dtype=dtype, device=dev())
        wide[:, :, 1:H + 1] = x
        return wide[:, :, 1:H + 1].permute(0, 2, 1, 3)
    return x[:, :, :1].permute(0, 2, 1, 3).expand(B, H, N, d)


def _case(rng, B, Hq, Hk, N, d, dtype, layout, rot, positions, weights):
    q, k = _heads(rng, B, Hq, N, d, dtype, layout), _heads(rng, B, Hk, N, d, dtype, layout)
    w = [None, None]
    if weights:
        w = [torch.from_numpy(1 + 0.3 * rng.standard_normal(d)).to(weights).to(dev()) for _ in range(2)]
    cos = sin = pos = None
    rows = np.broadcast_to(np.arange(N), (B, N))
    if rot:
        P = N if positions is None else N + 57
        angle = rng.uniform(-50, 50, (P, rot // 2))
        cos, sin = (torch.from_numpy(x).float().to(dev()) for x in (np.cos(angle), np.sin(angle)))
        if positions == "sample":
            rows = rng.integers(0, P, (B, N))
            pos = torch.from_numpy(rows).to(torch.int32).to(dev())
        elif positions == "shared":
            rows = np.broadcast_to(rng.integers(0, P, (1, N)), (B, N))
            pos = torch.from_numpy(rows[0].copy()).to(torch.int64).to(dev())
        elif positions == "outside":
            far = rng.integers(-2 ** 40, 2 ** 40, (B, N))
            rows = np.clip(far, 0, P - 1)
            pos = torch.from_numpy(far).to(dev())
    return q, k, w, cos, sin, pos, rows


def _check(x, w, cos, sin, rows, interleaved, y, up=None, dx=None, dw=None):
    """One of q and k; x, y, ... tensors."""
    c = s = None
    if cos is not None:
        c, s = f64(cos)[rows][:, None], f64(sin)[rows][:, None]
    weight = np.ones(x.shape[-1]) if w is None else f64(w)
    want, n = ref.norm_rotate(f64(x), weight, c, s, EPS, interleaved)
    size = np.abs(n) if c is None else ref.pair_sum(n, c.shape[-1], interleaved)
    assert y.dtype == torch.bfloat16
    err = np.abs(f64(y) - want)
    assert (err <= 2.0 ** -8 * np.abs(want) + 2.0 ** -19 * size).all(), err.max()
    if up is None:
        return
    wdx, wdw, dx_size, dw_size = ref.norm_rotate_bwd(f64(x), weight, c, s, EPS, interleaved, f64(up))
    one = 2.0 ** -8 if x.dtype == torch.bfloat16 else 2.0 ** -24
    assert dx.dtype == x.dtype and dx.shape == x.shape
    err = np.abs(f64(dx) - wdx)
    assert (err <= one * np.abs(wdx) + 2.0 ** -18 * dx_size).all(), (err / dx_size).max()
    if w is not None:
        # up to one addition a row on top of a term's own roundings, then the rounding to the weight's type
        one = 2.0 ** -8 if w.dtype == torch.bfloat16 else 2.0 ** -24
        terms = x.numel() // x.shape[-1]
        assert dw.dtype == w.dtype
        assert (np.abs(f64(dw) - wdw) <= one * np.abs(wdw) + (terms + 64) * 2.0 ** -24 * dw_size).all()


CASES = [
    # B, Hq, Hk, N, d, dtype, layout, rot, interleaved, positions, weights
    (1, 1, 1, 1, 64, torch.bfloat16, "bhnd", 64, False, None, torch.float32),
    (1, 3, 1, 1, 128, torch.bfloat16, "bnhd", 128, True, "sample", torch.float32),
    (16, 40, 8, 1, 128, torch.bfloat16, "bnhd", 128, False, "sample", torch.float32),
    (3, 5, 5, 1, 64, torch.float32, "fused", 32, True, "shared", torch.bfloat16),
    (2, 6, 2, 33, 64, torch.bfloat16, "fused", 16, False, "sample", torch.bfloat16),
    (2, 6, 2, 33, 128, torch.float32, "bhnd", 0, False, None, torch.float32),
    (2, 2, 1, 129, 128, torch.bfloat16, "shared", 64, True, "outside", torch.float32),
    (1, 7, 3, 200, 128, torch.float32, "bnhd", 112, False, None, None),
    (3, 4, 4, 77, 64, torch.bfloat16, "bnhd", 48, True, "shared", None),
    (1, 2, 2, 5003, 64, torch.bfloat16, "bnhd", 64, True, None, torch.float32),
    (4, 12, 12, 1281, 128, torch.float32, "fused", 128, True, None, torch.float32),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{c[0]}x{c[1]},{c[2]}x{c[3]}x{c[4]}-{str(c[5])[6:]}-{c[6]}-{c[7]}")
def test_results_and_gradients(case):
    B, Hq, Hk, N, d, dtype, layout, rot, interleaved, positions, weights = case
    print("case", case, flush=True)
    rng = np.random.default_rng(N + d + rot)
    q, k, w, cos, sin, pos, rows = _case(rng, B, Hq, Hk, N, d, dtype, layout, rot, positions, weights)
    with torch.no_grad():
        plain = spa2.qk_norm_rotate(q, k, w[0], w[1], cos, sin, pos, EPS, interleaved)
    leaves = [t.detach().requires_grad_(True) for t in (q, k, *[x for x in w if x is not None])]
    lw = leaves[2:] or [None, None]
    out = spa2.qk_norm_rotate(leaves[0], leaves[1], lw[0], lw[1], cos, sin, pos, EPS, interleaved)
    for y, z in zip(out, plain):
        assert torch.equal(y, z)
    up = [torch.from_numpy(rng.standard_normal(tuple(t.shape))).bfloat16().to(dev()) for t in out]
    grads = torch.autograd.grad(out, leaves, up)
    for z, x in enumerate((q, k)):
        _check(x, w[z], cos, sin, rows, interleaved, out[z], up[z], grads[z], grads[2 + z] if w[z] is not None else None)
    again = torch.autograd.grad(spa2.qk_norm_rotate(leaves[0], leaves[1], lw[0], lw[1], cos, sin, pos, EPS, interleaved), leaves, up)
    for a, b in zip(grads, again):
        assert torch.equal(a, b)                  # sums in a fixed order


def test_buffers_next_to_the_results_stay_untouched():
    from gpu_util import Guarded
    g, rng = Guarded(), np.random.default_rng(5)
    q, k = (_heads(rng, 2, h, 37, 64, torch.bfloat16, "bnhd") for h in (3, 2))
    outs = [g.alloc(t.shape, torch.bfloat16, dev(), float("nan")) for t in (q, k)]
    spa2.spa2_norm_rotate(q, k, None, None, None, None, None, EPS, False, *outs)
    dx = [g.alloc(t.shape, torch.bfloat16, dev(), float("nan")) for t in (q, k)]
    dw = [g.alloc((64,), torch.float32, dev(), float("nan")) for _ in range(2)]
    one = torch.ones(64, device=dev())
    ws = g.alloc((spa2.spa2_norm_rotate_bwd_workspace_bytes(q, k),), torch.uint8, dev(), 0)
    up = [torch.randn_like(t.contiguous()) for t in (q, k)]
    spa2.spa2_norm_rotate_bwd(q, k, one, one, None, None, None, *up, EPS, False, *dx, *dw, ws)
    torch.cuda.synchronize()
    g.check("norm and rotate")
    for t in (*outs, *dx, *dw):
        assert torch.isfinite(t).all()


def test_zero_heads_and_heads_with_infinities():
    """A head of zeros stays zero and has finite gradients; one that holds an infinity is lost, and only that one."""
    q = torch.randn(1, 2, 40, 128, device=dev()).bfloat16()
    q[0, 0, 3] = 0
    q[0, 1, 7, 5] = float("inf")
    q[0, 1, 9, 5] = float("nan")
    leaf = q.requires_grad_(True)
    cos, sin = spa2.rotary_table(40, 128, device=dev())
    y, _ = spa2.qk_norm_rotate(leaf, q.detach(), None, None, cos, sin)
    bad = torch.zeros(1, 2, 40, dtype=torch.bool, device=dev())
    bad[0, 1, 7] = bad[0, 1, 9] = True
    assert torch.equal(y[0, 0, 3], torch.zeros_like(y[0, 0, 3]))
    assert torch.isfinite(y[~bad]).all() and not torch.isfinite(y[bad]).all(-1).any()
    (dx,) = torch.autograd.grad(y, leaf, torch.ones_like(y))
    assert torch.isfinite(dx[~bad]).all()


@pytest.mark.parametrize("which", ["q", "k"])
def test_one_of_the_results_is_enough(which):
    q, k = torch.randn(1, 2, 9, 64, device=dev(), requires_grad=True), torch.randn(1, 1, 9, 64, device=dev(), requires_grad=True)
    out = spa2.qk_norm_rotate(q, k)
    a = torch.autograd.grad(out["qk".index(which)].float().square().sum() / 2, (q, k))
    other = a[1 - "qk".index(which)]
    assert torch.equal(other, torch.zeros_like(other)) and float(a["qk".index(which)].abs().max()) > 0


def test_refusals():
    q, k = torch.randn(2, 4, 10, 64, device=dev()), torch.randn(2, 2, 10, 64, device=dev())
    cos, sin = spa2.rotary_table(10, 64, device=dev())
    f = spa2.qk_norm_rotate
    for bad in (lambda: f(q.half(), k.half()), lambda: f(q, k.bfloat16()), lambda: f(q, k[:, :, :9]), lambda: f(q, k[:1]),
                lambda: f(q[0], k[0]), lambda: f(q.transpose(2, 3), k.transpose(2, 3)), lambda: f(q, k, cos[0]),
                lambda: f(q, k, None, None, cos), lambda: f(q, k, None, None, cos.double(), sin.double()),
                lambda: f(q, k, None, None, cos, sin[:9]), lambda: f(q, k, None, None, cos[:9], sin[:9]),
                lambda: f(q, k, None, None, cos[:, ::2], sin[:, ::2]),
                lambda: f(q, k, positions=torch.zeros(10, dtype=torch.int32, device=dev())),
                lambda: f(q, k, None, None, cos, sin, torch.zeros(9, dtype=torch.int32, device=dev())),
                lambda: f(q, k, None, None, cos, sin, torch.zeros(10, device=dev())),
                lambda: f(q, k, None, None, cos, sin, torch.zeros(10, dtype=torch.int32)),
                lambda: f(q, k.cpu())):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: f(q[..., :32], k[..., :32]), lambda: f(q, k, eps=0.0), lambda: f(q, k, None, None, *(t[:, :12].contiguous() for t in (cos, sin))),
                lambda: f(torch.randn(2 * 4 * 10 * 64 + 1, device=dev())[1:].view(2, 4, 10, 64), k)):
        with pytest.raises(spa2.Spa2Error):
            bad()
    with pytest.raises(RuntimeError):
        torch.func.vmap(lambda x: f(x, x)[0])(torch.randn(3, 1, 2, 4, 64, device=dev()))


def test_second_derivative_is_refused():
    q = torch.randn(1, 1, 8, 64, device=dev(), requires_grad=True)
    y, _ = spa2.qk_norm_rotate(q, q.detach())
    (dx,) = torch.autograd.grad(y, q, torch.ones_like(y), create_graph=True)
    with pytest.raises(RuntimeError, match="second derivative"):
        dx.sum().backward()


def test_another_stream_and_a_captured_graph():
    rng = np.random.default_rng(8)
    q, k, w, cos, sin, pos, _ = _case(rng, 2, 3, 1, 150, 64, torch.bfloat16, "bnhd", 64, "sample", torch.float32)
    leaves = [t.detach().requires_grad_(True) for t in (q, k, *w)]
    up = [torch.randn_like(t) for t in spa2.qk_norm_rotate(*(t.detach() for t in leaves), cos, sin, pos)]

    def step():
        out = spa2.qk_norm_rotate(*leaves, cos, sin, pos)
        return [t.detach() for t in out] + list(torch.autograd.grad(out, leaves, up))
    want = [t.clone() for t in step()]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = step()
    side.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for change in range(3):
        with torch.no_grad():
            leaves[0].mul_(1.5), leaves[2].add_(0.1)
        for t in held:
            t.zero_()
        want = [t.clone() for t in step()]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(held, want):
            assert torch.equal(a, b), change


@pytest.mark.parametrize("grad", [False, True])
def test_inputs_with_tangents_are_refused(grad):
    import torch.autograd.forward_ad as fwad
    x = torch.randn(1, 2, 8, 64, device=dev())
    f = lambda t: spa2.qk_norm_rotate(t, x)[0]
    with torch.set_grad_enabled(grad), fwad.dual_level():
        want = f(x)
        with pytest.raises(RuntimeError):
            f(fwad.make_dual(x, torch.ones_like(x)))
    assert torch.equal(f(x), want)
