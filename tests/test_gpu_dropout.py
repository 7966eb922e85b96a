"""Dropout with the residual sum against the generator in 64-bit integers: the mask exactly, values to one rounding (the
product with the factor, itself rounded, and the sum: 2 * 2^-24 of the product's magnitude, 2^-24 or 2^-8 of the result)."""
import numpy as np
import pytest
import torch

import block_ref as ref
import paper_2602_13515_amd as spa2
from gpu_util import dev

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32


def f64(t):
    return t.detach().double().cpu().numpy()


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


@pytest.mark.parametrize("x_dtype,r_dtype", [(BF, None), (BF, BF), (BF, F), (F, None), (F, F)], ids=str)
@pytest.mark.parametrize("n", [1, 7, 8, 9, 2047, 2048, 100_003, 5_000_005])
def test_values_and_gradients(n, x_dtype, r_dtype):
    p, seed, offset = (0.1, 0.5, 0.9)[n % 3], 2 ** 63 + 12345 * n, 2 ** 40 + n
    print(f"case n={n} {x_dtype} {r_dtype} p={p}", flush=True)
    g = torch.Generator(device=dev()).manual_seed(n)
    x = torch.randn(n, generator=g, device=dev()).to(x_dtype).requires_grad_(True)
    r = None if r_dtype is None else torch.randn(n, generator=g, device=dev()).to(r_dtype).requires_grad_(True)
    y = spa2.dropout_add(x, r, p, seed, offset)
    keep, factor = ref.keep_mask(n, p, seed, offset)
    assert y.dtype == (r_dtype or x_dtype) and y.shape == x.shape
    product = f64(x) * factor * keep
    want = product + (0 if r is None else f64(r))
    assert (np.abs(f64(y) - want) <= half_step(y.dtype) * np.abs(want) + 2.0 ** -23 * np.abs(product)).all()
    up = torch.randn(n, generator=g, device=dev()).to(y.dtype)
    grads = torch.autograd.grad(y, (x,) if r is None else (x, r), up)
    want = f64(up) * factor * keep
    assert grads[0].dtype == x_dtype
    assert (np.abs(f64(grads[0]) - want) <= (half_step(x_dtype) + 2.0 ** -23) * np.abs(want)).all()
    assert np.array_equal(f64(grads[0]) != 0, (keep & (f64(up) != 0)))
    if r is not None:
        assert torch.equal(grads[1], up)


def test_share_of_kept_elements_and_independence():
    """Counts within 6 standard deviations; another seed, offset or neighbour agrees as often as chance has it."""
    n, p = 1 << 22, 0.25
    one = torch.ones(n, device=dev())
    masks = [spa2.dropout_add(one, None, p, s, o) != 0 for s, o in ((1, 0), (2, 0), (1, 1), (1 + 2 ** 32, 0), (1, 2 ** 32))]
    q = 1 - p
    for m in masks:
        assert abs(int(m.sum()) - n * q) <= 6 * (n * p * q) ** 0.5
    same = p * p + q * q
    pairs = [(masks[a], masks[b]) for a in range(5) for b in range(a)] + [(masks[0][:-s], masks[0][s:]) for s in (1, 2, 8, 4096)]
    for a, b in pairs:
        assert abs(int((a == b).sum()) - a.numel() * same) <= 6 * (a.numel() * same * (1 - same)) ** 0.5


@pytest.mark.parametrize("p", [0.0, 2.0 ** -18, 1.0])
def test_borders_of_p(p):
    x, r = torch.randn(1001, device=dev(), requires_grad=True), torch.randn(1001, device=dev())
    y = spa2.dropout_add(x, r, p, 3)
    want = r if p == 1.0 else x.detach() + r
    assert torch.equal(y, want)
    (dx,) = torch.autograd.grad(y, x, r)
    assert torch.equal(dx, torch.zeros_like(r) if p == 1.0 else r)


def test_dropped_infinities_leave_the_residual():
    x = torch.full((4096,), float("inf"), device=dev())
    x[::2] = float("nan")
    r = torch.randn(4096, device=dev())
    y = spa2.dropout_add(x, r, 0.5, 9)
    keep = torch.from_numpy(ref.keep_mask(4096, 0.5, 9, 0)[0]).to(dev())
    assert torch.equal(y[~keep], r[~keep]) and not torch.isfinite(y[keep]).any()


def test_other_strides_alignment_and_shapes():
    """Element numbers are row-major whatever the memory order."""
    base = torch.randn(12, 50, 33, device=dev()).bfloat16()
    want = spa2.dropout_add(base, base, 0.3, 5, 6)
    turned = base.permute(2, 0, 1).contiguous().permute(1, 2, 0)
    assert turned.stride() != base.stride() and torch.equal(spa2.dropout_add(turned, base, 0.3, 5, 6), want)
    shifted = torch.empty(base.numel() + 1, dtype=BF, device=dev())[1:].view(base.shape).copy_(base).requires_grad_(True)
    y = spa2.dropout_add(shifted, shifted.detach(), 0.3, 5, 6)
    assert torch.equal(y, want)
    up = torch.empty(base.numel() + 1, dtype=BF, device=dev())[1:].view(base.shape).copy_(base)
    (dx,) = torch.autograd.grad(y, shifted, up)
    (dx2,) = torch.autograd.grad(spa2.dropout_add(shifted, None, 0.3, 5, 6), shifted, base.expand(base.shape))
    assert torch.equal(dx, dx2)
    scalar = torch.tensor(2.0, device=dev(), requires_grad=True)
    (ds,) = torch.autograd.grad(spa2.dropout_add(scalar, None, 0.5, 1), scalar)
    assert float(ds) in (0.0, 2.0) and float(ds) == 2.0 * bool(ref.keep_mask(1, 0.5, 1, 0)[0][0])


def test_in_place_result():
    from gpu_util import Guarded
    g = Guarded()
    x = torch.randn(1003, device=dev())
    y = g.alloc((1003,), F, dev(), 1.0)
    spa2.spa2_dropout_add(x, y, 0.5, 7, 8, y)
    torch.cuda.synchronize()
    g.check("dropout")
    assert torch.equal(y, spa2.dropout_add(x, torch.ones_like(x), 0.5, 7, 8))


def test_refusals():
    x = torch.randn(4, 8, device=dev())
    f = spa2.dropout_add
    two = torch.tensor([1, 2], device=dev())
    for bad in (lambda: f(x.half(), None, 0.5, 1), lambda: f(x, x.bfloat16(), 0.5, 1), lambda: f(x, x[:1], 0.5, 1),
                lambda: f(x, x.cpu(), 0.5, 1), lambda: f(x, None, 0.5, two.int()), lambda: f(x, None, 0.5, two[:1]),
                lambda: f(x, None, 0.5, two, 1), lambda: f(x, None, 0.5, two.cpu())):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: f(x, None, -0.1, 1), lambda: f(x, None, 1.01, 1), lambda: f(x, None, float("nan"), 1),
                lambda: f(x[:0], None, 0.5, 1)):
        with pytest.raises(spa2.Spa2Error):
            bad()


def test_second_derivative_is_refused():
    x = torch.randn(64, device=dev(), requires_grad=True)
    y = spa2.dropout_add(x, None, 0.5, 1)
    (dx,) = torch.autograd.grad(y, x, torch.ones_like(y), create_graph=True)
    with pytest.raises(RuntimeError, match="second derivative"):
        dx.sum().backward()


def test_seed_on_the_device():
    """Same numbers as from the host; changed between a forward pass and its backward pass it is refused; a captured graph
    draws the mask that the tensor says at each replay."""
    x, r = torch.randn(3001, device=dev(), requires_grad=True), torch.randn(3001, device=dev())
    so = torch.tensor([-5, 2 ** 35 + 1], device=dev())
    assert torch.equal(spa2.dropout_add(x, r, 0.3, so), spa2.dropout_add(x, r, 0.3, -5, 2 ** 35 + 1))
    y = spa2.dropout_add(x, r, 0.3, so)
    so[1] += 1
    with pytest.raises(RuntimeError):
        torch.autograd.grad(y, x, r)
    del y

    def step(seed, *offset):
        y = spa2.dropout_add(x, r, 0.3, seed, *offset)
        return [y.detach(), *torch.autograd.grad(y, x, r)]
    step(so)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step(so)
    for replay in range(3):
        so.copy_(torch.tensor([77 + replay, replay]))
        want = step(77 + replay, replay)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(held, want):
            assert torch.equal(a, b), replay


def test_capture_beside_an_eager_graph_of_the_same_leaf_is_refused():
    x = torch.randn(64, device=dev(), requires_grad=True)
    y = spa2.dropout_add(x, None, 0.5, 1)                   # alive, made on another stream than the capture's
    torch.cuda.synchronize()
    with pytest.raises(RuntimeError, match="eager graph"):
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            spa2.dropout_add(x, None, 0.5, 1)
    graph = torch.cuda.CUDAGraph()
    with torch.no_grad(), torch.cuda.graph(graph):
        held = spa2.dropout_add(x, None, 0.5, 1)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(held, y.detach())


@pytest.mark.parametrize("grad", [False, True])
def test_inputs_with_tangents_are_refused(grad):
    import torch.autograd.forward_ad as fwad
    x = torch.randn(1, 2, 8, 64, device=dev())
    f = lambda t: spa2.dropout_add(t, x, 0.5, 1)
    with torch.set_grad_enabled(grad), fwad.dual_level():
        want = f(x)
        with pytest.raises(RuntimeError):
            f(fwad.make_dual(x, torch.ones_like(x)))
    assert torch.equal(f(x), want)
