"""The norm over all gradients and their clipping, against sums in fp64."""
import math

import numpy as np
import pytest
import torch

import paper_2602_13515_amd as spa2
import step_ref as ref
from gpu_util import Guarded, dev

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def f64(t):
    return t.detach().double().cpu().numpy()


def _make(sizes, types, seed=0, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return [(scale * torch.randn(s, generator=g)).to(types[i % len(types)]).to(dev()) for i, s in enumerate(sizes)]


def _check_values(got, grads, f):
    """A product in fp64, rounded once (bf16: by way of fp32, 2^-24 more)."""
    for o, g in zip(got, grads):
        want = f64(g) * f
        half = torch.finfo(o.dtype).eps / 2 + 2.0 ** -24 * (o.dtype == BF)
        tiny = float(torch.finfo(o.dtype).smallest_normal) * torch.finfo(o.dtype).eps
        assert (np.abs(f64(o) - want) <= half * (1 + 2.0 ** -20) * np.abs(want) + tiny).all()


def _check_norm(norm, want):
    assert norm.dtype == F32 and norm.dim() == 0 and norm.is_cuda
    assert abs(float(norm) - want) <= 2.0 ** -24 * (1 + 2.0 ** -20) * want


SIZES = [(1,), (7,), (4095,), (4096,), (4097,), (3, 50, 41), (0,), (100, 1001), ()]


@pytest.mark.parametrize("out", ["in place", "same", "fp32"])
@pytest.mark.parametrize("types", [(F32,), (BF,), (F32, BF)], ids=["fp32", "bf16", "both"])
@pytest.mark.parametrize("limit", [0.0, 0.37, 1e9, math.inf])
def test_values(types, out, limit):
    grads = _make(SIZES, types)
    before = [g.clone() for g in grads]
    want, f = ref.clip_factor([f64(g) for g in grads], limit, 1e-6)
    outs = None if out == "in place" else [torch.full_like(g, float("nan"), dtype=F32 if out == "fp32" else g.dtype) for g in grads]
    norm = spa2.clip_gradients(grads, limit, out=outs)
    _check_norm(norm, want)
    _check_values(grads if outs is None else outs, before, f)
    if outs is not None or f == 1.0:
        assert all(torch.equal(a, b) for a, b in zip(grads, before))
    assert torch.equal(spa2.gradient_norm(before), norm)


def test_many_tensors_and_long_ones():
    """Several launches' tables; a tensor that all workgroups walk more than once; elements at odd addresses."""
    sizes = [(1 + 37 * i % 5000,) for i in range(391)] + [(9_000_001,), (3,)]
    for types in ((F32,), (BF, F32)):
        grads = _make(sizes, types, 1)
        before = [g.clone() for g in grads]
        want, f = ref.clip_factor([f64(g) for g in grads], 2.0, 1e-6)
        _check_norm(spa2.clip_gradients(grads, 2.0), want)
        _check_values(grads, before, f)
        again = [g.clone() for g in before]
        spa2.clip_gradients(again, 2.0)
        assert all(torch.equal(a, b) for a, b in zip(grads, again))
    counts = [math.prod(s) for s in sizes]
    for dtype, out_dtype in ((F32, F32), (BF, F32), (BF, BF)):
        whole = torch.randn(sum(counts) + 1, device=dev()).to(dtype)[1:]
        out = torch.full((sum(counts) + 3,), 5.0, dtype=out_dtype, device=dev())
        views, outs = list(whole.split(counts)), list(out[1:-2].split(counts))
        want, f = ref.clip_factor([f64(whole)], 3.0, 0.0)
        _check_norm(spa2.clip_gradients(views, 3.0, out=outs, eps=0.0), want)
        _check_values([out[1:-2]], [whole], f)
        assert (out[:1] == 5).all() and (out[-2:] == 5).all()
        spa2.clip_gradients(views, 3.0, eps=0.0)
        if dtype == out_dtype:
            assert torch.equal(whole, out[1:-2])


def test_large_and_small_numbers():
    """Squares that fp32 cannot hold; a norm of zero; products that end in subnormals."""
    big = [torch.full((1000,), 3e38, device=dev()), torch.full((5,), -1e30, device=dev())]
    before = [b.clone() for b in big]
    want, f = ref.clip_factor([f64(b) for b in big], 1.0, 1e-6)
    assert math.isinf(float(spa2.clip_gradients(big, 1.0))) and want > 3.5e38      # (the norm itself is beyond fp32)
    _check_values(big, before, f)
    small = [torch.full((1000,), 1e-30, device=dev())]
    before = [s.clone() for s in small]
    want, f = ref.clip_factor([f64(s) for s in small], 1e-38, 0.0)
    _check_norm(spa2.clip_gradients(small, 1e-38, eps=0.0), want)
    _check_values(small, before, f)
    zero = [torch.zeros(10, device=dev())]
    for limit, eps in ((1.0, 1e-6), (1.0, 0.0), (0.0, 0.0)):
        assert float(spa2.clip_gradients(zero, limit, eps=eps)) == 0.0 and not zero[0].any()


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_what_is_not_finite_follows_the_formula(bad):
    grads = _make([(100,), (5000,)], (F32,))
    grads[1][4999] = bad
    before = [g.clone() for g in grads]
    norm = spa2.clip_gradients(grads, 1.0)
    if math.isnan(bad):
        assert torch.isnan(norm) and all(torch.isnan(g).all() for g in grads)
    else:
        assert torch.isinf(norm) and not grads[0].any() and torch.isnan(grads[1][4999]) and not grads[1][:4999].any()
    assert float(spa2.clip_gradients(before, math.inf)) != 0.0 and torch.equal(before[0], _make([(100,), (5000,)], (F32,))[0])


def test_gaps_and_orders():
    """Transposed ones as they lie in memory; with gaps by way of copies."""
    wide = torch.randn(40, 60, device=dev())
    forms = [wide.clone().t(), wide.clone()[:, ::2], wide.clone()[3:17, 5:50], torch.randn(2, 3, 8, 9, device=dev()).to(memory_format=torch.channels_last)]
    before = [t.clone() for t in forms]
    want, f = ref.clip_factor([f64(t) for t in forms], 0.5, 1e-6)
    _check_norm(spa2.clip_gradients(forms, 0.5), want)
    _check_values(forms, before, f)
    outs = [torch.empty_like(t.contiguous(), dtype=BF) for t in forms]
    outs[0] = torch.empty(40, 60, dtype=BF, device=dev())[:, ::1].t()
    outs[1] = torch.zeros(40, 90, dtype=BF, device=dev())[:, ::3]
    _check_norm(spa2.clip_gradients(before, 0.5, out=outs), want)
    _check_values(outs, before, f)


def test_shared_memory_is_refused_before_anything_is_written():
    t = torch.randn(100, device=dev())
    kept = t.clone()
    other = torch.empty(100, device=dev())
    wide = torch.randn(10, 20, device=dev())
    calls = [lambda: spa2.clip_gradients([t, t], 0.1), lambda: spa2.clip_gradients([t[:60], t[40:]], 0.1),
             lambda: spa2.clip_gradients([t, other], 0.1, out=[other, t]), lambda: spa2.clip_gradients([t], 0.1, out=[t.view(BF)[:100]]),
             lambda: spa2.clip_gradients([t, t], 0.1, out=[other, other]), lambda: spa2.clip_gradients([t[:90]], 0.1, out=[t[10:]]),
             lambda: spa2.clip_gradients([wide, wide[:, ::2]], 0.1), lambda: spa2.clip_gradients([wide[:, ::2], wide[:, ::2]], 0.1)]
    for call in calls:
        with pytest.raises(ValueError, match="shares memory"):
            call()
    with pytest.raises(RuntimeError):
        spa2.clip_gradients([t[:1].expand(5)], 0.1)
    assert torch.equal(t, kept)
    # reading the same gradient twice is fine, as are views that lie between each other
    a, b = torch.empty(100, device=dev()), torch.empty(100, device=dev())
    assert abs(float(spa2.clip_gradients([t, t], math.inf, out=[a, b])) ** 2 - 2 * float((t.double() ** 2).sum())) < 1e-4
    assert torch.equal(a, t) and torch.equal(b, t)
    spa2.clip_gradients([wide[:, ::2], wide[:, 1::2]], 0.1)


def test_refusals():
    t = torch.zeros(4, device=dev())
    for bad in (dict(max_norm=-1.0), dict(max_norm=math.nan), dict(max_norm=1.0, eps=-1.0), dict(max_norm=1.0, eps=math.inf)):
        with pytest.raises(spa2.Spa2Error):
            spa2.clip_gradients([t], **bad)
    for call in (lambda: spa2.clip_gradients([], 1.0), lambda: spa2.clip_gradients([t.cpu()], 1.0), lambda: spa2.clip_gradients([t.half()], 1.0),
                 lambda: spa2.clip_gradients([t], 1.0, out=[t, t]), lambda: spa2.clip_gradients([t], 1.0, out=[t.half()]),
                 lambda: spa2.clip_gradients([t], 1.0, out=[t[:2]]), lambda: spa2.clip_gradients([t, t.cpu()], 1.0),
                 lambda: spa2.clip_gradients([t.clone().requires_grad_(True)], 1.0)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        spa2.clip_gradients([t, None], 1.0)
    leaf = torch.ones(4, device=dev(), requires_grad=True)
    with torch.no_grad():
        spa2.clip_gradients([leaf], 1.0)
    assert abs(float(leaf.detach().norm()) - 1.0) < 1e-5


def test_autograd_notices_what_was_written():
    x = torch.randn(8, device=dev(), requires_grad=True)
    g = torch.randn(8, device=dev())
    y = (x * g).sum()
    spa2.clip_gradients([g], 0.1)
    with pytest.raises(RuntimeError, match="modified by an inplace"):
        y.backward()


def test_captured_calls_and_another_stream():
    sizes = [(500, 33), (7,), (70001,)] + [(11,)] * 200
    grads, fresh = _make(sizes, (F32, BF), 3), _make(sizes, (F32, BF), 4)
    outs = [torch.empty_like(g, dtype=F32) for g in grads]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        norm = spa2.clip_gradients(grads, 1.5, out=outs)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = spa2.clip_gradients(grads, 1.5, out=outs)
        held_in_place = spa2.clip_gradients(fresh, 1.5)
    for replay in range(3):
        for g in grads + fresh:
            g.normal_()
        want_outs, copies = [torch.empty_like(o) for o in outs], [g.clone() for g in fresh]
        want, second = spa2.clip_gradients(grads, 1.5, out=want_outs), spa2.clip_gradients(copies, 1.5)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(held, want) and torch.equal(held_in_place, second), replay
        assert all(torch.equal(a, b) for a, b in zip(outs + fresh, want_outs + copies)), replay
    assert norm.isfinite()


def test_nothing_is_written_outside():
    from paper_2602_13515_amd import binding
    gd = Guarded()
    for n in (1, 5, 4099, 50001):
        x = torch.randn(n, device=dev())
        for dtype in (BF, F32):
            out, norm, ws = gd.alloc((n,), dtype, dev(), float("nan")), gd.alloc((1,), F32, dev(), 0.0), \
                gd.alloc((binding.spa2_clip_workspace_bytes(),), torch.uint8, dev(), 255)
            binding.spa2_clip_gradients([x], [out], 0.5, 1e-6, norm, ws)
            torch.cuda.synchronize()
            gd.check(str(n))
            assert torch.isfinite(out).all()


def test_tensors_behind_two_to_the_thirty_one():
    n = 2 ** 31 + 5001
    x = torch.zeros(n, dtype=BF, device=dev())
    x[-4000:] = 1.0
    x[:3] = 2.0
    assert float(spa2.gradient_norm(x)) == pytest.approx(math.sqrt(4012), rel=2.0 ** -23)
    spa2.clip_gradients(x, math.sqrt(4012) / 2, eps=0.0)
    assert (x[-4000:] == 0.5).all() and (x[:3] == 1.0).all() and not x[3:-4000:4099].any()
