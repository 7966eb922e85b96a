"""Attention over a window, forward and backward, against the fp64 formulas (bounds: step_ref.window)."""
import numpy as np
import pytest
import torch

import paper_2602_13515_amd as spa2
import step_ref as ref
from gpu_util import REL_L2, Guarded, dev

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def f64(t):
    return t.detach().double().cpu().numpy()


def _heads(g, B, H, N, d, layout="bnhd"):
    x = torch.randn((B, N, H, d), generator=g).to(BF).to(dev())
    if layout == "bnhd":
        return x.permute(0, 2, 1, 3)
    if layout == "bhnd":
        return x.permute(0, 2, 1, 3).contiguous()
    assert layout == "gaps"
    wide = torch.full((B, N, 2 * H + 1, d), float("nan"), dtype=BF, device=dev())
    wide[:, :, 1:H + 1] = x
    return wide[:, :, 1:H + 1].permute(0, 2, 1, 3)


def _inputs(B, Hq, Hk, Nq, Nk, d, layouts=("bnhd", "bnhd", "bnhd"), seed=0):
    g = torch.Generator().manual_seed(seed + Nq + 7 * Nk + d)
    q, k, v = _heads(g, B, Hq, Nq, d, layouts[0]), _heads(g, B, Hk, Nk, d, layouts[1]), _heads(g, B, Hk, Nk, d, layouts[2])
    return q, k, v, torch.randn((B, Nq, Hq, d), generator=g).to(BF).to(dev()).permute(0, 2, 1, 3)


def _i32(x):
    return None if x is None else torch.tensor(x, dtype=torch.int32, device=dev())


def _check(q, k, v, do, left, right, sinks, lengths=None, starts=None, scale=None, whole=True):
    """whole: 2-norms too (with few keys a row dS is a difference of nearly equal numbers, and with one it is zero: a bar relative
    to the result cannot hold for dQ and dK there, the bounds by magnitudes do)."""
    s = q.shape[-1] ** -0.5 if scale is None else scale
    args = dict(left=left, right=right, sinks=sinks, lengths=_i32(lengths), starts=_i32(starts), scale=scale)
    want, _ = ref.window(f64(q), f64(k), f64(v), lengths, starts, left, right, sinks, s, f64(do))
    with torch.no_grad():
        plain = spa2.window_attention(q, k, v, **args)
    leaves = [t.detach().requires_grad_(True) for t in (q, k, v)]
    o = spa2.window_attention(*leaves, **args)
    assert torch.equal(o, plain) and o.shape == q.shape
    grads = torch.autograd.grad(o, leaves, do)
    for name, t in zip(("o", "dq", "dk", "dv"), (o, *grads)):
        value, bound = want[name]
        x = f64(t)
        assert np.isfinite(x).all(), name
        err = np.abs(x - value)
        assert (err <= bound + 1e-30).all(), (name, (err - bound).max(), err.max())
        if whole or name in ("o", "dv"):
            assert np.linalg.norm(x - value) <= REL_L2 * np.linalg.norm(value) + 1e-30, name
    again = torch.autograd.grad(spa2.window_attention(*leaves, **args), leaves, do)
    assert all(torch.equal(a, b) for a, b in zip(grads, again))
    return o, grads


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("left,right,sinks", [(None, 0, 0), (0, 0, 0), (1, 0, 0), (7, 0, 3), (63, 0, 64), (64, 0, 65), (100, 0, 1), (None, None, 0),
                                              (127, 40, 0), (0, 9, 5), (200, 64, 130), (None, 33, 0), (30, None, 4), (5000, 5000, 5000)])
def test_windows_of_a_sequence(left, right, sinks, d):
    q, k, v, do = _inputs(1, 2, 2, 330, 330, d)
    _check(q, k, v, do, left, right, sinks, whole=left is None or left >= 7)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("N", [1, 2, 31, 63, 64, 65, 127, 128, 129, 193, 257, 640])
def test_lengths_of_a_sequence(N, d):
    q, k, v, do = _inputs(2, 4, 2, N, N, d)
    _check(q, k, v, do, 50, 0, 3, whole=N > 60)
    _check(q, k, v, do, 20, 11, 0, whole=N > 60)


@pytest.mark.parametrize("Hq,Hk", [(1, 1), (6, 2), (5, 1), (3, 3)])
@pytest.mark.parametrize("layouts", [("bnhd",) * 3, ("bhnd", "bnhd", "bnhd"), ("gaps", "bhnd", "bnhd"), ("bnhd", "gaps", "gaps")])
def test_heads_and_layouts(Hq, Hk, layouts):
    q, k, v, do = _inputs(2, Hq, Hk, 200, 200, 64, layouts)
    _check(q, k, v, do, 70, 0, 10)


@pytest.mark.parametrize("d", [64, 128])
def test_padded_samples(d):
    """Lengths of their own; places behind them see what the window still reaches, and the first keys."""
    q, k, v, do = _inputs(4, 6, 2, 321, 321, d)
    lengths = [321, 100, 0, 7]
    for left, right, sinks in ((80, 0, 5), (40, 40, 0), (None, 0, 0)):
        o, (dq, dk, dv) = _check(q, k, v, do, left, right, sinks, lengths=lengths)
        assert not o[2].any() and not dq[2].any() and not dk[2].any()
        for b, n in enumerate(lengths):
            assert not dk[b, :, n:].any() and not dv[b, :, n:].any()
        if sinks == 0 and left is not None:
            assert not o[3, :, 7 + left:].any() and not dq[3, :, 7 + left:].any()
    _check(q, k, v, do, 80, 0, 5, lengths=[999, -5, 2 ** 31 - 1, -2 ** 31])


@pytest.mark.parametrize("starts", [[0, 0, 0], [-50, 200, 500], [-400, 301, 2 ** 31 - 1], [-2 ** 31, 3, 297]])
@pytest.mark.parametrize("left,right,sinks", [(90, 0, 6), (30, 50, 0), (None, 0, 0), (2 ** 28, 0, 0), (10, None, 70)])
def test_places_anywhere(starts, left, right, sinks):
    """Queries before all keys, among them and behind them, places at the ends of 32 bits."""
    q, k, v, do = _inputs(3, 4, 2, 150, 300, 64)
    _check(q, k, v, do, left, right, sinks, starts=starts, lengths=[300, 280, 300], whole=False)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Nq,Hq,Hk", [(1, 8, 8), (1, 10, 2), (1, 40, 1), (3, 8, 2), (5, 6, 1), (17, 4, 2), (64, 3, 1), (65, 6, 2), (1, 33, 1)])
def test_last_tokens_of_caches(Nq, Hq, Hk, d):
    """One query, or a few, against caches of unlike length; heads that are taken together and not."""
    lengths = [2000, 1333, Nq, 70, 1999]
    for layout in ("bnhd", "bhnd"):
        q, k, v, do = _inputs(5, Hq, Hk, Nq, 2000, d, (layout, "bnhd", "bnhd"))
        for left, right, sinks in ((511, 0, 4), (100, 0, 0), (None, 0, 0), (1200, 3, 100)):
            _check(q, k, v, do, left, right, sinks, lengths=lengths, starts=[n - Nq for n in lengths], whole=False)


@pytest.mark.parametrize("Nq,B", [(1, 1), (1, 1100), (4, 3), (100, 1), (300, 1)])
@pytest.mark.parametrize("left,sinks", [(9000, 5), (None, 0), (8000, 700)])
def test_long_caches_are_shared_out(Nq, B, left, sinks):
    """Few rows and long lists: parts of rows, joined."""
    Nk = 12000 if B < 100 else 150
    q, k, v, do = _inputs(B, 2, 1, Nq, Nk, 64)
    _check(q, k, v, do, left, 0, sinks)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Nq,Hq,Hk", [(8, 10, 2), (20, 10, 2), (64, 6, 3), (33, 2, 1), (2, 40, 2), (63, 9, 3)])
@pytest.mark.parametrize("layout", ["bnhd", "bhnd", "gaps"])
def test_some_tokens_of_heads_that_share_keys(Nq, Hq, Hk, d, layout):
    """Rows of several heads as those of one, wherever they lie, in blocks that heads begin and end inside of; long lists in parts."""
    for B, Nk, lengths in ((2, 9000, [9000, 4321]), (3, 300, [300, 0, 17])):
        q, k, v, do = _inputs(B, Hq, Hk, Nq, Nk, d, (layout, "bnhd", "bnhd"))
        for left, right, sinks in ((200, 0, 4), (None, 0, 0)):
            _check(q, k, v, do, left, right, sinks, lengths=lengths, starts=[n - Nq for n in lengths], whole=False)


@pytest.mark.parametrize("B,Nk", [(63, 1100), (64, 1100), (65, 1100), (130, 1100), (256, 1100), (500, 1100), (1024, 1100), (70, 17000)])
def test_many_samples_share_a_line(B, Nk):
    """One query of many samples of unlike length and place, empty ones among them: stretches that begin and end inside samples."""
    g = torch.Generator().manual_seed(B)
    lengths = torch.randint(0, 1100, (B,), generator=g)
    lengths[::7] = 0
    lengths[B // 2] = Nk
    starts = (lengths - 1 - torch.randint(0, 90, (B,), generator=g)).tolist()
    q, k, v, do = _inputs(B, 3, 1, 1, Nk, 64)
    for left, right, sinks in ((300, 0, 5), (None, 100, 0), (40, 40, 0)):
        _check(q, k, v, do, left, right, sinks, lengths=lengths.tolist(), starts=starts, whole=False)
    want, _ = ref.window(f64(q), f64(k), f64(v), lengths.tolist(), None, None, None, 0, 64 ** -0.5, f64(do))
    value, bound = want["o"]
    with torch.no_grad():
        o = spa2.cross_attention(q, k, v, _i32(lengths.tolist()))
    assert (np.abs(f64(o) - value) <= bound + 1e-30).all()


def test_columns_of_first_keys_are_shared_out():
    """Long columns of first keys among short ones, one head: parts, joined by the last to arrive; and columns that are all long."""
    for d in (64, 128):
        q, k, v, do = _inputs(1, 2, 1, 4000, 4000, d)
        _check(q, k, v, do, 150, 0, 70)
        _check(q, k, v, do, 150, 20, 1)
        _check(q, k, v, do, None, 0, 0)
        _check(q, k, v, do, 2500, 2500, 0)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_what_nobody_sees_is_not_read(bad):
    """Keys and values outside every window and behind the lengths, at the edges of blocks too; queries that see nothing, with
    their upstream gradients."""
    for d in (64, 128):
        for Nq, start, left, sinks in ((1, 700, 99, 4), (40, 650, 33, 0), (200, 500, 77, 10), (300, 400, 200, 65)):
            q, k, v, do = _inputs(2, 4, 2, Nq, 1000, d)
            lengths, starts = [1000, start + Nq], [start, start]
            o, grads = _check(q, k, v, do, left, 0, sinks, lengths=lengths, starts=starts, whole=False)
            # what the first query's block of 128 and those behind it do not reach
            k2, v2 = k.clone(), v.clone()
            for t in (k2, v2):
                t[:, :, sinks:start - left] = bad
                t[:, :, start + Nq:] = bad
            leaves = [t.detach().requires_grad_(True) for t in (q, k2, v2)]
            o2 = spa2.window_attention(*leaves, left, 0, sinks, _i32(lengths), _i32(starts))
            grads2 = torch.autograd.grad(o2, leaves, do)
            assert torch.equal(o, o2) and all(torch.equal(a, b) for a, b in zip(grads, grads2))
    q, k, v, do = _inputs(1, 2, 2, 200, 200, 64)
    o, grads = _check(q, k, v, do, 30, 0, 0, starts=[-70])
    q2, do2 = q.clone(), do.clone()
    q2[:, :, :70], do2[:, :, :70] = bad, bad
    leaves = [t.detach().requires_grad_(True) for t in (q2, k, v)]
    o2 = spa2.window_attention(*leaves, 30, 0, 0, starts=_i32([-70]))
    grads2 = torch.autograd.grad(o2, leaves, do2)
    assert torch.equal(o, o2) and all(torch.equal(a, b) for a, b in zip(grads, grads2))


def test_equals_the_other_attention_where_there_is_no_limit():
    """No limits: attention to a sequence of all keys; the same sums in another order at most."""
    q, k, v, do = _inputs(2, 4, 2, 300, 500, 128)
    lens = _i32([500, 222])
    a, b = spa2.window_attention(q, k, v, None, None, lengths=lens), spa2.cross_attention(q, k, v, lens)
    assert (a.float() - b.float()).abs().max() <= 2.0 ** -8 * b.float().abs().max()


def test_minus_infinite_scores_take_no_part():
    """Products that overflow: keys whose score is minus infinity have no weight, a row with no other is lost, rows that see
    nothing are zero."""
    q, k, v, do = _inputs(1, 1, 1, 200, 200, 64)
    q = torch.full_like(q, 3e38)
    k = k.clone()
    k[..., :] = 0.0
    k[:, :, 10:40] = -3e38
    o = spa2.window_attention(q, k, v, 20, 0, 0, starts=_i32([-5]))
    p = np.arange(200) - 5
    lost = (p - 20 >= 10) & (p < 40)
    blind = p < 0
    x = f64(o)[0, 0]
    assert np.isnan(x[lost]).all() and not x[blind].any() and np.isfinite(x[~lost]).all()


@pytest.mark.parametrize("scale", [1e-3, 0.7])
def test_scales(scale):
    q, k, v, do = _inputs(1, 2, 2, 260, 260, 128)
    _check(q, k, v, do, 100, 0, 2, scale=scale)


def test_long_strides_and_offsets():
    """Elements behind 2^31 of a cache, far apart tokens."""
    N, H, d = 33000, 512, 128
    cache = torch.zeros((1, N, H, d), dtype=BF, device=dev())
    g = torch.Generator().manual_seed(5)
    near = torch.randn((1, 700, 2, d), generator=g).to(BF).to(dev())
    cache[:, -700:, -2:] = near
    k = v = cache[:, :, -2:].permute(0, 2, 1, 3)
    q, _, _, do = _inputs(1, 4, 2, 300, 300, d)
    o = spa2.window_attention(q, k, v, 350, 0, 0)
    # (not the bits of a call on those 700 keys alone: key 32300 is the 45th of its block of 64, so that other keys share a tile, and
    # the weights that are rounded are those against another running maximum: the bounds count each weight's rounding, whichever)
    small = f64(near.permute(0, 2, 1, 3))
    (value, bound), _ = ref.window(f64(q), small, small, None, None, 350, 0, 0, d ** -0.5)[0]["o"], None
    assert (np.abs(f64(o) - value) <= bound).all()
    one = spa2.window_attention(q[:, :, -1:], k, v, 350, 0, 3)
    assert torch.isfinite(one).all() and one.any()


def test_nothing_is_written_outside():
    from paper_2602_13515_amd import binding
    for B, Hq, Hk, Nq, Nk, d, left, right, sinks in ((2, 4, 2, 131, 131, 64, 40, 0, 3), (1, 2, 1, 300, 3000, 128, 2000, 0, 100),
                                                     (3, 4, 1, 2, 5000, 64, 4000, 0, 9), (1, 1, 1, 1, 1, 128, 0, 0, 0)):
        gd = Guarded()
        g = torch.Generator().manual_seed(1)
        q, k, v, do = (torch.randn((B, h, n, d), generator=g).to(BF).to(dev()) for h, n in ((Hq, Nq), (Hk, Nk), (Hk, Nk), (Hq, Nq)))
        o, o_res, dq = (gd.alloc(q.shape, BF, dev(), float("nan")) for _ in range(3))
        dk, dv = (gd.alloc(k.shape, BF, dev(), float("nan")) for _ in range(2))
        lse = gd.alloc((B, Hq, Nq), torch.float32, dev(), float("nan"))
        ws = gd.alloc((binding.spa2_window_fwd_workspace_bytes(q, k, left, right, sinks),), torch.uint8, dev(), 255)
        ws2 = gd.alloc((binding.spa2_window_bwd_workspace_bytes(q, k, left, right, sinks),), torch.uint8, dev(), 255)
        binding.spa2_window_fwd(q, k, v, None, None, left, right, sinks, d ** -0.5, o, lse, o_res, ws)
        binding.spa2_window_bwd(q, k, v, None, None, left, right, sinks, o, do, lse, d ** -0.5, dq, dk, dv, ws2, o_res)
        torch.cuda.synchronize()
        gd.check(f"{Nq} of {Nk}")
        assert all(torch.isfinite(t).all() for t in (o, o_res, dq, dk, dv, lse))
        _, want = ref.window(f64(q), f64(k), f64(v), None, None, left, right, sinks, d ** -0.5)
        assert np.abs(f64(lse) - want).max() <= 2.0 ** -8


def test_gradients_against_differences():
    """Along random directions of q, k and v, by the fp64 form: the formulas of step_ref.window are the derivatives."""
    rng = np.random.default_rng(2)
    q, k, v = rng.standard_normal((1, 2, 9, 8)), rng.standard_normal((1, 1, 12, 8)), rng.standard_normal((1, 1, 12, 8))
    do, h = rng.standard_normal(q.shape), 1e-5
    args = ([11], [2], 3, 1, 2, 0.4)
    got, _ = ref.window(q, k, v, *args, do)
    f = lambda q, k, v: (ref.window(q, k, v, *args)[0]["o"][0] * do).sum()
    for _ in range(6):
        w = [rng.standard_normal(x.shape) for x in (q, k, v)]
        diff = (f(*(x + h * y for x, y in zip((q, k, v), w))) - f(*(x - h * y for x, y in zip((q, k, v), w)))) / (2 * h)
        terms = [got[n][0] * y for n, y in zip(("dq", "dk", "dv"), w)]
        assert abs(diff - sum(t.sum() for t in terms)) <= 1e-7 * sum(np.abs(t).sum() for t in terms)


def test_captured_steps_and_another_stream():
    q, k, v, do = _inputs(2, 4, 2, 500, 500, 64)
    lens = _i32([500, 300])
    leaves = [t.detach().requires_grad_(True) for t in (q, k, v)]
    few = q[:, :, :1].contiguous()
    places = _i32([499, 299])

    def step():
        o = spa2.window_attention(*leaves, 200, 0, 80, lens)
        with torch.no_grad():
            one = spa2.window_attention(few, k, v, 200, 0, 80, lens, places)
        return [o.detach(), one, *torch.autograd.grad(o, leaves, do)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        first = step()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(first, step()))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for replay in range(3):
        with torch.no_grad():
            leaves[0].mul_(1.2)
            lens.sub_(17)
            places.sub_(17)
        want = step()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want)), replay


def test_second_derivatives_tangents_and_transforms_are_refused():
    q, k, v, _ = _inputs(1, 2, 2, 70, 70, 64)
    leaf = q.detach().requires_grad_(True)
    (d,) = torch.autograd.grad(spa2.window_attention(leaf, k, v, 10).float().sum(), leaf, create_graph=True)
    with pytest.raises(RuntimeError):
        d.float().sum().backward()
    import torch.autograd.forward_ad as fa
    with fa.dual_level(), pytest.raises(RuntimeError):
        spa2.window_attention(fa.make_dual(q, torch.ones_like(q)), k, v, 10)
    with pytest.raises(RuntimeError):
        torch.func.vmap(lambda t: spa2.window_attention(t, k, v, 10))(q[None])


def test_refusals():
    q, k, v, _ = _inputs(2, 4, 2, 20, 30, 64)
    for bad in (dict(left=-1), dict(left=3, right=-2), dict(left=3, sinks=-1), dict(left=2 ** 28 + 1), dict(left=3, sinks=2 ** 40),
                dict(left=3, lengths=_i32([1])), dict(left=3, starts=_i32([1])), dict(left=3, starts=torch.zeros(2, device=dev())),
                dict(left=3, starts=torch.zeros(2, dtype=torch.int32)), dict(left=3, lengths=torch.zeros(2, dtype=torch.int64, device=dev()))):
        with pytest.raises(ValueError):
            spa2.window_attention(q, k, v, **bad)
    for call in (lambda: spa2.window_attention(k, q[:, :, :20], q[:, :, :20], 3), lambda: spa2.window_attention(q.float(), k, v, 3),
                 lambda: spa2.window_attention(_inputs(2, 4, 2, 40, 30, 64)[0], k, v, 3), lambda: spa2.window_attention(q, k, v[:, :, :20], 3)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(spa2.Spa2Error):
        spa2.window_attention(q, k, v, 3, scale=0.0)
