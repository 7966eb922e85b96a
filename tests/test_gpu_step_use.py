"""The operators of a training step in use: captures beside living graphs, two calls at a time, inputs that share memory, saved-tensor
hooks and checkpointing."""
import numpy as np
import pytest
import torch
from torch.utils.checkpoint import checkpoint

import paper_2602_13515_amd as spa2
from gpu_util import dev

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def _gated(t):
    y, n = spa2.gate_add_norm(t, t.mean(-2, keepdim=True).expand_as(t), gate=t[0, 0, 0], scale=t[0, 1, 0], weight=t[0, 1, 1])
    return y + n


CALLS = {
    "window": lambda t: spa2.window_attention(t.bfloat16(), t.bfloat16(), t.bfloat16(), 9, 0, 2),
    "window of few rows": lambda t: spa2.window_attention(t[:, :, :3].bfloat16(), t.bfloat16(), t.bfloat16(), 9, 0, 2),
    "gate": _gated,
    "parameter": lambda t: spa2.gate_add_norm(t.detach(), shift=t[0, 0, 0])[1],
}


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("at", ["leaf", "middle"])
def test_capture_beside_an_eager_graph_of_what_an_input_was_computed_from(name, at):
    """Forward passes only: the backward pass of such a graph would end the process."""
    f = CALLS[name]
    leaf = torch.randn(1, 2, 40, 64, device=dev(), requires_grad=True)
    middle = leaf * 2
    alive = f(middle + 1)
    torch.cuda.synchronize()
    with pytest.raises(RuntimeError, match="eager graph"):
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            f((leaf if at == "leaf" else middle) * 2 + 1)
    assert alive.grad_fn is not None


@pytest.mark.parametrize("name", CALLS)
def test_captured_steps_on_a_computed_input(name):
    """Replayed four times with eager steps between: each equals the eager step on what the inputs hold then."""
    f = CALLS[name]
    leaf = torch.randn(1, 2, 40, 64, device=dev(), requires_grad=True)

    def step():
        y = f(leaf * 2 + 1)
        return [y.detach(), *torch.autograd.grad(y, leaf, torch.ones_like(y))]
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for replay in range(4):
        with torch.no_grad():
            leaf.mul_(1.1)
        want = step()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(held, want):
            assert torch.equal(a, b), replay


@pytest.mark.parametrize("name", CALLS)
def test_capture_behind_a_warm_up_whose_result_is_held(name):
    f = CALLS[name]
    leaf = torch.randn(1, 2, 40, 64, device=dev(), requires_grad=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        held = f(leaf)
        up = torch.ones_like(held)
        held.backward(up)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    leaf.grad = None
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        f(leaf).backward(up)
    for replay in range(3):
        with torch.no_grad():
            leaf.mul_(1.1)
        other = leaf.detach().requires_grad_(True)
        (want,) = torch.autograd.grad(f(other), other, up)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(leaf.grad, want), replay


def _work(seed):
    """Inputs of calls that need workspaces of all kinds, and the calls."""
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g).to(dev())
    q, k, v = (r(2, 900, 4, 64).to(BF).transpose(1, 2).requires_grad_(True) for _ in range(3))
    one, ck, cv = r(3, 4, 1, 128).to(BF), r(3, 2, 9000, 128).to(BF), r(3, 2, 9000, 128).to(BF)
    x, b = r(40, 30, 520).requires_grad_(True), r(40, 30, 520).requires_grad_(True)
    gate, w = r(40, 520).requires_grad_(True), r(520).requires_grad_(True)

    def run():
        o = spa2.window_attention(q, k, v, 300, 0, 70)
        with torch.no_grad():
            few = spa2.window_attention(one, ck, cv, 8000, 0, 4)
        y, n = spa2.gate_add_norm(x, b, gate=gate, weight=w)
        grads = torch.autograd.grad((o, y, n), (q, k, v, x, b, gate, w), (torch.ones_like(o), torch.ones_like(y), n.detach()))
        out = [torch.empty_like(t) for t in grads]
        norm = spa2.clip_gradients(grads, 0.5, out=out)
        return [o.detach(), few, y.detach(), n.detach(), norm, *grads, *out]
    return run


def test_two_streams_at_once():
    runs = [_work(i) for i in range(2)]
    want = [f() for f in runs]
    streams = [torch.cuda.Stream() for _ in runs]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    got = [[], []]
    for _ in range(6):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(runs[i]())
    for s in streams:
        torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    for i in range(2):
        for result in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(result, want[i]))


def test_two_graphs_of_one_memory_pool_and_two_of_their_own():
    """Graphs that take their workspaces from one pool are replayed one after another, those with pools of their own at a time."""
    runs = [_work(i) for i in range(2)]
    want = [f() for f in runs]
    torch.cuda.synchronize()
    for shared in (True, False):
        graphs, held = [torch.cuda.CUDAGraph() for _ in runs], []
        for g, f in zip(graphs, runs):
            with torch.cuda.graph(g, pool=graphs[0].pool() if shared and g is not graphs[0] else None):
                held.append(f())
        streams = [torch.cuda.current_stream()] * 2 if shared else [torch.cuda.Stream() for _ in runs]
        for replay in range(3):
            for t in (x for h in held for x in h):
                t.zero_()
            torch.cuda.synchronize()
            for g, s in zip(graphs, streams):
                with torch.cuda.stream(s):
                    g.replay()
            torch.cuda.synchronize()
            for h, w in zip(held, want):
                assert all(torch.equal(a, b) for a, b in zip(h, w)), (shared, replay)


def test_inputs_that_are_one_tensor():
    """Gradients of an input that is given twice are those of two inputs, added."""
    t = torch.randn(2, 100, 2, 64, device=dev()).to(BF).transpose(1, 2)
    up = torch.randn_like(t)
    for names in ((0, 0, 0), (0, 1, 1)):
        a = [t.clone().requires_grad_(True) for _ in range(max(names) + 1)]
        b = [t.clone().requires_grad_(True) for _ in range(3)]
        oa, ob = (spa2.window_attention(*x, 30, 0, 3) for x in ([a[i] for i in names], b))
        assert torch.equal(oa, ob)
        ga, gb = torch.autograd.grad(oa, a, up), torch.autograd.grad(ob, b, up)
        for i, g in enumerate(ga):
            parts = [x.float() for x, j in zip(gb, names) if j == i]
            # (added by PyTorch in bf16: half a step for each sum)
            assert ((g.float() - sum(parts)).abs() <= 2 * 2.0 ** -8 * sum(p.abs() for p in parts)).all()
    x = torch.randn(3, 50, 200, device=dev())
    p = torch.randn(3, 200, device=dev())
    one, two = [x.clone().requires_grad_(True) for _ in range(2)], [p.clone().requires_grad_(True) for _ in range(3)]
    n = spa2.gate_add_norm(one[0], one[1], gate=two[0], scale=two[1], shift=two[2])[1]
    sx, sp = x.clone().requires_grad_(True), p.clone().requires_grad_(True)
    m = spa2.gate_add_norm(sx, sx, gate=sp, scale=sp, shift=sp)[1]
    assert torch.equal(n, m)
    g = torch.autograd.grad(n, one + two, x)
    gx, gp = torch.autograd.grad(m, (sx, sp), x)
    assert (gx - (g[0] + g[1])).abs().max() <= 2.0 ** -22 * (g[0].abs() + g[1].abs()).max()
    assert (gp - (g[2] + g[3] + g[4])).abs().max() <= 2.0 ** -21 * (g[2].abs() + g[3].abs() + g[4].abs()).max()


def test_broadcast_inputs():
    """Samples that share their keys, a branch that is the same for all tokens: the sums over what was broadcast are PyTorch's."""
    q = torch.randn(3, 2, 70, 64, device=dev()).to(BF)
    k, v, up = (torch.randn(s, 2, 70, 64, device=dev()).to(BF) for s in (1, 1, 3))
    shared = [t.clone().requires_grad_(True) for t in (k, v)]
    whole = [t.expand(3, -1, -1, -1).contiguous().requires_grad_(True) for t in (k, v)]
    o = spa2.window_attention(q, *(t.expand(3, -1, -1, -1) for t in shared), 20, 0, 3)
    w = spa2.window_attention(q, *whole, 20, 0, 3)
    assert torch.equal(o, w)
    for a, b in zip(torch.autograd.grad(o, shared, up), torch.autograd.grad(w, whole, up)):
        # (PyTorch sums three numbers of bf16 and rounds: one step of the largest it holds on the way)
        assert ((a.float() - b.float().sum(0, keepdim=True)).abs() <= 2 * 2.0 ** -8 * b.float().abs().sum(0, keepdim=True)).all()
    x = torch.randn(2, 50, 200, device=dev())
    row = torch.randn(1, 1, 200, device=dev())
    a, b = row.clone().requires_grad_(True), row.expand(2, 50, 200).contiguous().requires_grad_(True)
    y, z = spa2.gate_add_norm(x, a.expand(2, 50, 200))[1], spa2.gate_add_norm(x, b)[1]
    assert torch.equal(y, z)
    ga, gb = torch.autograd.grad(y, a, x)[0], torch.autograd.grad(z, b, x)[0]
    # (a sum of 100 numbers in fp32, whatever the order: 99 roundings at most)
    assert ((ga - gb.double().sum((0, 1), keepdim=True)).abs() <= 100 * 2.0 ** -24 * gb.double().abs().sum((0, 1), keepdim=True)).all()


@pytest.mark.parametrize("name", CALLS)
def test_hooks_and_checkpointing(name):
    f = CALLS[name]
    leaf = torch.randn(1, 2, 40, 64, device=dev(), requires_grad=True)
    y = f(leaf)
    (want,) = torch.autograd.grad(y, leaf, torch.ones_like(y))
    with torch.autograd.graph.save_on_cpu():
        y = f(leaf)
    (got,) = torch.autograd.grad(y, leaf, torch.ones_like(y))
    assert torch.equal(got, want)
    y = checkpoint(f, leaf, use_reentrant=False)
    (got,) = torch.autograd.grad(y, leaf, torch.ones_like(y))
    assert torch.equal(got, want)


@pytest.mark.parametrize("change", ["host", "shorter", "another type"])
def test_hooks_that_bring_back_something_else_are_refused(change):
    """Every saved tensor in turn."""
    def bad(t):
        if change == "host":
            return t.cpu()
        if change == "shorter":
            return t[..., :-1].contiguous()
        return t.double()
    x, b = (torch.randn(2, 5, 64, device=dev(), requires_grad=True) for _ in range(2))
    gate, w = torch.randn(2, 64, device=dev(), requires_grad=True), torch.randn(64, device=dev(), requires_grad=True)
    q, k, v = (torch.randn(2, 2, 100, 64, device=dev()).to(BF).requires_grad_(True) for _ in range(3))
    lengths = torch.tensor([100, 50], dtype=torch.int32, device=dev())
    calls = {"gate": lambda: sum(t.sum() for t in spa2.gate_add_norm(x, b, gate=gate, weight=w, branch_weight=w)),
             "window": lambda: spa2.window_attention(q, k, v, 30, 0, 0, lengths, lengths - 100).float().sum()}
    for name, f in calls.items():
        seen = [0]
        def count(t):
            seen[0] += 1
            return t
        with torch.autograd.graph.saved_tensors_hooks(count, lambda t: t):
            f()
        assert seen[0] >= 6
        for i in range(seen[0]):
            at = [0]

            def pack(t):
                at[0] += 1
                return t.detach(), at[0] - 1
            with torch.autograd.graph.saved_tensors_hooks(pack, lambda p: bad(p[0]) if p[1] == i else p[0]):
                y = f()
            with pytest.raises((ValueError, RuntimeError)):
                y.backward()


def test_empty_calls_and_lists():
    e = lambda *s: torch.empty(s, dtype=BF, device=dev())
    for q, k in ((e(0, 2, 4, 64), e(0, 2, 4, 64)), (e(1, 2, 0, 64), e(1, 2, 4, 64)), (e(1, 2, 4, 64), e(1, 2, 0, 64))):
        with pytest.raises((ValueError, RuntimeError)):
            spa2.window_attention(q, k, k, 3, 0, starts=torch.zeros(len(q), dtype=torch.int32, device=dev()))
    for s in ((0, 64), (3, 0), (0,)):
        with pytest.raises((ValueError, RuntimeError)):
            spa2.gate_add_norm(e(*s))
    with pytest.raises((ValueError, TypeError, RuntimeError)):
        spa2.clip_gradients([torch.ones(3, device=dev()), None], 1.0)
    with pytest.raises(ValueError):
        spa2.clip_gradients([], 1.0)
    t = [torch.ones(3, device=dev()), e(0)]
    assert spa2.clip_gradients((x for x in t), 0.5).item() == np.float32(np.sqrt(3.0))
    assert spa2.gradient_norm([e(0), e(0, 7)]).item() == 0.0
    assert spa2.gradient_norm([t[0]] * 300).item() == pytest.approx(float(spa2.gradient_norm(t[0])) * 300 ** 0.5, rel=1e-6)
