"""Training steps in captured graphs: dropout draws other masks at every replay; eager graphs that are still alive."""
import pytest
import torch

import paper_2602_13515_amd as spa2
from paper_2602_13515_amd import distill as vd
from gpu_util import dev

pytestmark = pytest.mark.gpu


def _block(monkeypatch, dropout):
    """A block, and the list that the seeds of its dropout calls go to."""
    torch.manual_seed(3)
    block = vd.ToyBlock(128, 2, grid=(4, 5, 6), context_dim=96, dropout=dropout).to(dev())
    seeds, call = [], vd.dropout_add

    def kept(x, residual, p, seed, *offset):
        seeds.append(seed)
        return call(x, residual, p, seed, *offset)
    monkeypatch.setattr(vd, "dropout_add", kept)
    return block, seeds


def test_captured_training_steps_draw_other_masks(monkeypatch):
    block, seeds = _block(monkeypatch, 0.5)
    params = list(block.parameters())
    x, context, up = torch.randn(2, 120, 128, device=dev()), torch.randn(2, 9, 96, device=dev()), torch.randn(2, 120, 128, device=dev())

    def step():
        y = block(x, context)
        return [y.detach(), *torch.autograd.grad(y, params, up)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()                                              # (warms up, and makes the pattern of full attention)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    seeds.clear()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    captured = list(seeds)
    assert len(captured) == 2 and all(isinstance(s, torch.Tensor) for s in captured)
    seen = []
    for replay in range(4):
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in held]
        now = [s.clone() for s in captured]
        for earlier in seen:
            assert not torch.equal(got[0], earlier[0]) and not any(torch.equal(a, b) for a, b in zip(now, earlier[1]))
        assert not torch.equal(*now)                        # the branches differ
        seen.append((got[0], now))
        # the same step from these very seeds, eagerly
        with monkeypatch.context() as m:
            number, call = iter(now), vd.dropout_add
            m.setattr(vd, "dropout_add", lambda x, r, p, seed, *offset: call(x, r, p, next(number)))
            want = step()
        for a, b in zip(got, want):
            assert torch.equal(a, b), replay


def test_eager_steps_take_their_seed_from_the_host(monkeypatch):
    block, seeds = _block(monkeypatch, 0.5)
    x, context = torch.randn(1, 120, 128, device=dev()), torch.randn(1, 9, 96, device=dev())
    torch.manual_seed(4)
    a = block(x, context)
    torch.manual_seed(4)
    assert torch.equal(a, block(x, context)) and all(isinstance(s, int) for s in seeds)


CALLS = {
    "norm": lambda t: spa2.qk_norm_rotate(t, t)[0],
    "cross": lambda t: spa2.cross_attention(t.bfloat16(), t.bfloat16(), t.bfloat16()),
    "dropout": lambda t: spa2.dropout_add(t, None, 0.5, 1),
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
    f = CALLS[name]
    leaf, up = torch.randn(1, 2, 40, 64, device=dev(), requires_grad=True), torch.randn(1, 2, 40, 64, device=dev())

    def step():
        y = f(leaf * 2 + 1)
        return [y.detach(), *torch.autograd.grad(y, leaf, up.to(y.dtype))]
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for replay in range(3):
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
    """A warm-up on a stream of its own, and then the captured step, as PyTorch's documentation has it."""
    f = CALLS[name]
    leaf, up = torch.randn(1, 2, 40, 64, device=dev(), requires_grad=True), torch.randn(1, 2, 40, 64, device=dev())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        held = f(leaf)
        held.backward(up.to(held.dtype))
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    leaf.grad = None
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        f(leaf).backward(up.to(held.dtype))
    for replay in range(3):
        with torch.no_grad():
            leaf.mul_(1.1)
        other = leaf.detach().requires_grad_(True)
        (want,) = torch.autograd.grad(f(other), other, up.to(held.dtype))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(leaf.grad, want), replay
    assert held.grad_fn is not None
