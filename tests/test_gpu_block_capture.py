"""Training steps of the block in captured graphs: dropout draws other masks at every replay."""
import pytest
import torch

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
