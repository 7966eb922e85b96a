"""A training step of the distillation block with its gates, modulated norms, attention over a window and clipped gradients: the three
operators together, as they are used."""
import copy
import math

import pytest
import torch

import paper_2602_13515_amd as spa2
from paper_2602_13515_amd import distill as vd
from gpu_util import REL_L2, dev

pytestmark = pytest.mark.gpu


def _plain_gate_add_norm(x, branch=None, gate=None, branch_weight=None, weight=None, bias=None, scale=None, shift=None, kind="layer",
                         eps=1e-6, dtype=None):
    wide = lambda p: p if p.dim() == 1 else p[:, None]
    y = x if branch is None else x + (1.0 if gate is None else wide(gate)) * branch
    if kind is None:
        return y, None
    n = (y - y.mean(-1, keepdim=True)) * (y.var(-1, keepdim=True, unbiased=False) + eps).rsqrt() * weight + bias
    return y, n if scale is None else n * (1 + wide(scale)) + wide(shift)


def _plain_window(q, k, v, left, right, sinks):
    """In fp32, from the same bf16 q, k and v."""
    n = q.shape[2]
    i, j = torch.arange(n, device=q.device)[:, None], torch.arange(n, device=q.device)[None]
    sees = torch.ones(n, n, dtype=torch.bool, device=q.device)
    if right is not None:
        sees &= j <= i + right
    if left is not None:
        sees &= (j >= i - left) | (j < sinks)
    qf, kf, vf = q.float(), k.float(), v.float()
    s = (torch.matmul(qf, kf.transpose(2, 3).contiguous()) / math.sqrt(q.shape[3])).masked_fill(~sees, -math.inf)
    return torch.matmul(torch.softmax(s, -1), vf).to(torch.bfloat16)


def _block(**more):
    torch.manual_seed(1)
    block = vd.ToyBlock(128, 2, gated=True, **more).to(dev())
    with torch.no_grad():
        for p in block.parameters():
            p.add_(0.1 * torch.randn_like(p))
    return block


BLOCKS = {
    "window": dict(window=(60, 0, 4)),
    "window and condition": dict(window=(30, 20, 0), condition_dim=48),
    "context": dict(window=(None, 0, 0), context_dim=96, grid=(4, 5, 11)),
    "context and condition": dict(window=(100, 0, 1), context_dim=96, condition_dim=48, grid=(4, 5, 11)),
}


def _inputs(more, B=2, N=220):
    torch.manual_seed(2)
    x = torch.randn(B, N, 128, device=dev())
    args = {}
    if "context_dim" in more:
        args["context"], args["lengths"] = torch.randn(B, 9, 96, device=dev()), torch.tensor([9, 4], dtype=torch.int32, device=dev())
    if "condition_dim" in more:
        args["condition"] = torch.randn(B, 48, device=dev())
    return x, args, torch.randn(B, N, 128, device=dev())


@pytest.mark.parametrize("name", BLOCKS)
def test_block_against_plain_operators(name, monkeypatch):
    """Both sides take the same bf16 q, k and v.  The results differ by the attention's rounding, a relative REL_L2 in the 2-norm at
    most, the gradients by that of its four results (O, dQ, dK, dV): four times as much."""
    block = _block(**BLOCKS[name])
    x, args, up = _inputs(BLOCKS[name])
    x.requires_grad_(True)
    leaves = [x, *block.parameters()]

    def step():
        y = block(x, **args)
        return [y.detach(), *torch.autograd.grad(y, leaves, up)]
    got = step()
    with monkeypatch.context() as m:
        m.setattr(vd, "gate_add_norm", _plain_gate_add_norm)
        m.setattr(vd, "window_attention", _plain_window)
        want = step()
    for what, a, b in zip(["y", "x", *(n for n, _ in block.named_parameters())], got, want):
        assert torch.isfinite(a).all(), what
        assert (a - b).norm() <= (1 if what == "y" else 4) * REL_L2 * b.norm() + 1e-6, (what, float((a - b).norm() / b.norm()))


def test_gates_of_one_are_the_block_without():
    """Same sums and norms, in other kernels: fp32 roundings, some of which reach the other side of a bf16 rounding of q, k and v."""
    block = vd.ToyBlock(128, 2, window=(50, 0, 2)).to(dev())
    gated = vd.ToyBlock(128, 2, window=(50, 0, 2), gated=True).to(dev())
    gated.load_state_dict({**block.state_dict(), "gates": torch.ones(1, 128)})
    x = torch.randn(2, 150, 128, device=dev())
    a, b = block(x), gated(x)
    assert (a - b).norm() <= REL_L2 * a.norm()


def test_dropout_of_gated_branches():
    block = _block(window=(30, 0, 0), context_dim=96, dropout=0.5)
    x, args, _ = _inputs(dict(context_dim=96))
    torch.manual_seed(7)
    a = block(x, **args)
    torch.manual_seed(7)
    assert torch.equal(a, block(x, **args)) and not torch.equal(a, block(x, **args))
    block.eval()
    assert torch.equal(block(x, **args), block(x, **args))


def test_distillation_clips_its_gradients():
    """Sparse and window students; what the optimizer gets is the gradient of the loss, scaled to the largest norm."""
    torch.manual_seed(3)
    batches = [(torch.randn(2, 300, 128, device=dev()), torch.randn(2, 300, 128, device=dev()), torch.rand(2, device=dev()), None, None,
                torch.randn(2, 16, device=dev())) for _ in range(3)]
    for window in (None, (64, 0, 8)):
        teacher = vd.ToyBlock(128, 2, gated=True, condition_dim=16).to(dev())
        student = vd.make_student(teacher, 0.2, 0.5, window=window)
        reference = copy.deepcopy(student)
        x1, x0, t, *more = batches[0]
        xt = vd.noisy_latent(x1, x0, t)
        with torch.no_grad():
            u = teacher(xt, *more)
        vd.velocity_distillation_loss(reference(xt, *more), u).backward()
        norm = math.sqrt(sum(float((p.grad.double() ** 2).sum()) for p in reference.parameters()))
        seen = []
        limit = norm / 3
        hook = lambda step, loss: seen.append([p.grad.clone() for p in student.parameters()])
        r = vd.distill(student, teacher, batches, lr=1e-4, on_step=hook, max_norm=limit)
        assert len(r["loss"]) == len(r["norm"]) == 3 and all(math.isfinite(x) for x in r["loss"] + r["norm"])
        assert abs(r["norm"][0] - norm) <= 1e-5 * norm
        for g, p in zip(seen[0], reference.parameters()):
            assert torch.allclose(g, p.grad * (limit / (norm + 1e-6)), rtol=1e-5, atol=1e-12)
        for grads, n in zip(seen, r["norm"]):
            after = math.sqrt(sum(float((g.double() ** 2).sum()) for g in grads))
            assert after <= limit * (1 + 1e-6) and (n > limit) == (after < n * (1 - 1e-7))
        assert "norm" not in vd.distill(student, teacher, batches[:1])


def test_captured_step_with_clipping():
    """Forward, backward, clipping and an update in one graph, replayed, against the same steps eagerly."""
    def make():
        block = _block(window=(60, 0, 4), condition_dim=48)
        return block, torch.optim.SGD(block.parameters(), lr=0.05)
    x, args, up = _inputs(dict(condition_dim=48))

    def step(block, opt):
        opt.zero_grad(set_to_none=False)
        block(x, **args).backward(up)
        norm = spa2.clip_gradients([p.grad for p in block.parameters()], 0.5)
        opt.step()
        return norm
    eager, opt = make()
    captured, copt = make()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for b, o in ((eager, opt), (captured, copt)):
            step(b, o)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step(captured, copt)
    for replay in range(3):
        want = step(eager, opt)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(held, want), replay
        for a, b in zip(captured.parameters(), eager.parameters()):
            assert torch.equal(a, b) and torch.equal(a.grad, b.grad), replay
