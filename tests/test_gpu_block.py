"""The operators together, as a transformer block uses them: norm and rotation, attention, dropout with the residual sum,
attention to a padded batch of prompts, dropout again; against the same block in plain PyTorch in fp64."""
import copy

import numpy as np
import pytest
import torch

import block_ref as ref
from paper_2602_13515_amd import distill as vd
from gpu_util import REL_L2, dev

pytestmark = pytest.mark.gpu


def _rotate(x, cos, sin):
    a, b = x[..., 0::2], x[..., 1::2]
    return torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)


def _attend(q, k, v, lengths=None):
    s = q @ k.transpose(-1, -2) / q.shape[-1] ** 0.5
    if lengths is not None:
        s = s.masked_fill(torch.arange(k.shape[2])[None, None, None] >= lengths[:, None, None, None], float("-inf"))
        p = torch.where((lengths > 0)[:, None, None, None], torch.softmax(s.where((lengths > 0)[:, None, None, None], torch.zeros_like(s)), -1), 0.0)
    else:
        p = torch.softmax(s, -1)
    return p @ v


def _plain(block, x, context, lengths, seed):
    """block: an fp64 copy on the CPU, full attention."""
    B, N, C = x.shape
    H, d, p = block.heads, C // block.heads, block.dropout

    def heads(t):
        return t.view(B, -1, H, d).permute(0, 2, 1, 3)

    def add(x, branch, number):
        if seed is None:
            return x + branch
        keep, factor = ref.keep_mask(branch.numel(), p, seed, number)
        return x + branch * torch.from_numpy(keep.reshape(branch.shape) * factor)

    q, k, v = (heads(t) for t in block.qkv(block.norm(x)).chunk(3, -1))
    unit = lambda t: t * (t.square().mean(-1, keepdim=True) + 1e-6).rsqrt()
    q, k = (_rotate(unit(t) * w, block.cos, block.sin) for t, w in ((q, block.q_weight), (k, block.k_weight)))
    x = add(x, block.proj(_attend(q, k, v).permute(0, 2, 1, 3).reshape(B, N, C)), 0)
    q = heads(block.context_q(block.context_norm(x)))
    k, v = (heads(t) for t in block.context_kv(context).chunk(2, -1))
    return add(x, block.context_proj(_attend(q, k, v, lengths).permute(0, 2, 1, 3).reshape(B, N, C)), 1)


def _setup(dim, heads, grid, M, dropout):
    torch.manual_seed(dim + M)
    block = vd.ToyBlock(dim, heads, grid=grid, context_dim=96, dropout=dropout)
    with torch.no_grad():
        block.q_weight.copy_(1 + 0.5 * torch.randn(dim // heads)), block.k_weight.copy_(1 + 0.5 * torch.randn(dim // heads))
        block.context_q.weight.mul_(4.0)
    B, N = 3, int(np.prod(grid))
    x, context = torch.randn(B, N, dim), torch.randn(B, M, 96)
    return block, x, context, torch.tensor([M, 0, M // 2], dtype=torch.int32)


@pytest.mark.parametrize("dropout", [0.0, 0.3])
@pytest.mark.parametrize("dim,heads,grid,M", [(128, 2, (3, 5, 9), 40), (256, 2, (1, 7, 31), 77)])
def test_block_against_plain_pytorch(dim, heads, grid, M, dropout):
    """Two attentions in a row, each within REL_L2 of its own, and the operands of both rounded to bf16 (2^-8): three such bars
    for the result's branches and for every gradient."""
    block, x, context, lengths = _setup(dim, heads, grid, M, dropout)
    up = torch.randn_like(x)
    plain = copy.deepcopy(block).double()
    plain.cos, plain.sin = block.cos.double(), block.sin.double()
    mine = copy.deepcopy(block).to(dev())
    torch.manual_seed(11)
    y = mine(x.to(dev()), context.to(dev()), lengths.to(dev()))
    y.backward(up.to(dev()))
    torch.manual_seed(11)
    seed = int(torch.randint(2 ** 63 - 1, ()).item()) if dropout else None
    want = _plain(plain, x.double(), context.double(), lengths, seed)
    want.backward(up.double())
    bar = 3 * REL_L2
    err = (y.detach().cpu().double() - want).norm() / (want - x.double()).norm()
    assert err <= bar, err
    for (name, a), b in zip(mine.named_parameters(), plain.parameters()):
        err = (a.grad.cpu().double() - b.grad).norm() / b.grad.norm()
        print(f"{name}: {err:.1e}", flush=True)
        assert err <= bar, (name, err)


def test_dropout_is_of_training_mode_and_follows_the_generator():
    block, x, context, lengths = _setup(128, 1, (40,), 9, 0.5)
    block, args = block.to(dev()), [t.to(dev()) for t in (x, context, lengths)]
    torch.manual_seed(1)
    a, b = block(*args), block(*args)
    torch.manual_seed(1)
    c = block(*args)
    assert torch.equal(a, c) and not torch.equal(a, b)
    block.eval()
    assert torch.equal(block(*args), block(*args))


def test_distillation_with_context_and_dropout_runs():
    teacher, x, context, lengths = _setup(128, 2, (4, 8, 16), 30, 0.0)
    teacher = teacher.to(dev())
    student = vd.make_student(teacher, 0.3, 0.5, dropout=0.1)
    before = copy.deepcopy(student.state_dict())
    batch = (x.to(dev()), torch.randn_like(x).to(dev()), torch.rand(3, device=dev()), context.to(dev()), lengths.to(dev()))
    hist = vd.distill(student, teacher, [batch, batch], lr=1e-3)
    assert len(hist["loss"]) == 2 and all(np.isfinite(hist["loss"])) and teacher.dropout == 0.0
    for name, p in student.named_parameters():
        assert torch.isfinite(p).all() and not torch.equal(p, before[name]), name


def test_one_token_after_another_equals_all_at_once():
    """Serving: norm and rotation of single tokens at their positions and attention to a cache that grows, against the whole
    sequence at once (each query against the keys up to its own position)."""
    import paper_2602_13515_amd as spa2
    g = torch.Generator(device=dev()).manual_seed(2)
    B, Hq, Hk, N, d = 3, 4, 2, 70, 64
    q, k, v = (torch.randn((B, N, h, d), generator=g, device=dev()).bfloat16().permute(0, 2, 1, 3) for h in (Hq, Hk, Hk))
    wq, wk = (1 + 0.1 * torch.randn(d, generator=g, device=dev()) for _ in range(2))
    start = torch.tensor([0, 5, 1000], device=dev())
    cos, sin = spa2.rotary_table(1100, d, device=dev())
    qr, kr = spa2.qk_norm_rotate(q, k, wq, wk, cos, sin, start[:, None] + torch.arange(N, device=dev()))
    cache_k, cache_v = (torch.full((B, Hk, N, d), float("nan"), dtype=torch.bfloat16, device=dev()) for _ in range(2))
    for n in range(N):
        qn, kn = spa2.qk_norm_rotate(q[:, :, n:n + 1], k[:, :, n:n + 1], wq, wk, cos, sin, start[:, None] + n)
        assert torch.equal(qn, qr[:, :, n:n + 1]) and torch.equal(kn, kr[:, :, n:n + 1])
        cache_k[:, :, n:n + 1], cache_v[:, :, n:n + 1] = kn, v[:, :, n:n + 1]
        if n % 23:
            continue
        o = spa2.cross_attention(qn, cache_k, cache_v, torch.full((B,), n + 1, dtype=torch.int32, device=dev()))
        f64 = lambda t: t.double().cpu().numpy()
        want, _ = ref.cross(f64(qn), f64(kr[:, :, :n + 1]), f64(v[:, :, :n + 1]), None, d ** -0.5)
        value, bound = want["o"]
        assert (np.abs(f64(o) - value) <= bound).all(), n
