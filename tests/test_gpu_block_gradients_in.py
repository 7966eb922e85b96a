"""Upstream gradients and weights that start anywhere in memory: the backward of a concatenation, for one, hands out views of its
buffer at any element.  The results are those of the same numbers on an aligned address, bit for bit."""
import pytest
import torch

import paper_2602_13515_amd as spa2
from gpu_util import dev

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def _shifted(t, by):
    """t's numbers in t's strides, `by` elements behind the start of an allocation."""
    store = torch.empty(t.numel() + by, dtype=t.dtype, device=t.device)
    return store.as_strided(t.shape, t.stride(), by).copy_(t)


def _heads(B, H, N, d, dtype=BF):
    return torch.randn((B, N, H, d), device=dev()).to(dtype).permute(0, 2, 1, 3)


@pytest.mark.parametrize("by", [1, 4])
@pytest.mark.parametrize("Nq,Nk", [(3, 90), (150, 50), (150, 90)])
def test_attention_to_another_sequence(Nq, Nk, by):
    torch.manual_seed(Nq + Nk)
    leaves = [x.requires_grad_(True) for x in (_heads(2, 4, Nq, 64), _heads(2, 2, Nk, 64), _heads(2, 2, Nk, 64))]
    up = _heads(2, 4, Nq, 64)
    odd = _shifted(up, by)
    assert odd.stride() == up.stride() and odd.data_ptr() % 16
    want = torch.autograd.grad(spa2.cross_attention(*leaves), leaves, up)
    got = torch.autograd.grad(spa2.cross_attention(*leaves), leaves, odd)
    for a, b in zip(got, want):
        assert torch.equal(a, b)


@pytest.mark.parametrize("by", [1, 4])
@pytest.mark.parametrize("dtype", [BF, torch.float32])
def test_norm_and_rotation(dtype, by):
    torch.manual_seed(by)
    cos, sin = spa2.rotary_table(33, 64, device=dev())
    leaves = [_heads(2, 4, 33, 64, dtype), _heads(2, 2, 33, 64, dtype), torch.randn(64, device=dev()), torch.randn(64, device=dev())]
    leaves = [x.requires_grad_(True) for x in leaves]
    ups = [_heads(2, 4, 33, 64), _heads(2, 2, 33, 64)]
    odd = [_shifted(t, by) for t in ups]
    assert all(t.data_ptr() % 16 for t in odd)
    want = torch.autograd.grad(spa2.qk_norm_rotate(*leaves, cos, sin), leaves, ups)
    for ups in (odd, (odd[0], ups[1]), (ups[0], odd[1])):
        got = torch.autograd.grad(spa2.qk_norm_rotate(*leaves, cos, sin), leaves, ups)
        for a, b in zip(got, want):
            assert torch.equal(a, b)


def test_behind_a_concatenation():
    torch.manual_seed(5)
    q, k = (torch.randn((1, 2, 40, 64), device=dev()).to(BF).requires_grad_(True) for _ in range(2))
    head, up = torch.zeros(3, dtype=BF, device=dev()), torch.randn(3 + q.numel(), device=dev()).to(BF)
    for f in (lambda: spa2.cross_attention(q, k, k), lambda: spa2.qk_norm_rotate(q, k)[0]):
        want = torch.autograd.grad(f(), (q, k), up[3:].clone().view(q.shape))
        got = torch.autograd.grad(torch.cat([head, f().flatten()]), (q, k), up)
        for a, b in zip(got, want):
            assert torch.equal(a, b)


@pytest.mark.parametrize("by", [1, 2])
def test_weights_of_the_norm(by):
    torch.manual_seed(by)
    q, k, w = _heads(2, 4, 33, 128), _heads(2, 2, 33, 128), [torch.randn(128, device=dev()).requires_grad_(True) for _ in range(2)]
    odd = [_shifted(t.detach(), by).requires_grad_(True) for t in w]
    ups = [_heads(2, 4, 33, 128), _heads(2, 2, 33, 128)]
    results = []
    for weights in (w, odd):
        out = spa2.qk_norm_rotate(q, k, *weights)
        results.append([*(y.detach() for y in out), *torch.autograd.grad(out, weights, ups)])
    for a, b in zip(*results):
        assert torch.equal(a, b)


@pytest.mark.parametrize("overlap", [False, True])
@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("by", [1, 4])
def test_block_sparse_attention(by, given, overlap):
    torch.manual_seed(by)
    leaves = [_heads(1, 2, 300, 64).requires_grad_(True) for _ in range(3)]
    pattern = spa2.build_pattern(leaves[0].detach(), leaves[1].detach(), 0.5, 0.5) if given else None
    up = _heads(1, 2, 300, 64)
    want, got = (torch.autograd.grad(spa2.sparge_attn2(*leaves, 0.5, 0.5, pattern=pattern, overlap_backward=overlap), leaves, g)
                 for g in (up, _shifted(up, by)))
    for a, b in zip(got, want):
        assert torch.equal(a, b)
