"""Norm and rotation of layers whose results are stored past the memory-side cache (more than 256 MiB read and written): every
row as in a call on few tokens, bit for bit, and the weights' gradients against sums in 64 bits."""
import pytest
import torch

import paper_2602_13515_amd as spa2
from gpu_util import dev

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [BF, torch.float32], ids=str)
def test_large_layers_equal_their_pieces(dtype, d, interleaved):
    Hq, Hk = 24 * 128 // d, 8 * 128 // d
    N = 17_003 if dtype == BF else 11_501
    size = torch.finfo(dtype).bits // 8
    piece = 4_999
    # (bytes of the forward pass, which are fewer than those of the backward pass)
    assert N * (Hq + Hk) * d * (size + 2) > 256 << 20 > piece * (Hq + Hk) * d * (2 * size + 2)
    g = torch.Generator(device=dev()).manual_seed(d + size)

    def heads(H, t):
        return torch.randn((1, N, H, d), generator=g, device=dev()).to(t).permute(0, 2, 1, 3)
    q, k, ups = heads(Hq, dtype), heads(Hk, dtype), [heads(Hq, BF), heads(Hk, BF)]
    weights = [1 + 0.3 * torch.randn(d, generator=g, device=dev()) for _ in range(2)]
    cos, sin = spa2.rotary_table(N, d, device=dev())

    def step(at, stop):
        leaves = [t.detach().requires_grad_(True) for t in (q[:, :, at:stop], k[:, :, at:stop], *weights)]
        out = spa2.qk_norm_rotate(*leaves, cos[at:stop], sin[at:stop], interleaved=interleaved)
        return [t.detach() for t in out] + list(torch.autograd.grad(out, leaves, [t[:, :, at:stop] for t in ups]))
    whole = step(0, N)
    for at in range(0, N, piece):
        stop = min(at + piece, N)
        for x, y in zip(whole[:4], step(at, stop)):
            assert torch.equal(x[:, :, at:stop], y), at
    i = torch.arange(d // 2, device=dev())
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + d // 2)
    c, s = cos.double(), sin.double()
    for x, up, got in ((q, ups[0], whole[4]), (k, ups[1], whole[5])):
        total, size_of = torch.zeros(d, dtype=torch.float64, device=dev()), torch.zeros(d, dtype=torch.float64, device=dev())
        for h in range(x.shape[1]):
            xd, ud = x[0, h].double(), up[0, h].double()
            hat = xd * (xd.square().mean(-1, keepdim=True) + 1e-6).rsqrt()
            dn, mag = torch.empty_like(ud), torch.empty_like(ud)
            dn[:, a], dn[:, b] = c * ud[:, a] + s * ud[:, b], c * ud[:, b] - s * ud[:, a]
            mag[:, a] = mag[:, b] = ud[:, a].abs() + ud[:, b].abs()
            total += (dn * hat).sum(0)
            size_of += (mag * hat.abs()).sum(0)
        # as for the smaller layers: at most one fp32 addition a row on top of a term's own roundings, then the result's
        bar = 2.0 ** -24 * total.abs() + (x.shape[1] * N + 64) * 2.0 ** -24 * size_of
        assert ((got.double() - total).abs() <= bar).all()
        # (and what the order of the sums makes of it: a workgroup's walk of at most N terms, the rest in 64 bits.  Errors that
        # are as often up as down stay below the square root of their number, times 6)
        assert ((got.double() - total).abs() <= 6 * (x.shape[1] * N) ** 0.5 * 2.0 ** -24 * size_of).all()
