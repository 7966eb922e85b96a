"""Attention to another sequence where whole blocks of keys have a score of minus infinity: they take no part, wherever they
stand and however many there are, in the kernel for few rows and in the one for many.  The scores overflow in fp32 (bf16 keys of
-1e38 against queries of 100), so that keys and queries are finite and gradients are defined; the bounds are block_ref.cross's."""
import numpy as np
import pytest
import torch

import block_ref as ref
import paper_2602_13515_amd as spa2
from gpu_util import dev

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def f64(t):
    return t.detach().double().cpu().numpy()


def _inputs(B, Hq, Hk, Nq, Nk, d, lost):
    """Keys `lost` have a score of minus infinity for every second query, and an ordinary one for the others."""
    g = torch.Generator().manual_seed(Nq + 3 * Nk + d)
    q, k, v, do = (torch.randn((B, H, N, d), generator=g) for H, N in ((Hq, Nq), (Hk, Nk), (Hk, Nk), (Hq, Nq)))
    k[..., 0] = 0
    for a, b in lost:
        k[:, :, a:b, 0] = -1e38
    q[..., 0] = 0
    q[:, :, ::2, 0] = 100
    return [x.to(BF).to(dev()) for x in (q, k, v, do)]


CASES = [
    # B, Hq, Hk, Nq, Nk, d, stretches of lost keys, lengths
    (1, 2, 2, 40, 70, 64, [(0, 64)], None),
    (1, 2, 2, 40, 70, 128, [(0, 64)], None),
    (1, 2, 2, 3, 70, 128, [(0, 64)], None),
    (2, 2, 1, 130, 300, 64, [(0, 64), (128, 192)], [300, 65]),
    (2, 2, 1, 130, 300, 128, [(0, 200)], [300, 201]),
    (2, 4, 2, 2, 300, 64, [(0, 64), (100, 228)], [300, 65]),
    (1, 2, 1, 100, 9000, 128, [(0, 4000)], None),                # cut into parts, of which some are lost
    (1, 2, 1, 100, 9000, 64, [(5000, 9000)], None),
    (2, 2, 2, 1, 9000, 128, [(0, 4000), (6000, 8990)], [9000, 4001]),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "x".join(map(str, c[:6])))
def test_blocks_of_lost_keys(case):
    print("case", case, flush=True)
    *sizes, lost, lengths = case
    q, k, v, do = _inputs(*sizes, lost)
    lens = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device=dev())
    scale = q.shape[-1] ** -0.5
    with np.errstate(over="ignore", under="ignore"):
        want, _ = ref.cross(f64(q), f64(k), f64(v), None if lens is None else np.array(lengths), scale, f64(do))
    leaves = [t.detach().requires_grad_(True) for t in (q, k, v)]
    o = spa2.cross_attention(*leaves, lens, scale)
    for name, t in zip(("o", "dq", "dk", "dv"), (o, *torch.autograd.grad(o, leaves, do))):
        value, bound = want[name]
        x = f64(t)
        assert np.isfinite(x).all(), name
        assert (np.abs(x - value) <= bound + 1e-30).all(), (name, (np.abs(x - value) - bound).max())


def test_keys_of_minus_infinity_themselves():
    for Nq in (3, 40):
        q, k, v, _ = _inputs(2, 2, 2, Nq, 200, 64, [])
        q[..., 0] = q[..., 0].abs() + 1
        k[:, :, :130, 0] = float("-inf")
        want, _ = ref.cross(f64(q), f64(k[:, :, 130:]), f64(v[:, :, 130:]), None, 0.125)
        value, bound = want["o"]
        assert (np.abs(f64(spa2.cross_attention(q, k, v)) - value) <= bound).all(), Nq


@pytest.mark.parametrize("Nq", [3, 40])
def test_no_score_at_all_is_not_a_number(Nq):
    """softmax of minus infinities, as ever; the other rows are as they were"""
    q, k, v, _ = _inputs(1, 2, 2, Nq, 100, 64, [(0, 100)])
    o = spa2.cross_attention(q, k, v)
    assert torch.isnan(o[:, :, ::2]).all() and torch.isfinite(o[:, :, 1::2]).all()


@pytest.mark.parametrize("d", [64, 128])
def test_block_sparse_rows_that_begin_with_lost_blocks(d):
    """The block-sparse forward pass over every block: the same."""
    q, k, v, _ = _inputs(1, 2, 2, 300, 300, d, [(0, 192)])
    pattern = spa2.alloc_pattern(1, 2, 300, dev())
    spa2.spa2_pattern_full(q, pattern)
    with torch.no_grad():
        o = spa2.sparge_attn2(q, k, v, 0.0, 0.0, pattern=pattern)
    with np.errstate(under="ignore"):
        want, _ = ref.cross(f64(q), f64(k), f64(v), None, d ** -0.5)
    value, bound = want["o"]
    assert (np.abs(f64(o) - value) <= bound).all()
