"""Attention to another sequence for few query rows keeps what a rounding of the probabilities to bf16 drops: what is left is the
rounding of the result, in the 2-norm, and of fp32 in the log-sum-exp."""
import numpy as np
import pytest
import torch

import block_ref as ref
import paper_2602_13515_amd as spa2
from gpu_util import dev

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
CASES = [
    # B, Hq, Hk, Nq, Nk, d, lengths
    (2, 2, 2, 1, 5, 128, None),
    (1, 6, 6, 8, 4, 128, None),
    (2, 5, 1, 3, 20, 64, [20, 3]),
    (1, 2, 2, 1, 300, 64, None),
    (3, 8, 2, 8, 1000, 128, [1000, 65, 0]),
    (4, 4, 4, 32, 90, 64, [90, 64, 2, 33]),
    (2, 10, 2, 1, 9000, 128, [9000, 4097]),
    (300, 1, 1, 1, 70, 64, None),
]


def f64(t):
    return t.detach().double().cpu().numpy()


@pytest.mark.parametrize("case", CASES, ids=str)
def test_results_of_few_rows(case):
    B, Hq, Hk, Nq, Nk, d, lengths = case
    g = torch.Generator().manual_seed(Nq + Nk + d)
    q, k, v = (torch.randn((B, H, N, d), generator=g).to(BF).to(dev()) for H, N in ((Hq, Nq), (Hk, Nk), (Hk, Nk)))
    lens = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device=dev())
    want, lse = ref.cross(f64(q), f64(k), f64(v), None if lengths is None else np.array(lengths), d ** -0.5)
    value = want["o"][0]
    rounding = np.linalg.norm(f64(torch.from_numpy(value).float().to(BF)) - value)
    # P in two parts has 16 bits, a relative error of 2^-17: 1.1 of the result's own rounding, about 2^-9.2 of it, allows an error
    # of 0.46 of that besides, 2^-10.3 (with P in one part the two are alike where no sum averages them)
    o, got = torch.empty_like(q), torch.empty(q.shape[:3], device=dev())
    ws = torch.empty(max(spa2.spa2_cross_fwd_workspace_bytes(q, k), 16), dtype=torch.uint8, device=dev())
    spa2.spa2_cross_fwd(q, k, v, lens, d ** -0.5, o, got, None, ws)
    err = np.linalg.norm(f64(o) - value)
    print(f"error / rounding of the result: {err / rounding:.3f}", flush=True)
    assert err <= 1.1 * rounding, (err, rounding)
    # scores: d products in fp32 and the scaling; the sum: Nk terms, by as many lanes as there are and some joins; both logarithms'
    # units: far below 2^-13, which the bounds of block_ref grant them
    some = np.isfinite(lse)
    assert np.array_equal(np.isneginf(f64(got)), ~some)
    assert (np.abs(f64(got)[some] - lse[some]) <= 2.0 ** -13).all()
