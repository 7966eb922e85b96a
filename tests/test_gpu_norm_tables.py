"""Tables of the rotation that would need a gradient: there is none, and the call says so."""
import pytest
import torch

import paper_2602_13515_amd as spa2
from gpu_util import dev

pytestmark = pytest.mark.gpu


def test_tables_that_need_a_gradient_are_refused():
    import torch.autograd.forward_ad as fwad
    x = torch.randn(1, 2, 8, 64, device=dev())
    leaf = x.clone().requires_grad_(True)
    cos, sin = spa2.rotary_table(8, 64, device=dev())
    want = spa2.qk_norm_rotate(x, x, None, None, cos, sin)
    for tables in ((cos.clone().requires_grad_(True), sin), (cos, sin.clone().requires_grad_(True))):
        for q in (x, leaf):
            with pytest.raises(ValueError, match="gradient"):
                spa2.qk_norm_rotate(q, x, None, None, *tables)
        with torch.no_grad():                               # nobody asks for one
            for a, b in zip(spa2.qk_norm_rotate(x, x, None, None, *tables), want):
                assert torch.equal(a, b)
    for grad in (False, True):
        with torch.set_grad_enabled(grad), fwad.dual_level():
            with pytest.raises(ValueError, match="gradient"):
                spa2.qk_norm_rotate(x, x, None, None, fwad.make_dual(cos, torch.ones_like(cos)), sin)
