"""The C functions of the operators around the attention, called through the binding: a tensor that lies elsewhere than the others,
or a log-sum-exp of another size, is refused before its address reaches a kernel.  (Without a GPU: tensors on the CPU, and one of
them on PyTorch's device without memory.)"""
import pytest
import torch

from paper_2602_13515_amd import binding

BF, F = torch.bfloat16, torch.float32


def _norm():
    t = dict(q=torch.zeros(2, 4, 10, 64), k=torch.zeros(2, 2, 10, 64), q_weight=torch.ones(64), k_weight=torch.ones(64),
             cos=torch.ones(10, 32), sin=torch.zeros(10, 32), positions=torch.zeros(2, 10, dtype=torch.int32))
    outs = dict(q_out=torch.zeros(2, 4, 10, 64, dtype=BF), k_out=torch.zeros(2, 2, 10, 64, dtype=BF))
    return {**t, "eps": 1e-6, "interleaved": False, **outs}, binding.spa2_norm_rotate


def _norm_bwd():
    t, _ = _norm()
    t["d_q_out"], t["d_k_out"] = t.pop("q_out"), t.pop("k_out")
    return {**t, "dq": torch.zeros(2, 4, 10, 64), "dk": torch.zeros(2, 2, 10, 64), "d_q_weight": torch.ones(64),
            "d_k_weight": torch.ones(64), "workspace": torch.zeros(1 << 16, dtype=torch.uint8)}, binding.spa2_norm_rotate_bwd


def _cross():
    q, k = torch.zeros(2, 4, 10, 64, dtype=BF), torch.zeros(2, 2, 20, 64, dtype=BF)
    return dict(q=q, k=k, v=k.clone(), lengths=torch.zeros(2, dtype=torch.int32), scale=0.1, o=q.clone(), lse=torch.zeros(2, 4, 10),
                o_res=q.clone(), workspace=torch.zeros(16, dtype=torch.uint8)), binding.spa2_cross_fwd


def _cross_bwd():
    t, _ = _cross()
    return {**t, "d_o": t["q"].clone(), "dq": t["q"].clone(), "dk": t["k"].clone(), "dv": t["k"].clone(),
            "workspace": torch.zeros(1 << 16, dtype=torch.uint8)}, binding.spa2_cross_bwd


def _drop():
    return dict(x=torch.zeros(8), residual=torch.zeros(8), p=0.5, seed=1, offset=2, y=torch.zeros(8),
                seed_offset=torch.zeros(2, dtype=torch.int64)), binding.spa2_dropout_add


def _drop_bwd():
    return dict(d_y=torch.zeros(8), p=0.5, seed=1, offset=2, dx=torch.zeros(8),
                seed_offset=torch.zeros(2, dtype=torch.int64)), binding.spa2_dropout_bwd


CALLS = [_norm, _norm_bwd, _cross, _cross_bwd, _drop, _drop_bwd]
NAMED = [(f, n) for f in CALLS for n, t in f()[0].items() if isinstance(t, torch.Tensor)]


@pytest.mark.parametrize("make,name", NAMED, ids=[f"{f.__name__[1:]}-{n}" for f, n in NAMED])
def test_a_tensor_elsewhere_is_refused(make, name):
    args, call = make()
    args[name] = args[name].to("meta")
    with pytest.raises(ValueError, match="one GPU"):
        call(**args)


@pytest.mark.parametrize("make", CALLS, ids=lambda f: f.__name__[1:])
def test_host_tensors_are_refused(make):
    args, call = make()
    with pytest.raises(ValueError, match="GPU only"):
        call(**args)


@pytest.mark.parametrize("make", [_cross, _cross_bwd], ids=lambda f: f.__name__[1:])
def test_a_log_sum_exp_of_another_kind_is_refused(make, monkeypatch):
    monkeypatch.setattr(binding, "_one_gpu", lambda *tensors: None)          # (the device is not what is tested here)
    for bad in (torch.zeros(2, 4, 9), torch.zeros(2, 4, 10, dtype=torch.float64), torch.zeros(2, 10, 4).transpose(1, 2), torch.zeros(80)):
        args, call = make()
        with pytest.raises(ValueError, match="log-sum-exp"):
            call(**{**args, "lse": bad})
