"""The operators of a training step, without a GPU: refusals of the C entry points and of the binding, the formulas that their GPU tests
compare with, against differences."""
import ctypes
import os
import shutil
import subprocess
import tempfile

import numpy as np
import pytest
import torch

import paper_2602_13515_amd as spa2
import step_ref as ref
from paper_2602_13515_amd import binding

FAKE, ODD = 0x1000, 0x1001             # neither is read
BF, F = torch.bfloat16, torch.float32
CROSS = dict(B=2, Hq=4, Hk=2, Nq=10, Nk=20, d=128, q_sb=5120, q_sh=128, q_sn=512, k_sb=5120, k_sh=128, k_sn=256,
             d_sb=5120, d_sh=128, d_sn=256)


def _window_call(null=None, odd=None, scale=0.1, backward=False, ws_bytes=1 << 60, left=5, right=0, sinks=3, **change):
    s, w = binding._CrossShape(**{**CROSS, **change}), binding._Window(left, right, sinks)
    at = lambda n: None if n == null else (ODD if n == odd else FAKE)
    if backward:
        args = [at(n) for n in ("q", "k", "v", "lengths", "starts", "o", "o_res", "d_o", "lse")]
        return binding._load().spa2_window_bwd(*args, ctypes.byref(s), ctypes.byref(w), scale, at("dq"), at("dk"), at("dv"),
                                               at("workspace"), ws_bytes, None)
    args = [at(n) for n in ("q", "k", "v", "lengths", "starts")]
    return binding._load().spa2_window_fwd(*args, ctypes.byref(s), ctypes.byref(w), scale, at("o"), at("o_res"), at("lse"),
                                           at("workspace"), ws_bytes, None)


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("code,change", [
    (-1, dict(null="q")), (-1, dict(null="k")), (-1, dict(null="v")), (-1, dict(null="o")), (-1, dict(null="lse")),
    (-2, dict(B=0)), (-2, dict(Nq=0)), (-2, dict(Nk=-1)), (-2, dict(Hk=3)), (-2, dict(q_sn=64)), (-2, dict(k_sn=(1 << 23) + 8)),
    (-2, dict(B=1 << 13, Hq=1 << 11, Hk=1)), (-3, dict(d=96)),
    (-4, dict(odd="q")), (-4, dict(odd="k")), (-4, dict(odd="v")), (-4, dict(odd="o")), (-4, dict(odd="o_res")), (-4, dict(odd="lengths")),
    (-4, dict(odd="starts")), (-4, dict(q_sn=516)),
    (-5, dict(scale=0.0)), (-5, dict(scale=float("nan"))), (-5, dict(left=(1 << 28) + 1)), (-5, dict(right=1 << 30)), (-5, dict(sinks=-1)),
])
def test_window_attention_refuses(code, change, backward):
    assert _window_call(backward=backward, **change) == code


def test_window_attention_refuses_its_own():
    for name in ("d_o", "dq", "dk", "dv"):
        assert _window_call(null=name, backward=True) == -1 and _window_call(odd=name, backward=True) == -4
    assert _window_call(d_sb=0, backward=True) == -2 and _window_call(d_sn=260, backward=True) == -4
    assert _window_call(null="workspace", backward=True) == -6 and _window_call(ws_bytes=79, backward=True) == -6
    assert _window_call(odd="workspace", backward=True) == -4
    # one query with a long window is cut into parts: those need a workspace in the forward pass too
    long = dict(Nq=1, Nk=50000, k_sb=50000 * 256, left=40000)
    assert _window_call(null="workspace", **long) == -6 and _window_call(ws_bytes=1000, **long) == -6
    lib, s, w = binding._load(), binding._CrossShape(**CROSS), binding._Window(5, 0, 3)
    for f in (lib.spa2_window_fwd_workspace_bytes, lib.spa2_window_bwd_workspace_bytes):
        assert f(None, ctypes.byref(w)) == 0 and f(ctypes.byref(s), None) == 0
        assert f(ctypes.byref(s), ctypes.byref(binding._Window(1 << 29, 0, 0))) == 0
    assert lib.spa2_window_bwd_workspace_bytes(ctypes.byref(s), ctypes.byref(w)) >= 2 * 4 * 10 * 4


def test_workspaces_of_long_windows_do_not_grow_with_the_queries():
    """Partial results are those of a launch's parts, 2048 a kernel at most, whatever the sizes."""
    lib = binding._load()
    for Nq in (1, 300, 5000, 100_000):
        for left, sinks in ((-1, 0), (100, 0), (5000, 300), (90_000, 100_000)):
            for d in (64, 128):
                s = binding._CrossShape(1, 4, 2, Nq, 100_000, d, *[Nq * 4 * d, d, 4 * d], *[100_000 * 2 * d, d, 2 * d] * 2)
                w = binding._Window(left, 0, sinks)
                slots = 2048 * ((256 * d // 2 + 512) * 4 + 4) + 1024
                assert lib.spa2_window_fwd_workspace_bytes(ctypes.byref(s), ctypes.byref(w)) <= slots
                assert lib.spa2_window_bwd_workspace_bytes(ctypes.byref(s), ctypes.byref(w)) <= 2 * 4 * (4 * Nq + 64) + 3 * slots


GATE = dict(samples=2, tokens=10, gate_sb=0, scale_sb=64, shift_sb=64, width=64, kind=1, post=1, x_dtype=1, branch_dtype=1, out_dtype=1,
            param_dtype=1)
PARAMS = ("gate", "branch_weight", "weight", "bias", "scale", "shift")


def _gate_call(null=(), odd=None, eps=1e-6, backward=False, ws_bytes=1 << 60, grads=PARAMS, **change):
    s = binding._GateShape(**{**GATE, **change})
    null = (null,) if isinstance(null, str) else null
    at = lambda n: None if n in null else (ODD if n == odd else FAKE)
    p = binding._GateParams(*(at(n) for n in PARAMS))
    params = None if "params" in null else ctypes.byref(p)
    if backward:
        d = binding._GateParams(*(at("d_" + n) if n in grads else None for n in PARAMS))
        return binding._load().spa2_gate_norm_bwd(at("branch"), params, ctypes.byref(s), eps, at("y"), at("dy"), at("dn"), at("stats"),
                                                  at("dx"), at("dbranch"), ctypes.byref(d), at("workspace"), ws_bytes, None)
    return binding._load().spa2_gate_norm(at("x"), at("branch"), params, ctypes.byref(s), eps, at("y"), at("n"), at("stats"), None)


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("code,change", [
    (-1, dict(null="params")), (-2, dict(samples=0)), (-2, dict(tokens=0)), (-2, dict(samples=(1 << 22) + 1)), (-2, dict(tokens=1 << 40)),
    (-2, dict(width=7)), (-2, dict(width=8193)), (-2, dict(scale_sb=63)), (-2, dict(gate_sb=-64)),
    (-3, dict(kind=3)), (-3, dict(kind=-1)), (-3, dict(x_dtype=2)), (-3, dict(param_dtype=2)), (-3, dict(x_dtype=0)),
    (-3, dict(x_dtype=0, branch_dtype=0)), (-4, dict(odd="branch")), (-4, dict(odd="gate")), (-4, dict(odd="shift")), (-4, dict(odd="stats")),
    (-5, dict(eps=0.0)), (-5, dict(eps=float("inf"))), (-5, dict(eps=float("nan"))),
])
def test_gate_norm_refuses(code, change, backward):
    assert _gate_call(backward=backward, **change) == code


def test_gate_norm_refuses_its_own():
    for name in ("x", "y", "n"):
        assert _gate_call(null=name) == -1 and _gate_call(odd=name) == -4
    for name in ("y", "dn", "stats"):
        assert _gate_call(null=name, backward=True) == -1
    assert _gate_call(null="dy", kind=0, backward=True) == -1 and _gate_call(null="stats", kind=0, backward=True) == -1
    for name in ("dy", "dn", "dx", "dbranch", "d_gate", "d_bias"):
        assert _gate_call(odd=name, backward=True) == -4
    assert _gate_call(null="workspace", backward=True) == -6 and _gate_call(ws_bytes=64, backward=True) == -6
    assert _gate_call(odd="workspace", backward=True) == -4
    lib = binding._load()
    assert lib.spa2_gate_norm_bwd_workspace_bytes(None) == 0
    assert lib.spa2_gate_norm_bwd_workspace_bytes(ctypes.byref(binding._GateShape(**{**GATE, "width": 9000}))) == 0
    # at least a sum of each kind for every workgroup, of each sample one
    for samples in (1, 7, 5000):
        s = binding._GateShape(**{**GATE, "samples": samples})
        assert lib.spa2_gate_norm_bwd_workspace_bytes(ctypes.byref(s)) >= samples * 3 * 64 * 4


def test_clip_refuses():
    lib = binding._load()
    G = binding._Gradient

    def call(*entries, count=None, max_norm=1.0, eps=1e-6, norm=FAKE, ws=FAKE, ws_bytes=1 << 30):
        t = (G * max(len(entries), 1))(*(G(*e) for e in entries))
        return lib.spa2_clip_gradients(t, len(entries) if count is None else count, max_norm, eps, norm, ws, ws_bytes, None)
    ok = (FAKE, FAKE, 10, 1, 1)
    assert lib.spa2_clip_gradients(None, 1, 1.0, 1e-6, FAKE, FAKE, 1 << 30, None) == -1 and call(ok, norm=None) == -1
    assert call((None, FAKE, 10, 1, 1)) == -1 and call(ok, count=0) == -2 and call((FAKE, FAKE, -1, 1, 1)) == -2
    assert call((FAKE, FAKE, 1 << 42, 1, 1), ok) == -2
    assert call((FAKE, FAKE + 64, 10, 2, 1)) == -3 and call((FAKE, FAKE + 64, 10, 1, 5)) == -3 and call((FAKE, FAKE, 10, 1, 0)) == -3
    assert call((FAKE + 2, FAKE + 64, 10, 1, 1)) == -4 and call((FAKE, FAKE + 66, 10, 1, 1)) == -4 and call((ODD, None, 10, 0, 0)) == -4
    assert call(ok, norm=FAKE + 2) == -4 and call(ok, ws=FAKE + 8) == -4
    for bad in (dict(max_norm=-1.0), dict(max_norm=float("nan")), dict(eps=-1.0), dict(eps=float("inf")), dict(eps=float("nan"))):
        assert call(ok, **bad) == -5
    assert call(ok, ws=None) == -6 and call(ok, ws_bytes=16) == -6 and lib.spa2_clip_workspace_bytes() >= 256


def test_operators_have_no_cpu_path():
    x = torch.zeros((1, 2, 16, 64))
    with pytest.raises(ValueError):
        spa2.window_attention(x.bfloat16(), x.bfloat16(), x.bfloat16(), 4)
    with pytest.raises(ValueError):
        spa2.gate_add_norm(x)
    with pytest.raises(ValueError):
        spa2.clip_gradients([x], 1.0)
    with pytest.raises(ValueError):
        spa2.gradient_norm(x)
    with pytest.raises(ValueError):
        spa2.clip_gradients([], 1.0)
    with pytest.raises(TypeError):
        spa2.gate_add_norm(x, 1.0)


# ------------------------------------------------------------------ the binding, tensors elsewhere
def _window():
    q, k = torch.zeros(2, 4, 10, 64, dtype=BF), torch.zeros(2, 2, 20, 64, dtype=BF)
    return dict(q=q, k=k, v=k.clone(), lengths=torch.zeros(2, dtype=torch.int32), starts=torch.zeros(2, dtype=torch.int32), left=3, right=0,
                sinks=1, scale=0.1, o=q.clone(), lse=torch.zeros(2, 4, 10), o_res=q.clone(),
                workspace=torch.zeros(16, dtype=torch.uint8)), binding.spa2_window_fwd


def _window_bwd():
    t, _ = _window()
    return {**t, "d_o": t["q"].clone(), "dq": t["q"].clone(), "dk": t["k"].clone(), "dv": t["k"].clone(),
            "workspace": torch.zeros(1 << 16, dtype=torch.uint8)}, binding.spa2_window_bwd


def _gate():
    x = torch.zeros(2, 10, 64)
    return dict(x=x, branch=x.clone(), params=[torch.zeros(64) for _ in range(4)] + [torch.zeros(2, 64)] * 2, kind="layer", eps=1e-6,
                y=x.clone(), n=x.clone(), stats=torch.zeros(3, 20)), binding.spa2_gate_norm


def _gate_bwd():
    t, _ = _gate()
    x = t["x"]
    return dict(branch=x.clone(), params=t["params"], kind="layer", eps=1e-6, y=x, dy=x.clone(), dn=x.clone(), stats=torch.zeros(3, 20),
                dx=x.clone(), dbranch=x.clone(), grads=[p.clone() for p in t["params"]],
                workspace=torch.zeros(1 << 16, dtype=torch.uint8)), binding.spa2_gate_norm_bwd


def _clip():
    return dict(gradients=[torch.zeros(5), torch.zeros(6)], outs=[torch.zeros(5), torch.zeros(6)], max_norm=1.0, eps=1e-6,
                norm=torch.zeros(()), workspace=torch.zeros(1 << 16, dtype=torch.uint8)), binding.spa2_clip_gradients


CALLS = [_window, _window_bwd, _gate, _gate_bwd, _clip]
NAMED = [(f, n, i) for f in CALLS for n, t in f()[0].items()
         for i in (range(len(t)) if isinstance(t, list) else [None] if isinstance(t, torch.Tensor) else [])]


@pytest.mark.parametrize("make,name,i", NAMED, ids=[f"{f.__name__[1:]}-{n}-{i}" for f, n, i in NAMED])
def test_a_tensor_elsewhere_is_refused(make, name, i):
    args, call = make()
    if i is None:
        args[name] = args[name].to("meta")
    else:
        args[name][i] = args[name][i].to("meta")
    with pytest.raises(ValueError, match="one GPU"):
        call(**args)


@pytest.mark.parametrize("make", CALLS, ids=lambda f: f.__name__[1:])
def test_host_tensors_are_refused(make):
    args, call = make()
    with pytest.raises(ValueError, match="GPU only"):
        call(**args)


# ------------------------------------------------------------------ the formulas
@pytest.mark.parametrize("kind", ["layer", "rms", None])
@pytest.mark.parametrize("post", [False, True])
def test_gate_gradient_formula_against_differences(kind, post):
    """Central differences: the step's square times third derivatives, and 1e-16 over the step of rounding."""
    rng = np.random.default_rng(3)
    B, N, C, eps, h = 2, 3, 12, 1e-2, 1e-5
    t = {"x": rng.standard_normal((B, N, C)), "branch": rng.standard_normal((B, N, C)), "gate": rng.standard_normal((B, 1, C)),
         "branch_weight": rng.standard_normal(C), "weight": rng.standard_normal(C), "bias": rng.standard_normal(C),
         "scale": rng.standard_normal((B, 1, C)), "shift": rng.standard_normal((B, 1, C))}
    dy, dn = rng.standard_normal((2, B, N, C))
    w = lambda t: t["branch_weight"] if post else None

    def f(t):
        y = ref.gate_sum(t["x"], t["branch"], t["gate"], w(t), eps)[0]
        s = (y * dy).sum()
        return s if kind is None else s + (ref.gate_norm(y, kind, t["weight"], t["bias"], t["scale"], t["shift"], eps)[0] * dn).sum()
    y = ref.gate_sum(t["x"], t["branch"], t["gate"], w(t), eps)[0]
    got = ref.gate_bwd(y, t["branch"], t["gate"], w(t), kind, t["weight"], t["bias"], t["scale"], t["shift"], eps, dy,
                       None if kind is None else dn)
    for name, (g, _) in got.items():
        v = rng.standard_normal(t[name].shape)
        diff = (f({**t, name: t[name] + h * v}) - f({**t, name: t[name] - h * v})) / (2 * h)
        terms = g * (v if v.ndim == 3 and v.shape[1] > 1 else v.reshape(-1, C))
        assert abs(diff - terms.sum()) <= 1e-7 * max(np.abs(terms).sum(), 1.0), name


def test_window_gradient_formula_against_differences():
    rng = np.random.default_rng(2)
    q, k, v = rng.standard_normal((1, 2, 9, 8)), rng.standard_normal((1, 1, 12, 8)), rng.standard_normal((1, 1, 12, 8))
    do, h = rng.standard_normal(q.shape), 1e-5
    for args in (([11], [2], 3, 1, 2, 0.4), (None, None, None, 0, 0, 0.4), ([12], [-4], 2, 0, 1, 0.4)):
        got, _ = ref.window(q, k, v, *args, do)
        f = lambda q, k, v: (ref.window(q, k, v, *args)[0]["o"][0] * do).sum()
        for _ in range(4):
            w = [rng.standard_normal(x.shape) for x in (q, k, v)]
            diff = (f(*(x + h * y for x, y in zip((q, k, v), w))) - f(*(x - h * y for x, y in zip((q, k, v), w)))) / (2 * h)
            terms = [got[n][0] * y for n, y in zip(("dq", "dk", "dv"), w)]
            assert abs(diff - sum(t.sum() for t in terms)) <= 1e-7 * sum(np.abs(t).sum() for t in terms)


def test_window_mask():
    m = ref.window_mask(3, 8, 7, 4, 1, 1, 2)          # queries at places 4, 5, 6; key 7 is behind the length
    assert [np.flatnonzero(r).tolist() for r in m] == [[0, 1, 3, 4, 5], [0, 1, 4, 5, 6], [0, 1, 5, 6]]
    assert ref.window_mask(2, 4, 4, -1, None, 0, 0).tolist() == [[False] * 4, [True, False, False, False]]


def test_argument_checks_under_host_sanitizers():
    """csrc/step_api.hip with AddressSanitizer and UndefinedBehaviorSanitizer on the host side, launchers that abort, driven by
    tests/abi_sanitize/step_driver.c."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    hipcc, clang = shutil.which("hipcc") or "/opt/rocm/bin/hipcc", "/opt/rocm/lib/llvm/bin/clang"
    if not (os.path.exists(hipcc) and os.path.exists(clang)):
        pytest.skip("no ROCm toolchain")
    csrc, here = os.path.join(root, "paper_2602_13515_amd", "csrc"), os.path.join(root, "tests", "abi_sanitize")
    inc = ["-I", os.path.join(root, "include"), "-I", csrc]
    san = ["-fsanitize=address", "-fsanitize=undefined", "-fno-sanitize-recover=undefined"]
    host = ["--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-Wno-unused-command-line-argument",
            *(x for s in san for x in ("-Xarch_host", s))]
    with tempfile.TemporaryDirectory() as td:
        o = lambda n: os.path.join(td, n)
        for cmd in ([clang, "-std=c99", "-g", "-c", *san, *inc, os.path.join(here, "step_driver.c"), "-o", o("driver.o")],
                    [hipcc, *host, *inc, "-c", os.path.join(csrc, "step_api.hip"), "-o", o("api.o")],
                    [hipcc, *host, *inc, "-x", "hip", "-c", os.path.join(here, "step_stubs.cpp"), "-o", o("stubs.o")],
                    [hipcc, "--offload-arch=gfx950", "-fsanitize=address", "-fsanitize=undefined", "-fno-gpu-sanitize",
                     o("api.o"), o("stubs.o"), o("driver.o"), "-o", o("check")]):
            r = subprocess.run(cmd, capture_output=True, text=True)
            assert r.returncode == 0, r.stderr[-3000:]
        r = subprocess.run([o("check")], capture_output=True, text=True, timeout=120)
        assert r.returncode == 0 and "all rejected before launch" in r.stdout, (r.stdout[-2000:], r.stderr[-3000:])
        assert "runtime error" not in r.stderr and "AddressSanitizer" not in r.stderr, r.stderr[-3000:]
