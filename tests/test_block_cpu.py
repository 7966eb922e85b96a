"""The operators around the attention, without a GPU: refusals of the C entry points, the formulas that their GPU tests
compare with (against differences and published vectors), the rotary tables."""
import ctypes

import numpy as np
import pytest
import torch

import block_ref as ref
import paper_2602_13515_amd as spa2
from paper_2602_13515_amd import binding

FAKE, ODD = 0x1000, 0x1004             # an aligned and an unaligned address; neither is read
NORM = dict(B=2, Hq=4, Hk=2, N=10, d=128, dtype=0, rot=128, interleaved=0, table_rows=10, pos_bits=0, pos_sb=0,
            q_sb=5120, q_sh=128, q_sn=512, k_sb=2560, k_sh=128, k_sn=256,
            qo_sb=5120, qo_sh=128, qo_sn=512, ko_sb=2560, ko_sh=128, ko_sn=256)


def _norm_call(null=None, address=FAKE, eps=1e-6, backward=False, ws_bytes=1 << 30, **change):
    s = binding._NormShape(**{**NORM, **change})
    names = ["q", "k", "q_weight", "k_weight", "cos", "sin", "positions"] + (["d_q_out", "d_k_out"] if backward else [])
    args = [None if n == null else (address if n == "q" else FAKE) for n in names]
    outs = ["dq", "dk", "d_q_weight", "d_k_weight", "workspace"] if backward else ["q_out", "k_out"]
    tail = [None if n == null else FAKE for n in outs] + ([ws_bytes] if backward else [])
    f = binding._load().spa2_norm_rotate_bwd if backward else binding._load().spa2_norm_rotate
    return f(*args, ctypes.byref(s), eps, *tail, None)


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("code,change", [
    (-1, dict(null="q")), (-1, dict(null="k")), (-1, dict(null="cos")), (-1, dict(null="sin")),
    (-1, dict(null="positions", pos_bits=32)),
    (-2, dict(B=0)), (-2, dict(N=0)), (-2, dict(Hk=0)), (-2, dict(Hq=-1)), (-2, dict(table_rows=9)), (-2, dict(table_rows=0, pos_bits=64)),
    (-2, dict(q_sn=-512)), (-2, dict(qo_sh=-128)), (-2, dict(B=1 << 16, N=1 << 15, table_rows=1 << 15)),
    (-3, dict(d=96)), (-3, dict(d=256)), (-3, dict(dtype=2)), (-3, dict(rot=24)), (-3, dict(rot=144)), (-3, dict(rot=-16)),
    (-3, dict(pos_bits=16)),
    (-4, dict(address=ODD)), (-4, dict(q_sn=516)), (-4, dict(dtype=1, q_sn=514)), (-4, dict(dtype=1, ko_sn=260)),
    (-5, dict(eps=0.0)), (-5, dict(eps=-1.0)), (-5, dict(eps=float("inf"))), (-5, dict(eps=float("nan"))),
])
def test_norm_rotate_refuses(code, change, backward):
    assert _norm_call(backward=backward, **change) == code


def test_norm_rotate_refuses_its_own():
    assert _norm_call(null="q_out") == -1 and _norm_call(null="k_out") == -1
    for name in ("d_q_out", "d_k_out", "dq", "dk"):
        assert _norm_call(null=name, backward=True) == -1
    s = binding._NormShape(**NORM)
    need = binding._load().spa2_norm_rotate_bwd_workspace_bytes(ctypes.byref(s))
    assert need >= 2 * 128 * 4
    assert _norm_call(null="workspace", backward=True) == -6 and _norm_call(ws_bytes=16, backward=True) == -6
    assert binding._load().spa2_norm_rotate_bwd_workspace_bytes(None) == 0
    assert binding._load().spa2_norm_rotate_bwd_workspace_bytes(ctypes.byref(binding._NormShape(**{**NORM, "d": 80}))) == 0
    f = binding._load().spa2_norm_rotate
    assert f(FAKE, FAKE, None, None, FAKE, FAKE, None, None, 1e-6, FAKE, FAKE, None) == -1        # no shape
    assert f(FAKE, FAKE, None, None, FAKE, FAKE, None, ctypes.byref(s), 1e-6, FAKE, ODD, None) == -4


def test_dropout_refuses():
    f, b = binding._load().spa2_dropout_add, binding._load().spa2_dropout_bwd
    ok = [FAKE, FAKE, 8, 0, 1, 0.5, 1, 2, None, FAKE, None]

    def with_(at, value):
        return f(*[value if i == at else x for i, x in enumerate(ok)])
    assert with_(0, None) == -1 and with_(9, None) == -1
    assert with_(2, 0) == -2 and with_(2, -8) == -2
    assert with_(3, 2) == -3 and with_(4, 3) == -3
    assert f(FAKE, FAKE, 8, 1, 0, 0.5, 1, 2, None, FAKE, None) == -3          # fp32 into a bf16 residual
    assert with_(0, ODD) == -4 and with_(1, ODD) == -4 and with_(9, ODD) == -4 and with_(8, ODD) == -4
    for p in (-0.1, 1.1, float("nan"), float("inf")):
        assert with_(5, p) == -5
        assert b(FAKE, 8, 0, 0, p, 1, 2, None, FAKE, None) == -5
    assert b(None, 8, 0, 0, 0.5, 1, 2, None, FAKE, None) == -1 and b(FAKE, 8, 0, 0, 0.5, 1, 2, None, None, None) == -1
    assert b(FAKE, 0, 0, 0, 0.5, 1, 2, None, FAKE, None) == -2
    assert b(FAKE, 8, 0, 1, 0.5, 1, 2, None, FAKE, None) == -3                # bf16 gradient of an fp32 result
    assert b(ODD, 8, 0, 0, 0.5, 1, 2, None, FAKE, None) == -4


CROSS = dict(B=2, Hq=4, Hk=2, Nq=10, Nk=20, d=128, q_sb=5120, q_sh=128, q_sn=512, k_sb=5120, k_sh=128, k_sn=256,
             d_sb=5120, d_sh=128, d_sn=256)


def _cross_call(null=None, odd=None, scale=0.1, backward=False, ws_bytes=1 << 60, **change):
    s = binding._CrossShape(**{**CROSS, **change})
    at = lambda n: None if n == null else (ODD if n == odd else FAKE)
    if backward:
        args = [at(n) for n in ("q", "k", "v", "lengths", "o", "o_res", "d_o", "lse")]
        return binding._load().spa2_cross_bwd(*args, ctypes.byref(s), scale, at("dq"), at("dk"), at("dv"), at("workspace"), ws_bytes, None)
    args = [at(n) for n in ("q", "k", "v", "lengths")]
    return binding._load().spa2_cross_fwd(*args, ctypes.byref(s), scale, at("o"), at("o_res"), at("lse"), at("workspace"), ws_bytes, None)


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("code,change", [
    (-1, dict(null="q")), (-1, dict(null="k")), (-1, dict(null="v")), (-1, dict(null="o")), (-1, dict(null="lse")),
    (-2, dict(B=0)), (-2, dict(Nq=0)), (-2, dict(Nk=-1)), (-2, dict(Hk=3)), (-2, dict(Hk=0)), (-2, dict(Hq=0)),
    (-2, dict(q_sn=64)), (-2, dict(q_sh=0)), (-2, dict(k_sn=(1 << 23) + 8)), (-2, dict(k_sb=-8)),
    (-2, dict(B=1 << 13, Hq=1 << 11, Hk=1)), (-2, dict(Nq=1 << 30)), (-2, dict(Nk=1 << 29)),
    (-3, dict(d=96)), (-3, dict(d=32)),
    (-4, dict(odd="q")), (-4, dict(odd="k")), (-4, dict(odd="v")), (-4, dict(odd="o")), (-4, dict(odd="o_res")),
    (-4, dict(q_sn=516)), (-4, dict(k_sh=132)),
    (-5, dict(scale=0.0)), (-5, dict(scale=-1.0)), (-5, dict(scale=float("nan"))), (-5, dict(scale=float("inf"))),
])
def test_cross_attention_refuses(code, change, backward):
    assert _cross_call(backward=backward, **change) == code


def test_cross_attention_refuses_its_own():
    for name in ("d_o", "dq", "dk", "dv"):
        assert _cross_call(null=name, backward=True) == -1 and _cross_call(odd=name, backward=True) == -4
    assert _cross_call(d_sb=0, backward=True) == -2 and _cross_call(d_sn=260, backward=True) == -4
    assert _cross_call(null="workspace", backward=True) == -6 and _cross_call(ws_bytes=79, backward=True) == -6
    assert _cross_call(odd="workspace", backward=True) == -4
    # one query against a long cache is cut into parts: those need a workspace in the forward pass too
    long = dict(Nk=50000, k_sb=50000 * 256)
    assert _cross_call(null="workspace", **long) == -6 and _cross_call(ws_bytes=1000, **long) == -6
    assert _cross_call(odd="workspace", **long) == -4
    lib = binding._load()
    for f in (lib.spa2_cross_fwd_workspace_bytes, lib.spa2_cross_bwd_workspace_bytes):
        assert f(None) == 0 and f(ctypes.byref(binding._CrossShape(**{**CROSS, "d": 80}))) == 0
    assert lib.spa2_cross_bwd_workspace_bytes(ctypes.byref(binding._CrossShape(**CROSS))) >= 2 * 4 * 10 * 4
    assert lib.spa2_cross_fwd(FAKE, FAKE, FAKE, None, None, 0.1, FAKE, None, FAKE, None, 0, None) == -1


def test_operators_have_no_cpu_path():
    x = torch.zeros((1, 2, 16, 64))
    with pytest.raises(ValueError):
        spa2.cross_attention(x.bfloat16(), x.bfloat16(), x.bfloat16())
    with pytest.raises(ValueError):
        spa2.qk_norm_rotate(x, x)
    with pytest.raises(ValueError):
        spa2.dropout_add(x, None, 0.5, 1)
    with pytest.raises(TypeError):
        spa2.dropout_add(x, 0.0, 0.5, 1)


# ------------------------------------------------------------------ the formulas themselves
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rot", [0, 16, 64])
def test_gradient_formula_against_differences(rot, interleaved):
    rng = np.random.default_rng(rot + interleaved)
    x, dy, w = rng.standard_normal((5, 64)), rng.standard_normal((5, 64)), 1 + 0.3 * rng.standard_normal(64)
    angle = rng.uniform(-9, 9, (5, rot // 2))
    cos, sin = (np.cos(angle), np.sin(angle)) if rot else (None, None)
    dx, dw, _, _ = ref.norm_rotate_bwd(x, w, cos, sin, 1e-2, interleaved, dy)
    f = lambda x, w: (ref.norm_rotate(x, w, cos, sin, 1e-2, interleaved)[0] * dy).sum()
    h = 1e-5                 # central differences: h^2 of the third derivative, and 1e-16 / h of rounding
    for _ in range(8):
        vx, vw = rng.standard_normal(x.shape), rng.standard_normal(w.shape)
        diff = (f(x + h * vx, w + h * vw) - f(x - h * vx, w - h * vw)) / (2 * h)
        assert abs(diff - ((dx * vx).sum() + (dw * vw).sum())) <= 1e-7 * (np.abs(dx * vx).sum() + np.abs(dw * vw).sum())


@pytest.mark.parametrize("counter,key,words", [
    ((0, 0, 0, 0), (0, 0), (0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8)),
    ((0xffffffff,) * 4, (0xffffffff,) * 2, (0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd)),
    ((0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344), (0xa4093822, 0x299f31d0),
     (0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1)),
])
def test_generator_against_published_vectors(counter, key, words):
    assert tuple(int(x) for x in ref.philox(counter, key)) == words


def test_rotary_table():
    cos, sin = spa2.rotary_table(7, 64)
    angle = np.arange(7)[:, None] * 10000.0 ** (-np.arange(32) / 32)
    assert cos.dtype == torch.float32 and cos.shape == (7, 32)
    assert np.abs(cos.numpy() - np.cos(angle)).max() <= 2.0 ** -24 and np.abs(sin.numpy() - np.sin(angle)).max() <= 2.0 ** -24
    cos, _ = spa2.rotary_table((2, 3, 4), 128, theta=100.0)
    assert cos.shape == (24, 64)
    n = (1 * 3 + 2) * 4 + 3                  # frame 1, row 2, column 3; 22, 21 and 21 pairs
    want = np.concatenate([c * 100.0 ** (-np.arange(m) / m) for c, m in ((1, 22), (2, 21), (3, 21))])
    assert np.abs(cos[n].numpy() - np.cos(want)).max() <= 2.0 ** -24
    for sizes, d in (((), 64), ((0,), 64), ((2, 2, 2), 4), (4, 63)):
        with pytest.raises(ValueError):
            spa2.rotary_table(sizes, d)


def test_attention_gradient_formula_against_differences():
    rng = np.random.default_rng(1)
    q, k, v = rng.standard_normal((2, 4, 5, 8)), rng.standard_normal((2, 2, 7, 8)), rng.standard_normal((2, 2, 7, 8))
    do, lengths, h = rng.standard_normal(q.shape), np.array([7, 3]), 1e-5
    g, _ = ref.cross(q, k, v, lengths, 0.4, do)
    f = lambda q, k, v: (ref.cross(q, k, v, lengths, 0.4)[0]["o"][0] * do).sum()
    for _ in range(8):
        w = [rng.standard_normal(x.shape) for x in (q, k, v)]
        diff = (f(*(x + h * y for x, y in zip((q, k, v), w))) - f(*(x - h * y for x, y in zip((q, k, v), w)))) / (2 * h)
        terms = [(g[n][0] * y) for n, y in zip(("dq", "dk", "dv"), w)]
        assert abs(diff - sum(t.sum() for t in terms)) <= 1e-7 * sum(np.abs(t).sum() for t in terms)


def test_argument_checks_under_host_sanitizers():
    """csrc/block_api.hip with AddressSanitizer and UndefinedBehaviorSanitizer on the host side, launchers that abort, driven by
    tests/abi_sanitize/block_driver.c."""
    import os
    import shutil
    import subprocess
    import tempfile
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
        for cmd in ([clang, "-std=c99", "-g", "-c", *san, *inc, os.path.join(here, "block_driver.c"), "-o", o("driver.o")],
                    [hipcc, *host, *inc, "-c", os.path.join(csrc, "block_api.hip"), "-o", o("api.o")],
                    [hipcc, *host, *inc, "-x", "hip", "-c", os.path.join(here, "block_stubs.cpp"), "-o", o("stubs.o")],
                    [hipcc, "--offload-arch=gfx950", "-fsanitize=address", "-fsanitize=undefined", "-fno-gpu-sanitize",
                     o("api.o"), o("stubs.o"), o("driver.o"), "-o", o("check")]):
            r = subprocess.run(cmd, capture_output=True, text=True)
            assert r.returncode == 0, r.stderr[-3000:]
        r = subprocess.run([o("check")], capture_output=True, text=True, timeout=120)
        assert r.returncode == 0 and "all rejected before launch" in r.stdout, (r.stdout[-2000:], r.stderr[-3000:])
        assert "runtime error" not in r.stderr and "AddressSanitizer" not in r.stderr, r.stderr[-3000:]


@pytest.mark.parametrize("units,list_max", [(1, 1), (1, 4096), (2, 1024), (64, 512), (300, 7), (512, 40), (513, 100), (2049, 100)])
def test_workspaces_hold_what_the_kernels_use(units, list_max):
    """Sizes grow with the parts and never exceed what 2048 parts need; small ones are no larger than D and counters."""
    lib, d = binding._load(), 128
    s = binding._CrossShape(units, 1, 1, 128, 64 * list_max, d, 128 * d, 128 * d, d, 64 * list_max * d, 64 * list_max * d, d,
                            64 * list_max * d, 64 * list_max * d, d)
    slot = (256 * d // 2 + 512) * 4
    fwd, bwd = lib.spa2_cross_fwd_workspace_bytes(ctypes.byref(s)), lib.spa2_cross_bwd_workspace_bytes(ctypes.byref(s))
    assert fwd <= 2048 * (slot + 4) + 512 and bwd >= units * 128 * 4
    assert bwd <= units * 128 * 4 + 2 * (2048 * (slot + 4) + 512) + 512
    if units > 2048:
        assert fwd == 0
