"""Host-side checks of the layer and update calls (no GPU): every call made here is refused before anything could reach a device,
and the shape logic runs under sanitizers."""

import ctypes as C
import os
import shutil
import subprocess

import pytest
import torch

from paper_2605_21177_amd import autograd as A
from paper_2605_21177_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 0x10000                       # an address that is never touched


def _norm(**k):
    d = dict(kind=B.LAYERNORM, dtype=B.BF16, T=4, n=16, X=P, ldx=16, w=P, b=P, eps=1e-5)
    return B.NormLayer(*{**d, **k}.values())


def _linear(**k):
    d = dict(dtype=B.BF16, activation=B.ACT_GELU, out=24, n_in=16, T=4, X=P, ldx=16, W=P, ldw=16, bias=P, residual=P, ldr=24)
    return B.LinearLayer(*{**d, **k}.values())


def test_norm_calls_refuse_bad_arguments():
    lib = B.lib()
    fwd = lambda n, y=P, ldy=16, st=P: lib.chunkft_norm_forward(C.byref(n), y, ldy, st, None)  # noqa: E731
    bad = [(dict(kind=B.LINEAR), B.ERR_DTYPE), (dict(dtype=2), B.ERR_DTYPE), (dict(T=0), B.ERR_INVALID_ARG), (dict(T=(1 << 30) + 1), B.ERR_INVALID_ARG),
           (dict(n=0), B.ERR_INVALID_ARG), (dict(X=None), B.ERR_INVALID_ARG), (dict(X=P + 1), B.ERR_INVALID_ARG), (dict(ldx=15), B.ERR_INVALID_ARG),
           (dict(w=P + 1), B.ERR_INVALID_ARG), (dict(b=P + 1), B.ERR_INVALID_ARG), (dict(eps=-1e-9), B.ERR_INVALID_ARG), (dict(eps=float("nan")), B.ERR_INVALID_ARG),
           (dict(eps=1e300), B.ERR_INVALID_ARG), (dict(ldx=1 << 62), B.ERR_OVERFLOW), (dict(n=1 << 41, ldx=1 << 41), B.ERR_OVERFLOW)]
    for change, status in bad:
        assert fwd(_norm(**change)) == status, change
        assert lib.chunkft_norm_workspace_bytes(C.byref(_norm(**change))) == 0, change
    assert lib.chunkft_norm_forward(None, P, 16, P, None) == B.ERR_INVALID_ARG
    assert fwd(_norm(), y=None) == fwd(_norm(), y=P + 1) == fwd(_norm(), ldy=15) == fwd(_norm(), st=P + 2) == B.ERR_INVALID_ARG
    need = lib.chunkft_norm_workspace_bytes(C.byref(_norm()))
    assert need > 0

    def back(n=None, stats=P, dy=P, ldy=16, dx=P, ldx=16, dw=P, w=(0, 16), db=P, b=(0, 16), acc=0, ws=P, size=need):
        return lib.chunkft_norm_backward(C.byref(n or _norm()), stats, dy, ldy, dx, ldx, dw, *w, db, *b, acc, ws, size, None)

    for k in (dict(stats=None), dict(stats=P + 2), dict(dy=None), dict(dy=P + 1), dict(ldy=15), dict(dx=P + 1), dict(ldx=15), dict(dx=None, dw=None, db=None),
              dict(acc=2), dict(dw=P + 2), dict(db=P + 1)):
        assert back(**k) == B.ERR_INVALID_ARG, k
    for k in (dict(w=(3, 3)), dict(w=(-1, 2)), dict(w=(0, 17)), dict(b=(9, 8)), dict(b=(0, 17))):
        assert back(**k) == B.ERR_RANGE, k
    for k in (dict(ws=None), dict(ws=P + 8), dict(size=need - 1), dict(dw=None, ws=None), dict(db=None, size=0)):
        assert back(**k) == B.ERR_WORKSPACE, k


def test_linear_calls_refuse_bad_arguments():
    lib = B.lib()

    def fwd(l=None, y=P, ldy=24, z=P, ldz=24, ws=None, size=0):
        return lib.chunkft_linear_forward(C.byref(l or _linear()), y, ldy, z, ldz, ws, size, None)

    bad = [(dict(dtype=5), B.ERR_DTYPE), (dict(activation=4), B.ERR_DTYPE), (dict(activation=-1), B.ERR_DTYPE), (dict(out=0), B.ERR_INVALID_ARG), (dict(n_in=0), B.ERR_INVALID_ARG),
           (dict(T=0), B.ERR_INVALID_ARG), (dict(T=(1 << 30) + 1), B.ERR_INVALID_ARG), (dict(W=None), B.ERR_INVALID_ARG), (dict(ldw=15), B.ERR_INVALID_ARG), (dict(W=P + 1), B.ERR_INVALID_ARG),
           (dict(ldw=1 << 62), B.ERR_OVERFLOW), (dict(out=1 << 40, n_in=1 << 40, ldw=1 << 40), B.ERR_OVERFLOW)]
    for change, status in bad:
        assert fwd(_linear(**change)) == status, change
        assert lib.chunkft_linear_workspace_bytes(C.byref(_linear(**change)), 1) == 0
    for k in (dict(X=None), dict(X=P + 1), dict(ldx=15), dict(bias=P + 1), dict(residual=P + 1), dict(ldr=23)):
        assert fwd(_linear(**k)) == B.ERR_INVALID_ARG, k
    for k in (dict(y=None), dict(y=P + 1), dict(ldy=23), dict(z=P + 1), dict(ldz=23)):
        assert fwd(**k) == B.ERR_INVALID_ARG, k
    assert fwd(_linear(residual=P, ldr=24), y=P, ldy=32) == B.ERR_INVALID_ARG          # onto the residual, with another stride
    split = _linear(T=64, n_in=4096, ldx=4096, ldw=4096, out=512, ldr=512)
    need = lib.chunkft_linear_workspace_bytes(C.byref(split), 0)
    assert need > 0
    for ws, size in ((None, 0), (P, need - 1), (P + 8, need)):
        assert fwd(split, ldy=512, ldz=512, ws=ws, size=size) == B.ERR_WORKSPACE

    need = lib.chunkft_linear_workspace_bytes(C.byref(_linear()), 1)

    def back(l=None, dy=P, ldy=24, z=P, ldz=24, dz=P, lddz=24, dx=P, ldx=16, db=P, b=(0, 24), acc=0, ws=P, size=need):
        return lib.chunkft_linear_backward(C.byref(l or _linear()), dy, ldy, z, ldz, dz, lddz, dx, ldx, db, *b, acc, ws, size, None)

    for k in (dict(dy=None), dict(ldy=23), dict(z=None), dict(dz=None), dict(ldz=23), dict(lddz=23), dict(z=P + 1), dict(dx=P + 1), dict(ldx=15), dict(acc=-1),
              dict(l=_linear(activation=B.ACT_NONE)), dict(l=_linear(activation=B.ACT_NONE), z=None), dict(l=_linear(activation=B.ACT_NONE), z=None, dz=None, dx=None, db=None)):
        assert back(**k) == B.ERR_INVALID_ARG, k
    for b in ((0, 25), (5, 5), (-1, 3)):
        assert back(b=b) == B.ERR_RANGE
    for k in (dict(ws=None), dict(size=need - 1), dict(ws=P + 4)):
        assert back(**k) == B.ERR_WORKSPACE, k


def test_orthogonalised_updates_refuse_bad_arguments():
    lib = B.lib()
    size = lib.chunkft_orthogonalize_workspace_bytes
    assert size(B.F32, 64, 128) > size(B.BF16, 64, 128) > 0
    for bad in ((2, 8, 8), (B.F32, 0, 8), (B.F32, 8, (1 << 20) + 1), (B.BF16, (1 << 16) + 1, 1 << 17)):
        assert size(*bad) == 0
    need = size(B.BF16, 64, 128)

    def orth(g=P, ldg=128, dt=B.BF16, rows=64, cols=128, steps=5, eps=1e-7, o=P, ldo=128, ws=P, n=need):
        return lib.chunkft_orthogonalize(g, ldg, dt, rows, cols, steps, eps, o, ldo, ws, n, None)

    assert orth(dt=3) == B.ERR_DTYPE
    for k in (dict(g=None), dict(g=P + 1), dict(ldg=127), dict(o=None), dict(ldo=127), dict(steps=0), dict(steps=33), dict(eps=-1.0), dict(eps=float("inf")), dict(rows=0),
              dict(cols=(1 << 20) + 1, ldg=1 << 21, ldo=1 << 21), dict(ldo=136)):
        assert orth(**k) == B.ERR_INVALID_ARG, k
    assert orth(ldg=1 << 61, o=P + 2) == B.ERR_OVERFLOW
    for k in (dict(ws=None), dict(ws=P + 16), dict(n=need - 1)):
        assert orth(**k) == B.ERR_WORKSPACE, k

    need = size(B.F32, 64, 128)

    def muon(g=P, th=P, m=P, W=P, wd=B.BF16, rows=64, cols=128, ws=P, n=need, **hp):
        h = B.muon_hparams(**{**dict(lr=0.02), **hp})
        return lib.chunkft_muon_chunk(g, th, m, W, wd, rows, cols, C.byref(h), ws, n, None)

    assert muon(wd=4) == B.ERR_DTYPE and muon(precision=2) == B.ERR_DTYPE
    for k in (dict(g=None), dict(th=None), dict(m=None), dict(g=P + 2), dict(th=P + 1), dict(m=P + 2), dict(W=P + 1), dict(rows=0), dict(lr=-1.0), dict(lr=float("nan")),
              dict(momentum=1.0), dict(momentum=-0.1), dict(weight_decay=float("inf")), dict(eps=-1e-8), dict(scale=-1.0), dict(scale=1e300), dict(steps=0), dict(steps=33), dict(nesterov=2)):
        assert muon(**k) == B.ERR_INVALID_ARG, k
    h = B.muon_hparams(0.02)
    h.reserved = 1
    assert lib.chunkft_muon_chunk(P, P, P, P, B.BF16, 64, 128, C.byref(h), P, need, None) == B.ERR_INVALID_ARG
    assert lib.chunkft_muon_chunk(P, P, P, P, B.BF16, 64, 128, None, P, need, None) == B.ERR_INVALID_ARG
    for k in (dict(ws=None), dict(ws=P + 128), dict(n=need - 1)):
        assert muon(**k) == B.ERR_WORKSPACE, k


class _OnDevice:
    """A CPU tensor that says it is on the current device: what the binding checks before it makes a call."""

    def __init__(self, t, device=0):
        self.t, self.device = t, device
        self.dtype, self.shape, self.is_cuda = t.dtype, t.shape, True

    def __getattr__(self, name):
        return getattr(self.t, name)

    def get_device(self):
        return self.device


def test_binding_refuses_tensors_that_a_kernel_would_misread(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    bf = lambda *s: _OnDevice(torch.zeros(*s, dtype=torch.bfloat16))  # noqa: E731
    f32 = lambda *s: _OnDevice(torch.zeros(*s))  # noqa: E731
    x = bf(4, 16)
    for args in ((B.RMSNORM, _OnDevice(torch.zeros(4, 4, 16, dtype=torch.bfloat16))), (B.RMSNORM, _OnDevice(torch.zeros(16, 4, dtype=torch.bfloat16).t())),
                 (B.RMSNORM, x, bf(15)), (B.RMSNORM, x, _OnDevice(torch.zeros(32, dtype=torch.bfloat16)[::2])), (B.RMSNORM, torch.zeros(4, 16)),
                 (B.RMSNORM, _OnDevice(torch.zeros(4, 16), device=1))):
        with pytest.raises(ValueError):
            B.make_norm(*args)
    for args in ((B.RMSNORM, x, f32(16)), (B.RMSNORM, _OnDevice(torch.zeros(4, 16, dtype=torch.float16)))):
        with pytest.raises(TypeError):
            B.make_norm(*args)
    layer = B.make_norm(B.LAYERNORM, x, bf(16), bf(16))
    with pytest.raises(TypeError):
        B.chunkft_norm_forward(layer, f32(4, 16))
    for bad in (bf(5, 16), bf(4, 15)):
        with pytest.raises(ValueError):
            B.chunkft_norm_forward(layer, bad)
    with pytest.raises(ValueError):
        B.chunkft_norm_forward(layer, bf(4, 16), f32(4, 3))
    with pytest.raises(ValueError):
        B.chunkft_norm_backward(layer, f32(4, 2), bf(4, 16), bf(4, 16), dw=f32(16), w_range=(0, 8))
    with pytest.raises(TypeError):
        B.chunkft_norm_backward(layer, f32(4, 2), bf(4, 16), bf(4, 16), dw=bf(16))

    W = bf(24, 16)
    for k in (dict(X=bf(4, 15)), dict(X=x, bias=bf(23)), dict(X=x, residual=bf(4, 16)), dict(X=None), dict(X=x, residual=bf(5, 24))):
        with pytest.raises(ValueError):
            B.make_linear(k.pop("X"), W, **k)
    with pytest.raises(TypeError):
        B.make_linear(f32(4, 16), W)
    lin = B.make_linear(x, W, activation=B.ACT_SILU)
    for bad in (bf(4, 16), bf(3, 24)):
        with pytest.raises(ValueError):
            B.chunkft_linear_forward(lin, bad)
    with pytest.raises(ValueError):
        B.chunkft_linear_backward(lin, bf(4, 24), bf(4, 24), bf(4, 24), db=f32(24), b_range=(0, 8))
    with pytest.raises(ValueError):
        B.chunkft_orthogonalize(bf(4, 16), bf(4, 15))
    with pytest.raises(TypeError):
        B.chunkft_orthogonalize(bf(4, 16), f32(4, 16))
    hp = B.muon_hparams(0.1)
    for g, th, m, w in ((f32(63), f32(64), f32(64), bf(64)), (f32(64), f32(65), f32(64), bf(64)), (f32(64), f32(64), _OnDevice(torch.zeros(128)[::2]), bf(64)),
                        (f32(64), f32(64), f32(64), bf(63))):
        with pytest.raises(ValueError):
            B.chunkft_muon_chunk(g, th, m, w, 4, 16, hp)
    for g, w, wd in ((bf(64), bf(64), B.BF16), (f32(64), f32(64), B.BF16), (f32(64), bf(64), B.F32)):
        with pytest.raises(TypeError):
            B.chunkft_muon_chunk(g, f32(64), f32(64), w, 4, 16, hp, w_dtype=wd)


def test_autograd_layers_check_their_arguments():
    W, x, b = torch.zeros(8, 4), torch.zeros(3, 4), torch.zeros(8)
    seg = A.ChunkSegment(0, 8, torch.zeros(8))
    for k in (dict(bias_seg=seg), dict(bias=torch.zeros(7)), dict(bias=torch.zeros(8, requires_grad=True)), dict(bias=torch.zeros(8, dtype=torch.bfloat16)),
              dict(bias=b, bias_seg=A.ChunkSegment(0, 9, torch.zeros(9))), dict(residual=torch.zeros(3, 4)), dict(residual=torch.zeros(3, 8, dtype=torch.bfloat16)),
              dict(bias=torch.zeros(16)[::2])):
        with pytest.raises(ValueError):
            A.chunk_linear(x, W, None, **k)
    with pytest.raises(ValueError):
        A.chunk_linear(torch.zeros(3, 5), W, None, activation=B.ACT_RELU)
    for args, k in (((x, torch.zeros(5)), {}), ((x, torch.zeros(4, requires_grad=True)), {}), ((x, None), dict(seg=seg)), ((x, None, None), dict(bias_seg=seg)),
                    ((x, torch.zeros(4)), dict(seg=seg)), ((x, torch.zeros(4, dtype=torch.bfloat16)), {})):
        with pytest.raises(ValueError):
            A.chunk_norm(*args, **k)
    hp, t = B.muon_hparams(0.1), torch.zeros(8)
    with pytest.raises(ValueError):
        A.ChunkSegment(0, 8, master=t, m=t, v=t, hp=hp)
    with pytest.raises(ValueError):
        A.ChunkSegment(0, 8, master=t, hp=hp)
    with pytest.raises(ValueError):
        A.chunk_norm(x, torch.zeros(4), seg=A.ChunkSegment(0, 4, master=t, m=t, hp=hp))


def test_workspaces_are_a_pure_function_of_the_shape():
    a, b = _linear(T=64, n_in=4096, ldx=4096, ldw=4096, out=512, ldr=512), _linear(T=64, n_in=4096, ldx=8192, ldw=4104, out=512, ldr=520, X=P + 2)
    size = B.lib().chunkft_linear_workspace_bytes
    for backward in (0, 1):
        assert size(C.byref(a), backward) == size(C.byref(b), backward) > 0
    one = _linear(T=1, n_in=4096, ldx=4096, ldw=4096, out=512, ldr=512)
    assert size(C.byref(one), 0) == 0                              # few tokens need none


def test_host_code_of_the_layers_under_sanitizers(tmp_path):
    gxx = shutil.which("g++")
    assert gxx, "g++ is part of the image"
    csrc, exe = os.path.join(ROOT, "paper_2605_21177_amd", "csrc"), str(tmp_path / "layers_sanitize")
    cmd = [gxx, "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-static-libasan", "-I", os.path.join(ROOT, "include"), "-I", csrc,
           os.path.join(ROOT, "tests", "layers_sanitize.cpp"), os.path.join(csrc, "layers_api.cpp"), os.path.join(csrc, "layers_shape.cpp"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.startswith("ok:"), (r.stdout[-1000:], r.stderr[-3000:])


def test_segments_that_no_call_can_serve():
    x, W, b, w = torch.zeros(3, 8), torch.zeros(8, 8), torch.zeros(8), torch.zeros(8)
    seg, t = A.ChunkSegment(0, 8, torch.zeros(8)), torch.zeros(8)
    with pytest.raises(ValueError, match="of its own"):
        A.chunk_linear(x, W, seg, bias=b, bias_seg=seg)
    with pytest.raises(ValueError, match="of its own"):
        A.chunk_norm(x, w, b, B.LAYERNORM, seg=seg, bias_seg=seg)
    with pytest.raises(ValueError, match="lie in W"):
        A.chunk_linear(x, W, A.ChunkSegment(60, 65, torch.zeros(5)), activation=B.ACT_RELU)
    for activation in (B.ACT_NONE, B.ACT_RELU):
        with pytest.raises(ValueError, match="whole rows"):
            A.chunk_linear(x, W, A.ChunkSegment(4, 12, master=t, m=t, hp=B.muon_hparams(0.1)), activation=activation)
