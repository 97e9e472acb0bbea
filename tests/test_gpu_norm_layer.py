"""RMSNorm and LayerNorm layers on the GPU against their definitions in 64 bits."""

import pytest
import torch

from paper_2605_21177_amd import binding as B

import gpu_harness as H
from layers_harness import DEV, Placed, assert_close

pytestmark = pytest.mark.gpu

KINDS = {"rmsnorm": B.RMSNORM, "layernorm": B.LAYERNORM}
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    H.require_gpu()


def _inputs(seed, T, n, dtype, kind):
    gen = torch.Generator().manual_seed(seed)
    x = (torch.randn(T, n, generator=gen) * (1 + torch.rand(n, generator=gen)) + 0.5 * torch.randn(n, generator=gen)).to(dtype)
    w, b = (1 + 0.2 * torch.randn(n, generator=gen)).to(dtype), (0.2 * torch.randn(n, generator=gen)).to(dtype)
    dy = (0.01 * torch.randn(T, n, generator=gen)).to(dtype)
    return x, w, b, dy


def _stats64(x, kind, eps=EPS):
    x = x.double()
    mean = x.mean(1, keepdim=True) if kind == "layernorm" else torch.zeros_like(x[:, :1])
    rstd = 1 / ((x - mean).square().mean(1, keepdim=True) + eps).sqrt()
    return mean, rstd


def _check_forward(x, w, b, kind, y, stats, eps=EPS):
    n = x.shape[1]
    mean, rstd = _stats64(x, kind, eps)
    xd, wd, bd = x.double(), w.double() if w is not None else 1.0, b.double() if b is not None else 0.0
    xh = (xd - mean) * rstd
    size = xh.abs() + rstd * xd.abs().mean(1, keepdim=True)
    assert_close(y, xh * wd + bd, size * abs(wd) + abs(bd), 2 * n + 16, "y")
    if stats is not None:
        assert_close(stats[:, :1], mean, xd.abs().mean(1, keepdim=True), n + 4, "mean")
        assert_close(stats[:, 1:], rstd, rstd + rstd ** 2 * xd.abs().mean(1, keepdim=True), 2 * n + 16, "rstd")


def _check_backward(x, w, dy, stats, kind, dx=None, dw=None, db=None, w_range=None, b_range=None):
    T, n = x.shape
    st = stats.double().cpu()
    mean, rstd = (st[:, :1] if kind == "layernorm" else 0.0), st[:, 1:]
    xd, d = x.double(), dy.double()
    xh = (xd - mean) * rstd
    size = (xd.abs() + abs(mean)) * rstd                              # what x - mean is rounded against
    h = d * (w.double() if w is not None else 1.0)
    if dx is not None:
        c2 = (h * xh).mean(1, keepdim=True)
        c1 = h.mean(1, keepdim=True) if kind == "layernorm" else 0.0
        sums = rstd * (h.abs() + h.abs().mean(1, keepdim=True) + size * (h.abs() * size).mean(1, keepdim=True))
        assert_close(dx, rstd * (h - c1 - xh * c2), sums, 2 * n + 16, "dx")
    if dw is not None:
        s = slice(*(w_range or (0, n)))
        assert_close(dw, (d * xh).sum(0)[s], (d.abs() * size).sum(0)[s], T + 16, "dw")
    if db is not None:
        s = slice(*(b_range or (0, n)))
        assert_close(db, d.sum(0)[s], d.abs().sum(0)[s], T + 16, "db")


# widths on both sides of every change of lanes and pieces per lane (64, 128, 256, 512, 1024, 2048, 4096 pieces of 8 or 4), odd ones
SHAPES = [(1, 1), (3, 7), (5, 8), (70, 64), (33, 513), (9, 1024), (7, 1025), (5, 2048), (6, 2051), (17, 4096), (4, 8192), (3, 8200),
          (2, 16384), (2, 16391), (2, 32769), (1, 40000), (1200, 24)]


@pytest.mark.parametrize("kind", sorted(KINDS))
@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("T,n", SHAPES)
def test_forward_and_backward(T, n, dtype, kind):
    dt = DTYPES[dtype]
    x, w, b, dy = _inputs(T * 131 + n, T, n, dt, kind)
    odd = n % 2                                                       # odd widths also lie at odd places
    X, Wt, Bt, DY = Placed(x, pad=3 * odd, lead=odd), Placed(w, lead=odd), Placed(b, lead=odd), Placed(dy, pad=odd, lead=1)
    Y, DX = Placed(torch.zeros(T, n, dtype=dt), pad=5 * odd, lead=odd), Placed(torch.zeros(T, n, dtype=dt), pad=odd)
    ST = Placed(torch.zeros(2 * T))
    stats = ST.t.view(T, 2)
    layer = B.make_norm(KINDS[kind], X.t, Wt.t, Bt.t, EPS)
    B.chunkft_norm_forward(layer, Y.t, stats)
    ws = torch.empty(B.chunkft_norm_workspace_bytes(layer), dtype=torch.uint8, device=DEV)
    DW, DB = Placed(torch.zeros(n), lead=1), Placed(torch.zeros(n), lead=2)
    B.chunkft_norm_backward(layer, stats, DY.t, DX.t, dw=DW.t, db=DB.t, ws=ws)
    torch.cuda.synchronize()
    _check_forward(x, w, b, kind, Y.t, stats.cpu())
    _check_backward(x, w, dy, stats, kind, DX.t, DW.t, DB.t)
    assert all(p.untouched() for p in (X, Wt, Bt, DY, Y, DX, ST, DW, DB))


@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_parts_of_the_vectors_accumulate_and_stay_inside(dtype):
    dt, T, n = DTYPES[dtype], 530, 777
    x, w, b, dy = _inputs(3, T, n, dt, "layernorm")
    X, DY = x.to(DEV), dy.to(DEV)
    layer = B.make_norm(B.LAYERNORM, X, w.to(DEV), None, EPS)
    stats, y = torch.empty(T, 2, device=DEV), torch.empty_like(X)
    B.chunkft_norm_forward(layer, y, stats)
    ws = torch.empty(B.chunkft_norm_workspace_bytes(layer), dtype=torch.uint8, device=DEV)
    DW, DB = Placed(torch.zeros(300)), Placed(torch.zeros(1))
    B.chunkft_norm_backward(layer, stats, DY, None, dw=DW.t, w_range=(101, 401), db=DB.t, b_range=(776, 777), ws=ws)
    torch.cuda.synchronize()
    _check_backward(x, w, dy, stats, "layernorm", None, DW.t, DB.t, (101, 401), (776, 777))
    once = DW.t.clone(), DB.t.clone()
    B.chunkft_norm_backward(layer, stats, DY, None, dw=DW.t, w_range=(101, 401), db=DB.t, b_range=(776, 777), accumulate=True, ws=ws)
    torch.cuda.synchronize()
    assert torch.equal(DW.t, once[0] + once[0]) and torch.equal(DB.t, once[1] + once[1])
    assert DW.untouched() and DB.untouched()
    # the input gradient alone needs no workspace, and is the same
    dx, dx2 = torch.empty_like(X), torch.empty_like(X)
    B.chunkft_norm_backward(layer, stats, DY, dx)
    B.chunkft_norm_backward(layer, stats, DY, dx2, db=DB.t, b_range=(0, 1), ws=ws)
    torch.cuda.synchronize()
    assert torch.equal(dx, dx2)
    _check_backward(x, w, dy, stats, "layernorm", dx)


@pytest.mark.parametrize("kind", sorted(KINDS))
def test_no_vectors_no_statistics(kind):
    T, n = 37, 300
    x, _, _, dy = _inputs(8, T, n, torch.bfloat16, kind)
    layer = B.make_norm(KINDS[kind], x.to(DEV), eps=EPS)
    y, stats, dx = torch.empty_like(x, device=DEV), torch.empty(T, 2, device=DEV), torch.empty_like(x, device=DEV)
    B.chunkft_norm_forward(layer, y)
    _check_forward(x, None, None, kind, y, None)
    B.chunkft_norm_forward(layer, y, stats)
    B.chunkft_norm_backward(layer, stats, dy.to(DEV), dx)
    _check_backward(x, None, dy, stats, kind, dx)


def test_large_mean_keeps_its_digits():
    """Values 1000 +- 1: the variance is summed about the mean, not from squares of the values."""
    gen = torch.Generator().manual_seed(4)
    x = 1000 + torch.randn(6, 4097, generator=gen)
    y, stats = torch.empty(6, 4097, device=DEV), torch.empty(6, 2, device=DEV)
    B.chunkft_norm_forward(B.make_norm(B.LAYERNORM, x.to(DEV), eps=EPS), y, stats)
    mean, rstd = _stats64(x, "layernorm")
    # the mean's own error, n 2^-24 1000, is the sums'; a lane adds at most 16 values and 10 levels join them: 26 in place of n
    assert float((stats[:, :1].cpu().double() - mean).abs().max()) <= 40 * 2 ** -24 * 1000
    assert float((stats[:, 1:].cpu().double() / rstd - 1).abs().max()) <= 1e-4
    assert float((y.cpu().double() - (x.double() - mean) * rstd).abs().max()) <= 40 * 2 ** -24 * 1000 + 1e-4 * 6


def test_constant_rows_and_rows_with_infinities_keep_to_themselves():
    n = 520
    x, w, b, dy = _inputs(6, 7, n, torch.bfloat16, "layernorm")
    x[2] = 0
    x[4, 17] = float("inf")
    x[5, 3] = float("nan")
    y, stats, dx = torch.empty_like(x, device=DEV), torch.empty(7, 2, device=DEV), torch.empty_like(x, device=DEV)
    layer = B.make_norm(B.LAYERNORM, x.to(DEV), w.to(DEV), b.to(DEV), EPS)
    B.chunkft_norm_forward(layer, y, stats)
    B.chunkft_norm_backward(layer, stats, dy.to(DEV), dx)
    y, dx = y.cpu(), dx.cpu()
    fine = [0, 1, 2, 3, 6]
    assert torch.isnan(y[[4, 5]]).all() and torch.isnan(dx[[4, 5]]).all()
    assert torch.isfinite(y[fine]).all() and torch.isfinite(dx[fine]).all()
    assert torch.equal(y[2], b)                                       # a row without deviation is the shift
    _check_forward(x[fine], w, b, "layernorm", y[fine], stats.cpu()[fine])
    _check_backward(x[fine], w, dy[fine], stats.cpu()[fine], "layernorm", dx[fine])


def test_captured_and_replayed_on_another_stream_with_eager_work_between():
    T, n = 513, 1536
    x, w, b, dy = [t.to(DEV) for t in _inputs(9, T, n, torch.bfloat16, "layernorm")]
    layer = B.make_norm(B.LAYERNORM, x, w, b, EPS)
    ws = torch.empty(B.chunkft_norm_workspace_bytes(layer), dtype=torch.uint8, device=DEV)

    def outputs():
        return torch.empty_like(x), torch.empty(T, 2, device=DEV), torch.empty_like(x), torch.empty(n, device=DEV), torch.empty(n, device=DEV)

    def step(o, stream=None):
        B.chunkft_norm_forward(layer, o[0], o[1], stream=stream)
        B.chunkft_norm_backward(layer, o[1], dy, o[2], dw=o[3], db=o[4], ws=ws, stream=stream)

    eager, captured = outputs(), outputs()
    step(eager)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(captured)
    for _ in range(3):
        for t in captured:
            t.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(eager, captured))
        x.add_(0.25)
        step(eager)
        torch.cuda.synchronize()
    other = outputs()
    side.wait_stream(torch.cuda.current_stream())
    step(other, stream=side)
    side.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(eager, other))
