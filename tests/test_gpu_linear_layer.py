"""The linear layer with bias, activation and residual on the GPU against its definition in 64 bits, forward and backward."""

import pytest
import torch

from paper_2605_21177_amd import binding as B

import gpu_harness as H
from layers_harness import ACTS, DEV, Placed, act64, assert_close, slope64

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
CODES = {"none": B.ACT_NONE, "relu": B.ACT_RELU, "gelu": B.ACT_GELU, "silu": B.ACT_SILU}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    H.require_gpu()


def _inputs(seed, T, n_in, out, dtype):
    gen = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    return dict(x=r(T, n_in).to(dtype), W=(r(out, n_in) / n_in ** 0.5).to(dtype), b=(0.3 * r(out)).to(dtype), r=r(T, out).to(dtype),
                dy=(0.01 * r(T, out)).to(dtype), z=r(T, out).to(dtype))


def _check_forward(d, act, y, z, bias=True, residual=True):
    x, W = d["x"].double(), d["W"].double()
    b, r = (d["b"].double() if bias else torch.zeros(1)), (d["r"].double() if residual else torch.zeros(1))
    z64, size, K = x @ W.t() + b, x.abs() @ W.abs().t() + b.abs(), x.shape[1]
    if z is not None:
        assert_close(z, z64, size, K + 4, "z")
    # the steepest slope of the activations is 1.13; the functions themselves are good to a few steps of their arguments
    assert_close(y, act64(z64, act) + r, 1.13 * size + r.abs(), K + 40, "y")


def _check_backward(d, act, dz, dx, db, span=None):
    dy, z, W = d["dy"].double(), d["z"].double(), d["W"].double()
    T, out = dy.shape
    g = dy * slope64(z, act)
    size = dy.abs() * (1 + z.abs())                                   # slope: a handful of terms of size 1 and |z|
    if dz is not None:
        assert_close(dz, g, size, 32, "dz")
    if dx is not None:
        # dz enters the product rounded to its type, without an activation as it is
        u = torch.finfo(d["dy"].dtype).eps / 2 if act != "none" else 0.0
        off = u * (g.abs() @ W.abs()) / 2 ** -24                      # in units of the rule
        assert_close(dx, g @ W, (out + 40) * (size @ W.abs()) + off, 1, "dx")
    if db is not None:
        s = slice(*(span or (0, out)))
        assert_close(db, g.sum(0)[s], size.sum(0)[s], T + 40, "db")


def _ws(layer, backward):
    n = B.chunkft_linear_workspace_bytes(layer, backward=backward)
    return torch.empty(n, dtype=torch.uint8, device=DEV) if n else None


# T, in, out: one token to many, on both sides of tiles and of the pieces they are made of; odd sizes lie at odd places
SHAPES = [(1, 1, 1), (1, 64, 128), (1, 4096, 520), (2, 72, 264), (3, 130, 7), (5, 7, 130), (16, 512, 1024), (17, 520, 136), (33, 65, 257),
          (64, 256, 64), (65, 1000, 200), (127, 129, 131), (128, 128, 128), (130, 136, 392), (200, 328, 520), (257, 96, 300), (300, 2051, 40),
          (515, 640, 384)]


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("T,n_in,out", SHAPES)
def test_forward(T, n_in, out, dtype):
    dt = DTYPES[dtype]
    d = _inputs(T * 31 + n_in * 7 + out, T, n_in, out, dt)
    act = ACTS[(T + n_in + out) % 4]
    odd = (n_in | out) & 1
    X, W, b, R = Placed(d["x"], pad=odd, lead=odd), Placed(d["W"], pad=odd), Placed(d["b"], lead=odd), Placed(d["r"], pad=8)
    Y, Z = Placed(torch.zeros(T, out, dtype=dt), pad=odd, lead=odd), Placed(torch.zeros(T, out, dtype=dt), pad=16)
    layer = B.make_linear(X.t, W.t, b.t, CODES[act], R.t)
    B.chunkft_linear_forward(layer, Y.t, Z=Z.t, ws=_ws(layer, False))
    torch.cuda.synchronize()
    _check_forward(d, act, Y.t, Z.t)
    assert all(p.untouched() for p in (X, W, b, R, Y, Z))


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("T,n_in,out", SHAPES)
def test_backward(T, n_in, out, dtype):
    dt = DTYPES[dtype]
    d = _inputs(T * 37 + n_in * 5 + out, T, n_in, out, dt)
    act = ACTS[(T + n_in + out + 1) % 4]
    odd = (n_in | out) & 1
    W, DY, Z = Placed(d["W"], pad=odd, lead=odd), Placed(d["dy"], pad=odd), Placed(d["z"], pad=odd, lead=odd)
    DZ, DX, DB = Placed(torch.zeros(T, out, dtype=dt), lead=odd), Placed(torch.zeros(T, n_in, dtype=dt), pad=odd), Placed(torch.zeros(out), lead=1)
    layer = B.make_linear(None, W.t, activation=CODES[act], tokens=T)
    B.chunkft_linear_backward(layer, DY.t, Z.t, DZ.t, DX.t, db=DB.t, ws=_ws(layer, True))
    torch.cuda.synchronize()
    _check_backward(d, act, None if act == "none" else DZ.t, DX.t, DB.t)
    assert all(p.untouched() for p in (W, DY, Z, DZ, DX, DB))


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("act", ACTS)
def test_each_activation_with_and_without_the_rest(act, dtype):
    dt, T, n_in, out = DTYPES[dtype], 40, 96, 72
    d = _inputs(5, T, n_in, out, dt)
    dev = {k: v.to(DEV) for k, v in d.items()}
    for bias in (False, True):
        for residual in (False, True):
            y = dev["r"].clone() if residual else torch.empty(T, out, dtype=dt, device=DEV)
            layer = B.make_linear(dev["x"], dev["W"], dev["b"] if bias else None, CODES[act], y if residual else None)
            B.chunkft_linear_forward(layer, y, ws=_ws(layer, False))      # onto the residual itself
            torch.cuda.synchronize()
            _check_forward(d, act, y, None, bias, residual)


@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_activations_far_out_and_at_zero(dtype):
    """One input feature of 1 and one output: z is the bias. Slopes from z given."""
    dt = DTYPES[dtype]
    z = torch.tensor([-1e30, -200.0, -88.0, -30.0, -9.0, -1.0, -0.0, 0.0, 1e-30, 0.7, 5.0, 30.0, 200.0, 1e30]).to(dt)
    n = z.shape[0]
    x, W = torch.zeros(1, 8, dtype=dt, device=DEV), torch.zeros(n, 8, dtype=dt, device=DEV)
    for act in ACTS[1:]:
        y = torch.empty(1, n, dtype=dt, device=DEV)
        layer = B.make_linear(x, W, z.to(DEV), CODES[act])
        B.chunkft_linear_forward(layer, y, ws=_ws(layer, False))
        assert_close(y, act64(z.double(), act)[None], z.double().abs()[None].clamp(max=1e3) + 1e-30, 40, act)
        dz, dy = torch.empty(1, n, dtype=dt, device=DEV), torch.ones(1, n, dtype=dt, device=DEV)
        layer = B.make_linear(None, W, activation=CODES[act], tokens=1)
        B.chunkft_linear_backward(layer, dy, z.to(DEV)[None], dz, ws=_ws(layer, True))
        ref = slope64(z.double().clamp(-1e3, 1e3), act)[None]
        assert_close(dz, ref, 1 + z.double().abs()[None].clamp(max=1e3), 40, act)


def test_infinities_stay_in_their_rows_and_columns():
    T, n_in, out = 130, 200, 264
    d = _inputs(2, T, n_in, out, torch.bfloat16)
    d["x"][5, 190] = float("inf")
    d["x"][129, 0] = float("nan")
    d["W"][77, 3] = float("-inf")
    dev = {k: v.to(DEV) for k, v in d.items()}
    y = torch.empty(T, out, dtype=torch.bfloat16, device=DEV)
    layer = B.make_linear(dev["x"], dev["W"])
    B.chunkft_linear_forward(layer, y, ws=_ws(layer, False))
    finite = torch.isfinite(y).cpu()
    want = torch.ones(T, out, dtype=torch.bool)
    want[5], want[129], want[:, 77] = False, False, False
    assert torch.equal(finite, want)
    assert torch.isnan(y[129]).all()


@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_parts_of_the_bias_and_accumulation(dtype):
    dt, T, n_in, out = DTYPES[dtype], 700, 40, 333
    d = _inputs(12, T, n_in, out, dt)
    dev = {k: v.to(DEV) for k, v in d.items()}
    for act in ("none", "silu"):
        layer = B.make_linear(None, dev["W"], activation=CODES[act], tokens=T)
        dz, DB = torch.empty(T, out, dtype=dt, device=DEV), Placed(torch.zeros(100))
        ws = _ws(layer, True)
        B.chunkft_linear_backward(layer, dev["dy"], dev["z"], dz, db=DB.t, b_range=(200, 300), ws=ws)
        torch.cuda.synchronize()
        _check_backward(d, act, None, None, DB.t, (200, 300))
        once = DB.t.clone()
        B.chunkft_linear_backward(layer, dev["dy"], dev["z"], dz, db=DB.t, b_range=(200, 300), accumulate=True, ws=ws)
        torch.cuda.synchronize()
        assert torch.equal(DB.t, once + once) and DB.untouched()


def test_same_bits_again_and_in_a_graph_on_another_stream():
    T, n_in, out = 300, 520, 392
    d = {k: v.to(DEV) for k, v in _inputs(1, T, n_in, out, torch.bfloat16).items()}
    fwd, bwd = B.make_linear(d["x"], d["W"], d["b"], B.ACT_GELU, d["r"]), B.make_linear(None, d["W"], activation=B.ACT_GELU, tokens=T)
    wsf, wsb = _ws(fwd, False), _ws(bwd, True)

    def outputs():
        e = lambda *s: torch.empty(*s, dtype=torch.bfloat16, device=DEV)  # noqa: E731
        return e(T, out), e(T, out), e(T, out), e(T, n_in), torch.empty(out, device=DEV)

    def step(o, stream=None):
        B.chunkft_linear_forward(fwd, o[0], Z=o[1], ws=wsf, stream=stream)
        B.chunkft_linear_backward(bwd, d["dy"], o[1], o[2], o[3], db=o[4], ws=wsb, stream=stream)

    eager, captured = outputs(), outputs()
    step(eager)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(captured)
    for _ in range(3):
        for t in captured:
            t.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(eager, captured))
        d["x"].mul_(1.5)
        step(eager)
        torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("n_in", [1, 2, 3])
@pytest.mark.parametrize("out", [65, 66, 71, 128, 135])
def test_input_gradient_of_rows_narrower_than_a_piece(n_in, out, dtype):
    """16 bytes of W hold several of its rows; what lies behind the last one is not a number."""
    dt, T = DTYPES[dtype], 40
    d = _inputs(n_in * 100 + out, T, n_in, out, dt)
    room = torch.full((out * n_in + 64,), float("nan"), dtype=dt, device=DEV)
    room[:out * n_in] = d["W"].reshape(-1).to(DEV)
    dx = torch.empty(T, n_in, dtype=dt, device=DEV)
    layer = B.make_linear(None, room[:out * n_in].view(out, n_in), tokens=T)
    B.chunkft_linear_backward(layer, d["dy"].to(DEV), dX=dx, ws=_ws(layer, True))
    torch.cuda.synchronize()
    W, dy = d["W"].double(), d["dy"].double()
    assert_close(dx, dy @ W, (out + 4) * (dy.abs() @ W.abs()), 1, "dx")
