"""The linear layer on rows that lie in every way the products take them: along and across k, in 16-byte pieces by their sizes or by
their strides alone, elsewhere, in buffers that hold no numbers around them; and what a value that is no number reaches."""

import pytest
import torch

from paper_2605_21177_amd import binding as B

import gpu_harness as H
from layers_harness import DEV, U32, half_step

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    H.require_gpu()


def _randn(gen, *shape):
    return torch.randn(*shape, generator=gen, device=DEV)


def _close(got, ref, sums, count, what):
    """The rule of layers_harness.assert_close, on the device."""
    u = half_step(got.dtype)
    bound = u * ref.abs() * (1 + 2 * u) + count * U32 * sums
    worst = float(((got.double() - ref).abs() / bound).max())
    assert worst <= 1, (what, worst)


def _inside(t, pad, lead):
    """A copy of t, `pad` elements between its rows and `lead` in front of them, in a buffer of NaN."""
    rows, cols = t.shape
    raw = torch.full((lead + rows * (cols + pad) + 64,), float("nan"), dtype=t.dtype, device=DEV)
    return raw[lead:lead + rows * (cols + pad)].view(rows, cols + pad)[:, :cols].copy_(t)


def _ws(n):
    return torch.full((n // 4,), float("nan"), device=DEV) if n else None


# tokens, in, out, elements between the rows and in front of them
ROWS = [(512, 1024, 2049, 0, 0), (300, 4096, 1001, 0, 0), (700, 520, 777, 0, 0),              # W has an odd number of rows
        (600, 1003, 1000, 5, 0), (600, 1003, 1000, 5, 8), (900, 2907, 1200, 5, 16), (64, 4091, 520, 5, 0),   # pieces by their strides
        (512, 1024, 2048, 8, 3), (512, 1024, 2048, 1, 0), (1024, 4096, 520, 2, 2),              # sizes of pieces, elsewhere
        (300, 40, 1001, 0, 0), (300, 1001, 40, 0, 0), (100, 33, 1000, 7, 0),                     # fewer values than a stage
        (200, 1608, 300, 0, 0)]                                                                  # slabs whose last one would hold 8 values


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("T,n_in,out,pad,lead", ROWS)
def test_rows(T, n_in, out, pad, lead, dtype):
    gen, dt = torch.Generator(device=DEV).manual_seed(T + n_in + out + pad), DTYPES[dtype]
    x, W, dy = (_inside(t.to(dt), pad, lead) for t in (_randn(gen, T, n_in), _randn(gen, out, n_in) / n_in ** 0.5, _randn(gen, T, out)))
    y, dx = (_inside(torch.zeros(s, dtype=dt, device=DEV), pad, lead) for s in ((T, out), (T, n_in)))
    layer = B.make_linear(x, W)
    B.chunkft_linear_forward(layer, y, ws=_ws(B.chunkft_linear_workspace_bytes(layer)))
    _close(y, x.double() @ W.double().t(), x.double().abs() @ W.double().abs().t(), n_in + 4, "y")
    layer = B.make_linear(None, W, tokens=T)
    B.chunkft_linear_backward(layer, dy, dX=dx, ws=_ws(B.chunkft_linear_workspace_bytes(layer, backward=True)))
    _close(dx, dy.double() @ W.double(), dy.double().abs() @ W.double().abs(), out + 4, "dx")


# the pass over the weights, registers, direct loads with and without a partial stage, copies, slabs
@pytest.mark.parametrize("act", ["none", "gelu", "silu", "relu"])
@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("T,n_in,out", [(1, 200, 264), (7, 201, 263), (130, 200, 264), (130, 201, 263), (300, 1001, 1203), (96, 4096, 520), (520, 1024, 777)])
def test_values_that_are_no_numbers_stay_in_their_rows_and_columns(T, n_in, out, dtype, act):
    """An infinity or NaN in x reaches its token's outputs alone, in W its column, in the bias its column, in the residual its element; in
    dy its token's input gradient, in z its own element of dz and its token's input gradient, and both their column of the bias'."""
    gen, dt = torch.Generator(device=DEV).manual_seed(T + n_in), DTYPES[dtype]
    code = dict(none=B.ACT_NONE, gelu=B.ACT_GELU, silu=B.ACT_SILU, relu=B.ACT_RELU)[act]
    nan, inf = float("nan"), float("inf")
    x, W, b, r = _randn(gen, T, n_in).to(dt), _randn(gen, out, n_in).to(dt), _randn(gen, out).to(dt), _randn(gen, T, out).to(dt)
    x[T - 1, n_in - 1], W[77, 3], W[out - 1, n_in - 1], b[5], r[T // 2, 9] = nan, nan, nan, nan, inf
    y, z = torch.empty_like(r), torch.empty_like(r)
    layer = B.make_linear(x, W, b, code, r)
    B.chunkft_linear_forward(layer, y, Z=z, ws=_ws(B.chunkft_linear_workspace_bytes(layer)))
    want = torch.ones(T, out, dtype=torch.bool, device=DEV)
    want[T - 1], want[:, 77], want[:, out - 1], want[:, 5] = False, False, False, False
    assert torch.equal(torch.isfinite(z), want)
    want[T // 2, 9] = False
    assert torch.equal(torch.isfinite(y), want)

    W, dy, z = _randn(gen, out, n_in).to(dt), _randn(gen, T, out).to(dt), _randn(gen, T, out).to(dt)
    t = T // 3
    dy[T - 1, out - 1], W[out // 2, 1] = nan, nan
    if act != "none" and act != "relu":                       # (relu's slope at NaN is that of a z that is not above zero)
        z[t, 4] = nan
    dz, dx, db = torch.empty_like(dy), torch.empty(T, n_in, dtype=dt, device=DEV), torch.empty(out, device=DEV)
    layer = B.make_linear(None, W, activation=code, tokens=T)
    B.chunkft_linear_backward(layer, dy, z, dz, dx, db=db, ws=_ws(B.chunkft_linear_workspace_bytes(layer, backward=True)))
    rows, cols = torch.ones(T, n_in, dtype=torch.bool, device=DEV), torch.ones(out, dtype=torch.bool, device=DEV)
    rows[T - 1], rows[:, 1], cols[out - 1] = False, False, False
    if act in ("gelu", "silu"):
        rows[t], cols[4] = False, False
    assert torch.equal(torch.isfinite(dx), rows) and torch.equal(torch.isfinite(db), cols)
    if act != "none":
        elements = torch.ones(T, out, dtype=torch.bool, device=DEV)
        elements[T - 1, out - 1] = False
        if act != "relu":
            elements[t, 4] = False
        assert torch.equal(torch.isfinite(dz), elements)
