"""The layers and orthogonalised updates at sizes of many tiles (each width of tile, slabs of them, partial last stages), at offsets past
32 bits, and in two streams at once.  References in 64 bits on the device, products of two plain matrices."""

import pytest
import torch

from paper_2605_21177_amd import binding as B

import gpu_harness as H
from layers_harness import DEV, U32, half_step

pytestmark = pytest.mark.gpu


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


def _ws(n):
    return torch.empty(n, dtype=torch.uint8, device=DEV) if n else None


# both directions of: one tile of 256 a unit, more columns than rows, a partial last stage, slabs of 256- and 128-wide tiles, 64 x 128
# tiles, rows without pieces
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,n_in,out", [(4096, 512, 4096), (2048, 520, 8192), (1024, 14336, 4096), (4100, 264, 2056), (2056, 264, 4104),
                                        (1024, 2048, 2048), (3000, 328, 5000), (1001, 2907, 2705)])
def test_linear(T, n_in, out, dtype):
    gen = torch.Generator(device=DEV).manual_seed(T + n_in + out)
    x, W, b = _randn(gen, T, n_in).to(dtype), (_randn(gen, out, n_in) / n_in ** 0.5).to(dtype), _randn(gen, out).to(dtype)
    r, dy = _randn(gen, T, out).to(dtype), _randn(gen, T, out).to(dtype)
    layer = B.make_linear(x, W, b, B.ACT_RELU, r)
    y, dx = torch.empty_like(r), torch.empty_like(x)
    B.chunkft_linear_forward(layer, y, ws=_ws(B.chunkft_linear_workspace_bytes(layer)))
    z, size = torch.addmm(b.double(), x.double(), W.double().t()), x.double().abs() @ W.double().abs().t() + b.double().abs()
    _close(y, z.clamp(min=0) + r.double(), size + r.double().abs(), n_in + 4, "y")
    layer = B.make_linear(None, W, tokens=T)
    B.chunkft_linear_backward(layer, dy, dX=dx, ws=_ws(B.chunkft_linear_workspace_bytes(layer, backward=True)))
    _close(dx, dy.double() @ W.double(), dy.double().abs() @ W.double().abs(), out + 4, "dx")


def _newton_schulz(u):
    x = u / u.norm()
    x = x.t().contiguous() if u.shape[0] > u.shape[1] else x
    for _ in range(5):
        a = x @ x.t()
        x = 3.4445 * x + (-4.7750 * a + 2.0315 * (a @ a)) @ x
    return x.t() if u.shape[0] > u.shape[1] else x


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols", [(2000, 2100), (2600, 2700), (900, 3000), (2907, 1003), (4096, 4096), (8192, 2048)])
def test_orthogonalize(rows, cols, dtype):
    """bf16: 2.4e-3 as for smaller matrices (rounding of the result, and of operands of 11 digits).  fp32: three steps from small singular
    values leave 1.6e-6, two more multiply it by at most 1.6^2; in these the products are of the result's size, sqrt(3 K / 32) roundings of 2^-24
    with K = 8192: 1.7e-6 a product, 2 products a step, 1 + 1.6 times: 8.8e-6; together 1.3e-5."""
    gen = torch.Generator(device=DEV).manual_seed(rows + cols)
    rank = min(rows, cols) // 64
    g = (1e-3 * (_randn(gen, rows, rank) @ _randn(gen, rank, cols) / rank ** 0.5 + _randn(gen, rows, cols))).to(dtype)
    o = torch.empty_like(g)
    B.chunkft_orthogonalize(g, o, eps=0.0, ws=_ws(B.chunkft_orthogonalize_workspace_bytes(B._torch_dtype_code(g), rows, cols)))
    want = _newton_schulz(g.double())
    off = float((o.double() - want).norm() / want.norm())
    assert off <= (2.4e-3 if dtype is torch.bfloat16 else 1.3e-5), off


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_offsets_past_32_bits(dtype):
    """Rows 2^27 elements apart: the same bits as from rows side by side."""
    gen, T, n, out = torch.Generator(device=DEV).manual_seed(1), 40, 72, 136
    far = torch.empty(T * (1 << 27), dtype=dtype, device=DEV).view(T, 1 << 27)

    def apart(t, at):
        v = far[:t.shape[0], at:at + t.shape[1]]
        v.copy_(t)
        return v

    x, W, dy = _randn(gen, T, n).to(dtype), _randn(gen, n, out).to(dtype).t().contiguous(), _randn(gen, T, n).to(dtype)
    X, DY, Y, Y2 = apart(x, 0), apart(dy, 1024), apart(torch.zeros_like(x), 2048), apart(torch.zeros(T, out, dtype=dtype, device=DEV), 4096)
    w = _randn(gen, n).to(dtype)
    got, want = [], []
    for x_, dy_, y_, y2_, to in ((X, DY, Y, Y2, got), (x, dy, torch.empty_like(x), torch.empty(T, out, dtype=dtype, device=DEV), want)):
        stats, dw = torch.empty(T, 2, device=DEV), torch.empty(n, device=DEV)
        layer = B.make_norm(B.LAYERNORM, x_, w)
        B.chunkft_norm_forward(layer, y_, stats)
        to.append(y_.clone())
        B.chunkft_norm_backward(layer, stats, dy_, y_, dw=dw, ws=_ws(B.chunkft_norm_workspace_bytes(layer)))
        to += [y_.clone(), dw, stats]
        for tokens in (5, T):                                              # the pass over the weights, and tiles
            lin = B.make_linear(x_[:tokens], W)
            B.chunkft_linear_forward(lin, y2_[:tokens], ws=_ws(B.chunkft_linear_workspace_bytes(lin)))
            to.append(y2_[:tokens].clone())
        B.chunkft_orthogonalize(x_, y_, ws=_ws(B.chunkft_orthogonalize_workspace_bytes(B._torch_dtype_code(x), T, n)))
        to.append(y_.clone())
    for i, (a, b) in enumerate(zip(got, want)):
        if i in (4, 5) and dtype is torch.bfloat16:                        # other rows, other loads: equal up to the sums' order
            assert float((a.double() - b.double()).norm() / b.double().norm()) <= 2.0 ** -8, i
        else:
            assert torch.equal(a, b), i


def test_two_streams_at_once_with_workspaces_of_their_own():
    gen = torch.Generator(device=DEV).manual_seed(2)
    g = [_randn(gen, 700, 900).bfloat16() for _ in range(2)]
    x, W = [_randn(gen, 200, 4096).bfloat16() for _ in range(2)], _randn(gen, 520, 4096).bfloat16()

    def enqueue(i, stream):
        o, y = torch.empty_like(g[i]), torch.empty(200, 520, dtype=torch.bfloat16, device=DEV)
        layer = B.make_linear(x[i], W, activation=B.ACT_SILU)
        ws = _ws(B.chunkft_orthogonalize_workspace_bytes(B.BF16, 700, 900)), _ws(B.chunkft_linear_workspace_bytes(layer))
        torch.cuda.synchronize()
        return lambda: (B.chunkft_orthogonalize(g[i], o, ws=ws[0], stream=stream), B.chunkft_linear_forward(layer, y, ws=ws[1], stream=stream)), (o, y), ws

    alone = [enqueue(i, torch.cuda.current_stream()) for i in range(2)]
    for run, _, _ in alone:
        run()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    both = [enqueue(i, s) for i, s in enumerate(streams)]
    for _ in range(4):
        for run, _, _ in both:
            run()
    torch.cuda.synchronize()
    for (_, a, _), (_, b, _) in zip(alone, both):
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("T,n_in,out,pad,lead", [(2047, 1023, 1025, 0, 0), (2000, 500, 500, 12, 4), (1500, 1001, 1200, 7, 1), (1500, 1024, 1201, 0, 0), (3001, 1090, 1100, 2, 3)])
def test_linear_rows_without_pieces(T, n_in, out, pad, lead):
    """bf16 rows at odd places, copied or not, inside buffers that hold no numbers elsewhere; a workspace that holds none either."""
    gen = torch.Generator(device=DEV).manual_seed(T + n_in + out)

    def inside(t):
        rows, cols = t.shape
        v = torch.full((lead + rows * (cols + pad) + 64,), float("nan"), dtype=torch.bfloat16, device=DEV)[lead:lead + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
        return v.copy_(t)

    def ws(n):
        return torch.full((n // 4,), float("nan"), device=DEV) if n else None

    x, W, dy = inside(_randn(gen, T, n_in)), inside(_randn(gen, out, n_in) / n_in ** 0.5), inside(_randn(gen, T, out))
    y, dx = inside(torch.zeros(T, out, device=DEV)), inside(torch.zeros(T, n_in, device=DEV))
    layer = B.make_linear(x, W)
    B.chunkft_linear_forward(layer, y, ws=ws(B.chunkft_linear_workspace_bytes(layer)))
    _close(y, x.double() @ W.double().t(), x.double().abs() @ W.double().abs().t(), n_in + 4, "y")
    layer, db = B.make_linear(None, W, tokens=T), torch.empty(out, device=DEV)
    B.chunkft_linear_backward(layer, dy, dX=dx, db=db, ws=ws(B.chunkft_linear_workspace_bytes(layer, backward=True)))
    _close(dx, dy.double() @ W.double(), dy.double().abs() @ W.double().abs(), out + 4, "dx")
    _close(db, dy.double().sum(0), dy.double().abs().sum(0), T + 4, "db")
