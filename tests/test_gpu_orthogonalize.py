"""Newton-Schulz orthogonalisation and the chunk update with it on the GPU, against 64 bits.

The bounds follow the roundings through the steps (layers_harness.newton_schulz_bound): 11 digits for bf16 results, 22 for fp32."""

import pytest
import torch

from paper_2605_21177_amd import binding as B

import gpu_harness as H
from layers_harness import DEV, Placed, newton_schulz64, newton_schulz_bound

pytestmark = pytest.mark.gpu

EPS = 1e-7


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    H.require_gpu()


def _matrix(seed, rows, cols, scale=1e-3):
    gen = torch.Generator().manual_seed(seed)
    rank = max(1, min(rows, cols) // 16)
    low = torch.randn(rows, rank, generator=gen) @ torch.randn(rank, cols, generator=gen) / rank ** 0.5
    return scale * (low + torch.randn(rows, cols, generator=gen))


def _ws(precision, rows, cols):
    return torch.empty(B.chunkft_orthogonalize_workspace_bytes(precision, rows, cols), dtype=torch.uint8, device=DEV)


def _bound(u, steps, dtype):
    out = float(torch.linalg.matrix_norm(newton_schulz64(u, steps, EPS)))
    digits, last = (11, 2.0 ** -8) if dtype is torch.bfloat16 else (22, 2.0 ** -24)
    return newton_schulz_bound(u, steps, EPS, digits, dtype is torch.bfloat16) + last * out


SHAPES = [(1, 1), (1, 300), (300, 1), (3, 5), (64, 64), (65, 130), (128, 128), (130, 65), (129, 257), (400, 72), (72, 400), (256, 512), (301, 299)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_orthogonalize(rows, cols, dtype):
    g = _matrix(rows * 7 + cols, rows, cols).to(dtype)
    odd = cols & 1
    G, O = Placed(g, pad=3 * odd, lead=odd), Placed(torch.zeros(rows, cols, dtype=dtype), pad=5 * odd, lead=odd)
    for steps in (1, 5):
        B.chunkft_orthogonalize(G.t, O.t, steps=steps, eps=EPS, ws=_ws(B.BF16 if dtype is torch.bfloat16 else B.F32, rows, cols))
        torch.cuda.synchronize()
        u = g.double()
        err = float(torch.linalg.matrix_norm(O.t.cpu().double() - newton_schulz64(u, steps, EPS)))
        assert err <= _bound(u, steps, dtype), (steps, err, _bound(u, steps, dtype))
        assert G.untouched() and O.untouched()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_scale_does_not_matter_until_eps_does(dtype):
    g = _matrix(3, 40, 90, 1.0).to(dtype)
    ws = _ws(B.BF16 if dtype is torch.bfloat16 else B.F32, 40, 90)
    o, p = torch.empty_like(g, device=DEV), torch.empty_like(g, device=DEV)
    B.chunkft_orthogonalize(g.to(DEV), o, eps=0.0, ws=ws)
    for exponent in (-100, -40, 60, 100):
        B.chunkft_orthogonalize((g * 2.0 ** exponent).to(DEV), p, eps=0.0, ws=ws)
        torch.cuda.synchronize()
        assert torch.equal(o, p), exponent
    # in place, and the same bits
    q = g.to(DEV)
    B.chunkft_orthogonalize(q, q, eps=0.0, ws=ws)
    torch.cuda.synchronize()
    assert torch.equal(o, q)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_zero_tiny_and_non_finite_matrices(dtype):
    ws = _ws(B.BF16 if dtype is torch.bfloat16 else B.F32, 30, 200)
    o = torch.empty(30, 200, dtype=dtype, device=DEV)
    B.chunkft_orthogonalize(torch.zeros_like(o), o, ws=ws)
    assert bool((o == 0).all())
    for value in (float("inf"), float("nan")):
        g = _matrix(5, 30, 200).to(dtype)
        g[7, 11] = value
        B.chunkft_orthogonalize(g.to(DEV), o, ws=ws)
        assert bool(torch.isnan(o).all())
    g = _matrix(5, 30, 200, 1e-10).to(dtype)                            # eps is most of the denominator: linear, a^5 U / eps
    B.chunkft_orthogonalize(g.to(DEV), o, eps=1.0, ws=ws)
    ref = newton_schulz64(g.double(), 5, 1.0)
    assert float(torch.linalg.matrix_norm(o.cpu().double() - ref)) <= 1e-2 * float(torch.linalg.matrix_norm(ref))


def test_rank_one_and_a_spike():
    """One direction: its singular value goes the scalar way; what the roundings leave beside it stays inside the bound."""
    gen = torch.Generator().manual_seed(2)
    g = torch.randn(100, 1, generator=gen) @ torch.randn(1, 260, generator=gen)
    spike = torch.zeros(100, 260)
    spike[31, 200] = -5.0
    for u in (g, spike):
        o = torch.empty_like(u, device=DEV)
        B.chunkft_orthogonalize(u.to(DEV), o, eps=EPS, ws=_ws(B.F32, 100, 260))
        err = float(torch.linalg.matrix_norm(o.cpu().double() - newton_schulz64(u.double(), 5, EPS)))
        assert err <= _bound(u.double(), 5, torch.float32), err


@pytest.mark.parametrize("precision,digits", [(B.F32, 22), (B.BF16, 11)])
@pytest.mark.parametrize("rows,cols,nesterov", [(8, 264, True), (136, 72, False), (200, 301, True), (1, 50, True)])
def test_muon_chunk(rows, cols, nesterov, precision, digits):
    n = rows * cols
    gen = torch.Generator().manual_seed(rows + cols)
    g, m0 = _matrix(rows, rows, cols), _matrix(cols, rows, cols, 3e-3)
    th0 = 0.02 * torch.randn(rows, cols, generator=gen)
    hp = dict(lr=0.02, momentum=0.95, weight_decay=0.1, eps=EPS, scale=1.5)
    G, M, TH = Placed(g.reshape(-1), lead=1), Placed(m0.reshape(-1), lead=3), Placed(th0.reshape(-1), lead=2)
    Wt = Placed(torch.zeros(n, dtype=torch.bfloat16), lead=5)
    B.chunkft_muon_chunk(G.t, TH.t, M.t, Wt.t, rows, cols, B.muon_hparams(**hp, nesterov=nesterov, precision=precision), ws=_ws(precision, rows, cols))
    torch.cuda.synchronize()
    mu = float(torch.tensor(hp["momentum"]))
    m = mu * m0.double() + g.double()
    assert float((M.t.cpu().double().view(rows, cols) - m).abs().max()) <= 4 * 2 ** -24 * float((mu * m0.abs() + g.abs()).max())
    u = g.double() + mu * m if nesterov else m
    o = newton_schulz64(u, 5, EPS)
    th = th0.double() - hp["lr"] * (hp["scale"] * o + hp["weight_decay"] * th0.double())
    got = TH.t.cpu().double().view(rows, cols)
    # U itself is good to a few fp32 steps; the update's own arithmetic to three roundings of theta
    start = 8 * 2.0 ** -24 * float(torch.linalg.matrix_norm(u)) / float(torch.linalg.matrix_norm(u)) * 3.96 ** 5
    far = hp["lr"] * hp["scale"] * (newton_schulz_bound(u, 5, EPS, digits, False) + start) + 4 * 2 ** -24 * float(torch.linalg.matrix_norm(th))
    err = float(torch.linalg.matrix_norm(got - th))
    assert err <= far, (err, far)
    assert torch.equal(Wt.t, TH.t.bfloat16())
    assert all(p.untouched() for p in (G, M, TH, Wt))


def test_muon_chunk_without_weights_with_fp32_weights_and_in_a_graph():
    rows, cols = 144, 328
    g = _matrix(1, rows, cols).to(DEV)
    hp = B.muon_hparams(0.01, 0.9, 0.0, scale=0.5)
    start = 0.02 * torch.randn(rows, cols, generator=torch.Generator().manual_seed(3)).to(DEV)

    def fresh():
        return start.clone(), torch.zeros(rows, cols, device=DEV), torch.zeros(rows, cols, device=DEV)

    ws, ws2 = _ws(B.F32, rows, cols), _ws(B.F32, rows, cols)
    a, b = fresh(), fresh()
    for _ in range(4):
        B.chunkft_muon_chunk(g, a[0], a[1], a[2], rows, cols, hp, w_dtype=B.F32, ws=ws)
    B.chunkft_muon_chunk(g, b[0], b[1], None, rows, cols, hp, ws=ws2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        B.chunkft_muon_chunk(g, b[0], b[1], None, rows, cols, hp, ws=ws2)
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        B.chunkft_orthogonalize(g, torch.empty_like(g), ws=ws)
    torch.cuda.synchronize()
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]) and torch.equal(a[2], a[0])


@pytest.mark.parametrize("rows,cols", [(512, 512), (300, 1100), (1100, 300)])
def test_three_steps_from_small_singular_values_keep_float32(rows, cols):
    """Every singular value is small, so each step is nearly x -> a x and keeps relative errors as they are.  A step adds at most
    2^-22 / 3 from the two parts (each residue is uniform: its root mean square is its largest value over sqrt 3), 2^-24 / sqrt 3 each
    from the product a x and the sum, and four roundings of 2^-24 of factors common to all values: 3.8e-7.  The last step's products
    add sqrt(3 K / 32) roundings of 2^-24 of a part smaller than a x: 4.4e-7 for K = 512.  Three steps: 1.6e-6."""
    g = torch.randn(rows, cols, generator=torch.Generator().manual_seed(rows))
    o = torch.empty(rows, cols, device=DEV)
    B.chunkft_orthogonalize(g.to(DEV), o, steps=3, eps=0.0, ws=_ws(B.F32, rows, cols))
    torch.cuda.synchronize()
    want = newton_schulz64(g.double(), 3, 0.0)
    err = float(torch.linalg.matrix_norm(o.cpu().double() - want) / torch.linalg.matrix_norm(want))
    assert err <= 1.6e-6, err


@pytest.mark.parametrize("rows,cols", [(200, 2000), (2000, 200), (64, 4096), (256, 256)])
def test_five_steps_leave_bf16_results_little_more_than_their_rounding(rows, cols):
    """The rounding of the result is 1.7e-3 of its norm (root mean square of half steps over the mantissas).  Operands of 11 digits
    are off by 1e-4 of theirs; a step multiplies what is off by up to 1.6 once the singular values have arrived (the slope of
    a x + b x^3 + c x^5 near 0.87), 1 + 1.6 + 1.6^2 + 1.6^3 = 9.3 times that in the end for each of X, A and the polynomial: sqrt(3) x 9.3e-4
    = 1.6e-3.  Together 2.4e-3."""
    gen = torch.Generator().manual_seed(rows + cols)
    low = torch.randn(rows, 3, generator=gen) @ torch.randn(3, cols, generator=gen) / 3 ** 0.5
    g = (1e-3 * (low + torch.randn(rows, cols, generator=gen))).bfloat16()
    o = torch.empty_like(g, device=DEV)
    B.chunkft_orthogonalize(g.to(DEV), o, eps=EPS, ws=_ws(B.BF16, rows, cols))
    torch.cuda.synchronize()
    want = newton_schulz64(g.double(), 5, EPS)
    err = float(torch.linalg.matrix_norm(o.cpu().double() - want) / torch.linalg.matrix_norm(want))
    assert err <= 2.4e-3, err
