"""Limits of the orthogonalised results that are far below the results themselves, for every size and for the update of a chunk.

Relative to the norm of the result, five steps.  A step multiplies what is off by at most 1.6 once the singular values have arrived (the
slope of a x + b x^3 + c x^5 near 0.87); before, relative errors do not grow.  What X, A and the polynomial are rounded to is so
multiplied by 1 + 1.6 + 1.6^2 + 1.6^3 = 9.3 in the end.

  many values (a small side of 64 or more): roundings are off by their root mean square, and the three add up as such: 2.4e-3 with the
  result's own in bf16 (11 digits), 1.3e-5 in fp32 (22 digits, and the roundings of the sums)
  fewer: each is off by up to half a step, and the three add up as they are: 3 x 9.3 x 2^-11 = 1.4e-2 and the result's half step 2^-8, together
  1.8e-2; in fp32 3 x 9.3 x 2^-22 = 6.7e-6 and the roundings of sums of few terms: 1.3e-5 again."""

import pytest
import torch

from paper_2605_21177_amd import binding as B

from layers_harness import A_, B_, C_, DEV, newton_schulz64

EPS = 1e-7
SHAPES = [(1, 1), (1, 50), (1, 300), (300, 1), (3, 5), (8, 264), (16, 16), (33, 100), (64, 64), (65, 130), (128, 128), (130, 65), (129, 257), (400, 72),
          (72, 400), (256, 512), (301, 299), (512, 1500)]


def limit(rows, cols, digits):
    if digits == 22:
        return 1.3e-5
    return 2.4e-3 if min(rows, cols) >= 64 else 1.8e-2


def matrix(seed, rows, cols, scale=1e-3):
    gen = torch.Generator().manual_seed(seed)
    rank = max(1, min(rows, cols) // 16)
    low = torch.randn(rows, rank, generator=gen) @ torch.randn(rank, cols, generator=gen) / rank ** 0.5
    return scale * (low + torch.randn(rows, cols, generator=gen))


def off(got, want):
    return float(torch.linalg.matrix_norm(got.double().cpu() - want) / torch.linalg.matrix_norm(want))


def rounded(u, digits, steps=5):
    """The steps in 64 bits with X, A and the polynomial without its diagonal rounded to `digits` digits between the products."""
    def to(x):
        m, e = torch.frexp(x)
        return torch.ldexp(torch.round(m * 2.0 ** digits) / 2.0 ** digits, e)

    tall = u.shape[0] > u.shape[1]
    x = u.t() if tall else u
    x = x / (torch.linalg.matrix_norm(x) + EPS)
    for k in range(steps):
        a = to(x @ x.t())
        p = B_ * a + C_ * a @ a
        d = torch.diagonal(p) + A_
        x = to(p - torch.diag(torch.diagonal(p))) @ x + d[:, None] * x
        x = to(x) if k + 1 < steps else x
    return x.t() if tall else x


@pytest.mark.parametrize("rows,cols", SHAPES)
def test_the_limits_hold_the_roundings_and_little_else(rows, cols):
    """On the CPU: the stated roundings stay inside; no result, half of one, one of a step less and one without the polynomial do not."""
    for seed in range(3):
        u = matrix(seed, rows, cols).bfloat16().double()
        want = newton_schulz64(u, 5, EPS)
        assert off(rounded(u, 11).bfloat16(), want) <= limit(rows, cols, 11)
        assert off(rounded(u, 22).float(), want) <= limit(rows, cols, 22)
        for wrong in (torch.zeros_like(want), 0.5 * want, newton_schulz64(u, 4, EPS), A_ ** 5 * u / torch.linalg.matrix_norm(u)):
            assert off(wrong, want) > 2 * limit(rows, cols, 11)


def _ws(precision, rows, cols):
    return torch.empty(B.chunkft_orthogonalize_workspace_bytes(precision, rows, cols), dtype=torch.uint8, device=DEV)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_orthogonalize(rows, cols, dtype):
    precision, digits = (B.BF16, 11) if dtype is torch.bfloat16 else (B.F32, 22)
    for seed in range(3):
        g = matrix(seed, rows, cols).to(dtype)
        o = torch.empty_like(g, device=DEV)
        B.chunkft_orthogonalize(g.to(DEV), o, eps=EPS, ws=_ws(precision, rows, cols))
        torch.cuda.synchronize()
        err = off(o, newton_schulz64(g.double(), 5, EPS))
        assert err <= limit(rows, cols, digits), (seed, err)


@pytest.mark.gpu
@pytest.mark.parametrize("precision,digits", [(B.F32, 22), (B.BF16, 11)])
@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("rows,cols", [(1, 50), (8, 264), (136, 72), (200, 301), (72, 400), (512, 1500)])
def test_the_orthogonalised_part_of_the_update(rows, cols, nesterov, precision, digits):
    """theta before minus theta after, over lr scale, against O(U): what the rounding of theta leaves of it (half a step of what is near
    0.02, 2^-24 of its norm, three times) is added to the limit, and so is that of U (a few steps of fp32, times 9.3)."""
    g, m0 = matrix(rows, rows, cols), matrix(cols, rows, cols, 3e-3)
    th0 = 0.02 * torch.randn(rows, cols, generator=torch.Generator().manual_seed(rows + cols))
    lr, mu, scale = 0.02, 0.95, 1.5
    master, m, W = th0.to(DEV), m0.to(DEV), torch.empty(rows, cols, dtype=torch.bfloat16, device=DEV)
    hp = B.muon_hparams(lr, mu, 0.0, EPS, scale, nesterov=nesterov, precision=precision)
    B.chunkft_muon_chunk(g.to(DEV), master, m, W, rows, cols, hp, ws=_ws(precision, rows, cols))
    torch.cuda.synchronize()
    mu = float(torch.tensor(mu))
    m1 = mu * m0.double() + g.double()
    want = newton_schulz64(g.double() + mu * m1 if nesterov else m1, 5, EPS)
    got = (th0.double() - master.cpu().double()) / (lr * scale)
    theta = 3 * 2.0 ** -24 * float(th0.double().norm()) / (lr * scale) / float(want.norm())
    assert off(got, want) <= limit(rows, cols, digits) + 9.3 * 8 * 2.0 ** -24 + theta, (off(got, want), theta)
    assert limit(rows, cols, digits) + theta < 0.05
    assert torch.equal(W, master.bfloat16())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("exponent", [-130, -120, 110, 125])
def test_norms_at_the_ends_of_the_range(exponent, dtype):
    """Elements that are subnormal, or near the largest: the same digits."""
    g = (matrix(3, 72, 130, 0.25).double() * 2.0 ** exponent).to(dtype)
    o = torch.empty_like(g, device=DEV)
    precision, digits = (B.BF16, 11) if dtype is torch.bfloat16 else (B.F32, 22)
    B.chunkft_orthogonalize(g.to(DEV), o, eps=0.0, ws=_ws(precision, 72, 130))
    torch.cuda.synchronize()
    err = off(o, newton_schulz64(g.double(), 5, 0.0))
    assert err <= limit(72, 130, digits), err
