"""The activations by themselves, through the layer's calls: an input of zeros, so that z is the bias (forward) or what is given
(backward).  Relative limits, in units of 2^-24 (half a step of fp32): functions whose argument is rounded are off in proportion to it."""

import math

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


def _values(lo, hi, n, dtype):
    z = torch.cat([torch.linspace(lo, hi, n, dtype=torch.float64), torch.tensor([0.0, -1e-3, 1e-3, -0.751, -1.2785], dtype=torch.float64)])
    return z.to(dtype)


def _run(z, act, tokens):
    """act(z) of `tokens` tokens and dz for dy = 1."""
    n, dtype = z.shape[0], z.dtype
    x, W, zd = torch.zeros(tokens, 8, dtype=dtype, device=DEV), torch.zeros(n, 8, dtype=dtype, device=DEV), z.to(DEV)
    y, dz = torch.empty(tokens, n, dtype=dtype, device=DEV), torch.empty(tokens, n, dtype=dtype, device=DEV)
    layer = B.make_linear(x, W, zd, act)
    need = B.chunkft_linear_workspace_bytes(layer)
    B.chunkft_linear_forward(layer, y, ws=torch.empty(need, dtype=torch.uint8, device=DEV) if need else None)
    layer = B.make_linear(None, W, activation=act, tokens=tokens)
    B.chunkft_linear_backward(layer, torch.ones_like(y), zd.expand(tokens, n).contiguous(), dz)
    torch.cuda.synchronize()
    assert torch.equal(y, y[:1].expand_as(y)) and torch.equal(dz, dz[:1].expand_as(dz))
    return y[0].cpu().double(), dz[0].cpu().double()


def _within(got, ref, size, count, dtype, what):
    """|got - ref| <= count 2^-24 size, and the rounding to the type."""
    u = half_step(dtype) if dtype is not torch.float32 else 0.0
    bound = u * ref.abs() * (1 + 2 * u) + count * U32 * size
    worst = (got - ref).abs() / bound.clamp(min=1e-37)
    assert float(worst.max()) <= 1, (what, float(worst.max()), int(worst.argmax()), float(ref[worst.argmax()]), float(got[worst.argmax()]))


@pytest.mark.parametrize("tokens", [1, 70])
@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_gelu_is_good_to_a_few_steps_of_its_value_far_out_too(dtype, tokens):
    """fp32: the complementary error function to 4 units, of an argument whose rounding is made up for; the product and the final sum: 8.
    bf16: the fitted form is off by 9 units, its reciprocal, polynomial and products by 15, and e^(-z^2 / 2) by the rounding of an exponent of 0.72 z^2:
    2.5 roundings times ln 2: 1.25 z^2."""
    dt = DTYPES[dtype]
    z = _values(-12.5, 12.5, 5001, dt)
    y, dz = _run(z, B.ACT_GELU, tokens)
    z = z.double()
    count = 8 + 0 * z if dt is torch.float32 else 24 + 1.25 * z * z
    cdf, bell = 0.5 * torch.special.erfc(-z / math.sqrt(2)), torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    _within(y, z * cdf, (z * cdf).abs(), count, dt, "gelu")
    _within(dz, cdf + z * bell, cdf + z.abs() * bell, count, dt, "slope")


@pytest.mark.parametrize("tokens", [1, 70])
@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_silu_is_good_to_a_few_steps_of_its_value_far_out_too(dtype, tokens):
    """fp32: an exponential to 2 units, three roundings and the product: 8.  bf16: the exponent 1.44 |z| is rounded, 1.3 |z| on top."""
    dt = DTYPES[dtype]
    z = _values(-80, 80, 5001, dt)
    y, dz = _run(z, B.ACT_SILU, tokens)
    z = z.double()
    count = 8 + 0 * z if dt is torch.float32 else 8 + 1.3 * z.abs()
    s, rest = torch.sigmoid(z), torch.sigmoid(-z)
    _within(y, z * s, (z * s).abs(), count, dt, "silu")
    _within(dz, s * (1 + z * rest), s * (1 + z.abs() * rest), count, dt, "slope")


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("T,n_in,out", [(3, 40, 72), (200, 136, 520), (130, 201, 263), (300, 4096, 520)])
def test_the_input_gradient_is_the_product_of_dz_as_it_is_stored(T, n_in, out, dtype):
    """The same bits from dz handed in as the gradient of a layer without an activation."""
    gen, dt = torch.Generator(device=DEV).manual_seed(T + out), DTYPES[dtype]
    W, dy, z = (torch.randn(*s, generator=gen, device=DEV).to(dt) for s in ((out, n_in), (T, out), (T, out)))
    dz, dx, again = torch.empty_like(dy), torch.empty(T, n_in, dtype=dt, device=DEV), torch.empty(T, n_in, dtype=dt, device=DEV)
    for act, g, d, to in ((B.ACT_GELU, dy, dz, dx), (B.ACT_NONE, dz, None, again)):
        layer = B.make_linear(None, W, activation=act, tokens=T)
        need = B.chunkft_linear_workspace_bytes(layer, backward=True)
        B.chunkft_linear_backward(layer, g, z, d, to, ws=torch.empty(need, dtype=torch.uint8, device=DEV))
    torch.cuda.synchronize()
    assert torch.equal(dx, again)
