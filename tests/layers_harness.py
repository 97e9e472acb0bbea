"""Shared plumbing of the tests of the layer and update operators: tensors at odd places inside buffers whose other elements are
watched, 64-bit definitions, and the comparison rule.  Not a test module itself.

Comparison rule, element by element: |got - ref| <= u |ref| + c 2^-24 S.  u is half a step of the result's type (one rounding),
S the sum of the magnitudes of the terms that the fp32 arithmetic adds up to the element, c their number plus a few for the
functions in between: the standard bound on a sum of c fp32 terms in any order.
"""

import math

import torch

DEV = "cuda:0"
CANARY = -77.0
U32 = 2.0 ** -24
ACTS = ("none", "relu", "gelu", "silu")


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


class Placed:
    """A copy of `t` on the device as rows of a wider buffer that starts `lead` elements into its allocation."""

    def __init__(self, t, dtype=None, pad=0, lead=0, device=DEV):
        dtype = dtype or t.dtype
        rows, cols = (1, t.shape[0]) if t.dim() == 1 else t.shape
        self.ld = cols + pad
        self.raw = torch.full((lead + rows * self.ld + 16,), CANARY, dtype=dtype, device=device)
        grid = self.raw[lead:lead + rows * self.ld].view(rows, self.ld)
        self.mask = torch.ones_like(self.raw, dtype=torch.bool)
        self.mask[lead:lead + rows * self.ld].view(rows, self.ld)[:, :cols] = False
        self.t = grid[:, :cols] if t.dim() == 2 else grid[0, :cols]
        self.t.copy_(t)

    def untouched(self):
        return bool((self.raw[self.mask] == CANARY).all())


def assert_close(got, ref, sums, count, what):
    """ref, sums: float64 on the CPU; got: the device's result."""
    dtype = got.dtype
    g = got.detach().cpu().double()
    bound = half_step(dtype) * ref.abs() * (1 + 2 * half_step(dtype)) + count * U32 * sums + 1e-37
    bad = ~((g - ref).abs() <= bound)
    assert not bad.any(), (what, int(bad.sum()), float((g - ref).abs().max()), float((((g - ref).abs()) / bound).max()))


def act64(z, act):
    if act == "relu":
        return z.clamp(min=0)
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z / math.sqrt(2)))
    return z * torch.sigmoid(z) if act == "silu" else z


def slope64(z, act):
    if act == "relu":
        return (z > 0).double()
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z / math.sqrt(2))) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if act == "silu":
        s = torch.sigmoid(z)
        return s + z * s * (1 - s)
    return torch.ones_like(z)


# ------------------------------------------------------------------ Newton-Schulz in 64 bits
A_, B_, C_ = 3.4445, -4.7750, 2.0315
# |f'| <= 3.96 and f(x) / x <= 3.4445 on [0, 1.2023], the interval that f = a x + b x^3 + c x^5 maps into itself: a perturbation of X
# grows by at most this much in the Frobenius norm in a step (divided differences of an odd function of singular values).
GROWTH = 3.96


def newton_schulz64(u, steps, eps):
    tall = u.shape[0] > u.shape[1]
    x = u.t() if tall else u
    x = x / (torch.linalg.matrix_norm(x) + eps)
    for _ in range(steps):
        a = x @ x.t()
        x = A_ * x + (B_ * a + C_ * a @ a) @ x
    return x.t() if tall else x


def newton_schulz_bound(u, steps, eps, digits, exact_start):
    """How far (Frobenius) results may be off to first order, from what each step rounds to `digits` digits (half a step
    2^-digits): X, A = X X^T and the polynomial P, and from the fp32 sums of k terms (k 2^-24 of the products of norms);
    every later step lets it grow by GROWTH."""
    unit = 2.0 ** -digits
    norm = torch.linalg.matrix_norm
    x = (u.t() if u.shape[0] > u.shape[1] else u)
    x = x / (norm(x) + eps)
    err = 0.0 if exact_start else unit * float(norm(x))
    r, c = x.shape
    for _ in range(steps):
        a = x @ x.t()
        p = B_ * a + C_ * a @ a + A_ * torch.eye(r, dtype=torch.float64)
        two, fro_x = float(torch.linalg.matrix_norm(x, 2)), float(norm(x))
        da = unit * float(norm(a)) + c * U32 * fro_x ** 2
        dp = unit * float(norm(p)) + (abs(B_) + 2 * C_ * two ** 2) * da + r * U32 * C_ * float(norm(a)) ** 2
        nx = p @ x
        err = GROWTH * err + dp * two + unit * float(norm(nx)) + r * U32 * float(norm(p)) * fro_x
        x = nx
    return err
