"""switch_linear's activations value by value: unit matrices make the products exact, so that what is left is the
activation's own arithmetic.

Tolerances, relative to the value, in half steps of fp32 (2^-24).  Phi(-|u|) = t poly(t) exp(-u^2 / 2),
t = 1 / (1 + q |u|): t is off by 3 (q, the sum, the quotient), to which Phi answers with at most its power, 2.4 (at
u = 0); the polynomial by 3 and its fit by 1, two products by 2, the exponential by 4: 18, and 2 more for the products with u
and the linear part: 20.  In bf16 the exponential's argument is rounded like any other value: with |u| <= 12, 104 in powers of
two, off by three roundings, 3 * 104 * ln 2 * 2^-24 = 1.3e-5; with the 20 above 1.5e-5, less than a hundredth of bf16's
half step, which is added to it.  A derivative, Phi(u) + u phi(u), is off by so much of the magnitudes of its two terms.
"""
import math

import pytest
import torch

from paper_2101_03961_amd.layer import SwitchLinear
from test_operators_gpu import DEV, DT, U, U32, phi

pytestmark = pytest.mark.gpu

OWN = {"f32": 20 * U32, "bf16": 1.5e-5}
# few rows, tiles, and k in parts of either
SHAPES = [(48, 264), (300, 264), (48, 1032), (70, 1032)]


def points(M, N, dtype):
    """Pre-activations from -12 to 12, closer around zero and at the tails, and some far beyond."""
    n = M * N
    grid = torch.linspace(-12.0, 12.0, n, dtype=torch.float64)
    grid[::3] = grid[::3] ** 3 / 144.0
    grid[1::50] = 1e-30
    grid[:6] = torch.tensor([0.0, 100.0, -100.0, 1e20, -1e20, 3e38])
    return grid.reshape(M, N).to(DT[dtype])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,N", SHAPES)
@pytest.mark.parametrize("act", ["gelu", "geglu"])
def test_gelu_value_by_value(act, M, N, dtype):
    u = points(M, N, dtype)
    gen = torch.Generator().manual_seed(N)
    # linear parts that bring the tails' values back to the size of the others
    v = (torch.randn(M, N, generator=gen, dtype=torch.float64) * 2.0 ** torch.randint(0, 60, (M, N), generator=gen)).to(DT[dtype])
    v[:, :6] = 1.0
    z = torch.cat((u, v), 1) if act == "geglu" else u
    K = z.shape[1]
    unit = torch.eye(K, dtype=DT[dtype], device=DEV)
    op = SwitchLinear(M, K, N, act, 0.0, 0, dtype, DEV, train=True)
    y = op.forward(z.to(DEV), unit).cpu().double()
    assert torch.equal(op.z.cpu(), z)
    u64, v64 = u.double(), v.double() if act == "geglu" else torch.ones(1, dtype=torch.float64)
    cdf = phi(u64)
    half = 0.0 if dtype == "f32" else U[dtype]
    want = u64 * cdf * v64
    ok = ((y - want).abs() <= (half * (1 + OWN[dtype]) + OWN[dtype]) * want.abs())
    assert ok.all(), (u64[~ok][:4], y[~ok][:4], want[~ok][:4])
    # the gradient of z itself
    dy = torch.randn(M, N, generator=gen, dtype=torch.float64).to(DT[dtype])
    dx = op.backward(dy.to(DEV), z.to(DEV), unit)["dx"].cpu().double()
    g, pdf = dy.double(), torch.exp(-u64 * u64 / 2) / math.sqrt(2 * math.pi)
    own = OWN[dtype] + (2.0 ** -16 if dtype == "bf16" else 4 * U32)   # (dz in two terms; the products with dy and v)
    upd = torch.where(pdf > 0, u64 * pdf, 0.0)
    slope, size = cdf + upd, cdf + upd.abs()
    # (|dy| 3e38 is past the largest number from |dy| = 1.14 on: a row with an infinity has no products with zeros)
    fits = ((g * u64).abs() < torch.finfo(DT[dtype]).max).all(1)
    assert fits[1:].all()
    g, u64, dx, slope, size, cdf = (t[fits] for t in (g, u64, dx, slope, size, cdf))
    v64 = v64[fits] if act == "geglu" else v64
    ok = (dx[:, :N] - g * v64 * slope).abs() <= (g * v64).abs() * (half * slope.abs() + own * (1 + half) * size)
    assert ok.all(), (u64[~ok][:4], dx[:, :N][~ok][:4], (g * v64 * slope)[~ok][:4])
    if act == "geglu":
        want = g * u64 * cdf
        ok = (dx[:, N:] - want).abs() <= (half * (1 + own) + own) * want.abs()
        assert ok.all(), (u64[~ok][:4], dx[:, N:][~ok][:4], want[~ok][:4])
