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
from test_operators_gpu import ACTS, DEV, DT, U, U32, phi

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


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,K,N", [(48, 72, 264), (300, 72, 264), (48, 1032, 1032), (70, 1032, 520)])
@pytest.mark.parametrize("act", ACTS)
def test_nan_and_infinity_of_pre_activations(act, M, K, N, dtype):
    """A value that is no number stays none through every activation, in y and in the gradients; beside its row and
    column the same bits as without it.  An infinite pre-activation has its limit."""
    gen = torch.Generator().manual_seed(M + N)
    cols = N * (2 if act == "geglu" else 1)
    normal = lambda *s: torch.randn(s, generator=gen).to(DT[dtype]).to(DEV)
    x, W, dy = normal(M, K), normal(K, cols) * K ** -0.5, normal(M, N)
    bias = torch.randn(cols, generator=gen).to(DEV)
    op = SwitchLinear(M, K, N, act, 0.0, 0, dtype, DEV, train=True)
    y = op.forward(x, W, bias).clone()
    grads = {k: t.clone() for k, t in op.backward(dy, x, W).items()}
    z = None if op.z is None else op.z.clone()
    r, c = M // 2, N // 3
    rows, at = torch.arange(M, device=DEV) != r, torch.arange(N, device=DEV) != c
    bad = x.clone()
    bad[r, 1] = float("nan")
    out = op.forward(bad, W, bias)
    assert torch.isnan(out[r]).all() and torch.equal(out[rows], y[rows])
    b = bias.clone()
    b[c] = float("nan")
    out = op.forward(x, W, b)
    assert torch.isnan(out[:, c]).all() and torch.equal(out[:, at], y[:, at])
    b[c] = float("inf")
    if act != "geglu":   # (there: infinity times a linear part)
        assert (op.forward(x, W, b)[:, c] == float("inf")).all()
    b[c] = -float("inf")
    if act in ("none", "relu"):
        assert (op.forward(x, W, b)[:, c] == (0.0 if act == "relu" else -float("inf"))).all()
    if act == "none":
        return
    op.z.copy_(z)
    op.z[r, c] = float("nan")
    got = op.backward(dy, x, W)
    assert torch.isnan(got["dx"][r]).all() and torch.equal(got["dx"][rows], grads["dx"][rows])
    assert torch.isnan(got["dW"][:, c]).all() and torch.isnan(got["db"][c])
    others = torch.arange(cols, device=DEV) % N != c
    assert torch.equal(got["dW"][:, others], grads["dW"][:, others]) and torch.equal(got["db"][others], grads["db"][others])
