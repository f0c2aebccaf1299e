"""switch_linear's 256 x 256 tiles against the definition in 64 bits, evaluated on the device.

Tolerances as in test_operators_gpu.py: half a step of bf16 (2^-8 of the value) where an output is stored; a sum of n
products in fp32 is off by at most (n + 2) 2^-24 of the sum of their magnitudes, its norm by (sqrt(n) + 16) 2^-24; dz
of GELU, rounded to bf16 for the products, makes each of them off by another 2^-8.
"""
import math

import pytest
import torch

import paper_2101_03961_amd as sw
from linear_sizes import LARGE_BACKWARD, LARGE_FORWARD
from test_operators_gpu import DEV, U, U32, act64, dz64, keep_factor

from paper_2101_03961_amd.layer import SwitchLinear

pytestmark = pytest.mark.gpu
u = U["bf16"]


def operand(gen, *size):
    return torch.randn(size, generator=gen, device=DEV)


def close(name, got, want, bound, norm):
    got = got.double()
    assert torch.isfinite(got).all(), name
    err = (got - want).abs()
    assert (err <= bound).all(), (name, float((err - bound).max()))
    total = float(torch.linalg.norm(err) / torch.linalg.norm(want))
    assert total <= norm, (name, total, norm)


@pytest.mark.parametrize("M,K,N,act,rate,parts", LARGE_FORWARD)
def test_large_tiles_forward(M, K, N, act, rate, parts):
    gen = torch.Generator(device=DEV).manual_seed(M + K)
    cols, seed = N * (2 if act == "geglu" else 1), 0x1234567800000000 + M
    x, W = operand(gen, M, K).bfloat16(), operand(gen, K, cols).mul_(K ** -0.5).bfloat16()
    bias, residual = operand(gen, cols), operand(gen, M, N).bfloat16()
    z = x.double() @ W.double() + bias.double()
    ez = (K + 2) * U32 * (x.double().abs() @ W.double().abs() + bias.double().abs())
    want = act64(act, z)
    ea = ez
    if act == "geglu":
        zu, zv = z.chunk(2, dim=1)
        eu, ev = ez.chunk(2, dim=1)
        ea = zv.abs() * (1.13 * eu + 4e-7 * zu.abs()) + zu.abs() * ev + 1.13 * eu * ev
    elif act == "gelu":
        ea = 1.13 * ez + 4e-7 * z.abs()
    factor = keep_factor(M * N, rate, seed).reshape(M, N).to(DEV)
    want, ea = want * factor, (ea + 4 * U32 * want.abs()) * factor
    norm = (math.sqrt(K) + 16) * U32 + u
    cfg = sw.SwitchLinearConfig(M, K, N, sw.SW_BF16, ("none", "relu", "gelu", "geglu").index(act), rate, 0, seed)
    size = sw.switch_linear_workspace_size(cfg, False)
    ws = torch.full((max(size, 1),), 255, dtype=torch.uint8, device=DEV)
    # outputs inside larger buffers: the rows around them stay as they were
    y, zs = (torch.full((M + 600, n), 3.0, dtype=torch.bfloat16, device=DEV) for n in (N, cols))
    stream = torch.cuda.current_stream().cuda_stream
    sw.switch_linear(cfg, x, W, bias, residual, y[300:300 + M], zs[300:300 + M], ws, size, stream)
    total, et = want + residual.double(), ea + U32 * (want.abs() + residual.double().abs())
    close("y", y[300:300 + M], total, u * (total.abs() + et) + et, norm)
    close("z", zs[300:300 + M], z, u * (z.abs() + ez) + ez, norm)
    for t in (y, zs):
        assert (t[:300] == 3.0).all() and (t[300 + M:] == 3.0).all()
    # without bias, residual and z
    z = z - bias.double()
    want = act64(act, z) * factor
    if act == "geglu":
        zu, zv = z.chunk(2, dim=1)
        ea = (zv.abs() * (1.13 * eu + 4e-7 * zu.abs()) + zu.abs() * ev + 1.13 * eu * ev + 4 * U32 * want.abs()) * factor
    elif act == "gelu":
        ea = (1.13 * ez + 4e-7 * z.abs() + 4 * U32 * want.abs()) * factor
    y.fill_(float("nan"))
    sw.switch_linear(cfg, x, W, None, None, y[:M], None, ws, size, stream)
    close("y", y[:M], want, u * (want.abs() + ea) + ea, norm)


@pytest.mark.parametrize("M,K,N,act,rate,dx_parts,dW_parts", LARGE_BACKWARD)
def test_large_tiles_backward(M, K, N, act, rate, dx_parts, dW_parts):
    gen = torch.Generator(device=DEV).manual_seed(M + K)
    cols, seed = N * (2 if act == "geglu" else 1), 0x8765432100000000 + M
    x, W = operand(gen, M, K).bfloat16(), operand(gen, K, cols).mul_(K ** -0.5).bfloat16()
    dy, z = operand(gen, M, N).bfloat16(), operand(gen, M, cols).bfloat16()
    op = SwitchLinear(M, K, N, act, rate, seed, "bf16", DEV, train=True)
    if act != "none":
        op.z.copy_(z)
    op.workspace.fill_(255)
    big = {k: torch.full((r + 600, c), 3.0, dtype=torch.bfloat16, device=DEV) for k, r, c in (("dx", M, K), ("dW", K, cols))}
    op.dx, op.dW = big["dx"][300:300 + M], big["dW"][300:300 + K]
    op.db.fill_(float("nan"))
    got = op.backward(dy, x, W)
    g = dy.double() * keep_factor(M * N, rate, seed).reshape(M, N).to(DEV)
    dz = dz64(act, z.double(), g)
    edz = dz.abs() * 8 * U32
    rounded = 0.0
    if act in ("gelu", "geglu"):
        rounded = u
        lin = g if act == "gelu" else torch.cat((g * z.double().chunk(2, 1)[1], g * z.double().chunk(2, 1)[0]), 1)
        edz = edz + 4e-7 * lin.abs() * (1 + z.double().abs())
    close("db", got["db"], dz.sum(0), edz.sum(0) + (M + 2) * U32 * dz.abs().sum(0),
          (math.sqrt(M) + 16) * U32 * max(1.0, float(torch.linalg.norm(dz) / torch.linalg.norm(dz.sum(0)))))
    ep = edz + rounded * dz.abs()
    for name, a, b, e, n in (("dx", dz, W.double().t().contiguous(), ep @ W.double().abs().t().contiguous(), cols),
                             ("dW", x.double().t().contiguous(), dz, x.double().abs().t().contiguous() @ ep, M)):
        want = a @ b
        e = e + (n + 2) * U32 * (a.abs() @ b.abs())
        close(name, got[name], want, u * (want.abs() + e) + e, (math.sqrt(n) + 16) * U32 + u + rounded)
        assert (big[name][:300] == 3.0).all() and (big[name][300 + got[name].shape[0]:] == 3.0).all(), name


@pytest.mark.parametrize("act", ["gelu", "geglu"])
@pytest.mark.parametrize("M,K,N", [(257, 264, 136), (1000, 72, 520), (2823, 2984, 728), (8929, 744, 512)])
def test_two_terms_of_dz_on_request(M, K, N, act):
    """dz in two bf16 terms is off by 2^-16 (the second, at most 2^-8 of dz, is rounded to 2^-8 of itself): the gradients
    are off by their own rounding.  In small and in large tiles."""
    gen = torch.Generator(device=DEV).manual_seed(M)
    cols, seed = N * (2 if act == "geglu" else 1), M
    x, W = operand(gen, M, K).bfloat16(), operand(gen, K, cols).mul_(K ** -0.5).bfloat16()
    dy, z = operand(gen, M, N).bfloat16(), operand(gen, M, cols).bfloat16()
    op = SwitchLinear(M, K, N, act, 0.1, seed, "bf16", DEV, train=True, dz_two_terms=True)
    op.z.copy_(z)
    op.workspace.fill_(255)
    for t in (op.dx, op.dW, op.db):
        t.fill_(float("nan"))
    got = op.backward(dy, x, W)
    g = dy.double() * keep_factor(M * N, 0.1, seed).reshape(M, N).to(DEV)
    dz = dz64(act, z.double(), g)
    lin = g if act == "gelu" else torch.cat((g * z.double().chunk(2, 1)[1], g * z.double().chunk(2, 1)[0]), 1)
    edz = dz.abs() * (2.0 ** -16 + 8 * U32) + 4e-7 * lin.abs() * (1 + z.double().abs())
    for name, a, b, e, n in (("dx", dz, W.double().t().contiguous(), edz @ W.double().abs().t().contiguous(), 2 * cols),
                             ("dW", x.double().t().contiguous(), dz, x.double().abs().t().contiguous() @ edz, 2 * M)):
        want = a @ b
        e = e + (n + 2) * U32 * (a.abs() @ b.abs())
        close(name, got[name], want, u * (want.abs() + e) + e, (math.sqrt(n) + 16) * U32 + u + 2.0 ** -15)
        # an evenly distributed rounding, 2^-8 / sqrt(3) of the bottom of a value's binade, is 0.426 of 2^-8 in the norm of normally
        # distributed values of any variance (one term's and the gradient's own together: sqrt(2) times that)
        rms = float(torch.linalg.norm(got[name].double() - want) / torch.linalg.norm(want))
        assert rms <= 0.45 * u, (name, rms)
    dx, dW, db = (t.clone() for t in (got["dx"], got["dW"], got["db"]))
    one = SwitchLinear(M, K, N, act, 0.1, seed, "bf16", DEV, train=True)
    one.z.copy_(z)
    assert torch.equal(one.backward(dy, x, W)["db"], db)
    assert not torch.equal(one.dx, dx) and not torch.equal(one.dW, dW)
