"""Which kernels switch_linear launches, recorded without a GPU (linear_recorder.c stands in for the HIP runtime)."""
import os
import shutil
import subprocess

import pytest

import paper_2101_03961_amd as sw
from linear_sizes import LARGE_BACKWARD, LARGE_FORWARD

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.skipif(shutil.which("gcc") is None, reason="needs gcc")
ACTS = ("none", "relu", "gelu", "geglu")


@pytest.fixture(scope="module")
def record(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("launches") / "linear_recorder")
    # (launch_recorder.c's own main is not called)
    subprocess.run(["gcc", "-O1", "-Wall", "-Werror", "-Wno-unused-function", "-rdynamic", "-I", os.path.join(ROOT, "include"),
                    "-o", exe, os.path.join(ROOT, "tests", "linear_recorder.c"), "-ldl"], check=True)

    def call(what, M, K, N, act="none", dropout=0.0, dtype=sw.SW_BF16, flags=0):
        """(status, workspace bytes, [(kernel, grid)]) of a call with every tensor it can have."""
        line = "%s %d %d %d %d %d %r %d\n" % (what, M, K, N, dtype, ACTS.index(act), dropout, flags)
        out = subprocess.run([exe, sw.library_path()], input=line, capture_output=True, text=True, check=True).stdout
        words = [row.split() for row in out.splitlines()]
        (_, status, size), = [w for w in words if w[0] == "call"]
        return int(status), int(size), [(w[1], tuple(int(v) for v in w[2:5])) for w in words if w[0] == "launch"]
    return call


def names(launches):
    """The kernels' names without what the compiler put around them."""
    return [next(part for part in ("linear_few", "linear_fwd_large", "linear_fwd_small", "linear_fwd_f32", "linear_finish",
                                   "linear_dz", "linear_bwd_large", "linear_bwd_small", "linear_bwd_f32", "linear_join")
                 if part in kernel) for kernel, _ in launches]


@pytest.mark.parametrize("M,K,N,act,dropout,parts", LARGE_FORWARD)
def test_large_tiles_forward(record, M, K, N, act, dropout, parts):
    status, _, launches = record("forward", M, K, N, act, dropout)
    assert status == 0 and names(launches) == ["linear_fwd_large"] + ["linear_finish"] * parts


@pytest.mark.parametrize("M,K,N,act,dropout,dx_parts,dW_parts", LARGE_BACKWARD)
def test_large_tiles_backward(record, M, K, N, act, dropout, dx_parts, dW_parts):
    status, _, launches = record("backward", M, K, N, act, dropout)
    assert status == 0 and names(launches) == ["linear_dz", "linear_bwd_large", "linear_join"]
    # the join's blocks: 32 columns of db each, 8192 elements of a gradient that was summed in parts
    cols = N * (2 if act == "geglu" else 1)
    blocks = -(-cols // 32) + dx_parts * -(-M * K // 8192) + dW_parts * -(-K * cols // 8192)
    assert launches[-1][1] == (blocks, 1, 1)


@pytest.mark.parametrize("act", ACTS)
def test_two_terms_of_dz_on_request(record, act):
    """Twice the rows in dx's products and twice the k in dW's, for GELU in bf16 only; other flags are refused."""
    assert sw.SW_FLAG_DZ_TWO_TERMS == 2
    M, K, N = 8192, 4096, 1024
    one, two = (record("backward", M, K, N, act, flags=flags) for flags in (0, sw.SW_FLAG_DZ_TWO_TERMS))
    assert one[0] == two[0] == 0
    gelu = act in ("gelu", "geglu")
    assert (two == one) == (not gelu)
    if gelu:   # both terms' sums of dx, at least
        assert two[1] >= one[1] + 2 * M * K * 4
    assert record("backward", M, K, N, act, dtype=sw.SW_F32, flags=2) == record("backward", M, K, N, act, dtype=sw.SW_F32)
    assert record("forward", M, K, N, act, flags=2) == record("forward", M, K, N, act)
    for flags in (1, 3, 4, -1):
        for what in ("forward", "backward"):
            assert record(what, M, K, N, act, flags=flags)[0] == -3
    # few rows have them anyway
    assert record("backward", 256, K, N, act, flags=2) == record("backward", 256, K, N, act)


@pytest.mark.parametrize("act", ["none", "geglu"])
@pytest.mark.parametrize("M,K,N,dtype", [(16, 8192, 256, sw.SW_BF16), (16, 8192, 256, sw.SW_F32), (100, 4096, 256, sw.SW_BF16)])
def test_forward_refuses_a_workspace_that_is_too_small(record, M, K, N, dtype, act):
    """Forward passes in parts of k need one: never followed, too small, none, and not on 256 bytes."""
    at = 0x1000
    status, need, launches = record("forward", M, K, N, act, dtype=dtype)
    assert status == 0 and need > 0 and names(launches)[1:] == ["linear_finish"]
    cfg = sw.SwitchLinearConfig(M, K, N, dtype, ACTS.index(act), 0.0, 0, 0)
    assert sw.switch_linear_workspace_size(cfg, False) == need
    for ws, size in ((at, need - 1), (at, 0), (None, need), (at + 16, need)):
        assert sw.switch_linear(cfg, at, at, None, None, at, None, ws, size, check=False) == -5
