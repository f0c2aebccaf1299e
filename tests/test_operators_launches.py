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
