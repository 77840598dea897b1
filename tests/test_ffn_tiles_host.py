"""The plans of the sizes in ffn_tiles, by tests/native/ffn_plan_host.cpp against the built library: a change of what tiles cost that takes one of them out of the GPU tests is seen."""
import os
import subprocess

import pytest

from ffn_tiles import GATED, GRADIENTS, LINEAR
from ffn_util import FMT

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PACKAGE = os.path.join(ROOT, "paper_2601_22101_amd")


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    if not os.path.exists(os.path.join(PACKAGE, "libeco.so")):
        from paper_2601_22101_amd import build
        build.build()
    exe = str(tmp_path_factory.mktemp("plan") / "ffn_plan_host")
    cmd = ["g++", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I", os.path.join(PACKAGE, "csrc_ffn"),
           os.path.join(ROOT, "tests", "native", "ffn_plan_host.cpp"), "-L", PACKAGE, "-l:libeco.so", "-Wl,-rpath," + PACKAGE, "-Wl,--allow-shlib-undefined", "-o", exe]
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, r.stdout

    def run(*args):
        out = subprocess.run([exe, *map(str, args)], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=60,
                             env={**os.environ, "LD_LIBRARY_PATH": "/opt/rocm/lib:" + os.environ.get("LD_LIBRARY_PATH", "")})
        assert out.returncode == 0, out.stdout
        return [int(n) for n in out.stdout.split()]
    return run


@pytest.mark.parametrize("case,tile,round_full,split", LINEAR)
def test_linear(plans, case, tile, round_full, split):
    rows, in_dim, out_dim, group, fmt, _, out = case
    got = plans("forward", 0, rows, in_dim, out_dim, group, FMT[fmt], int(out == "fp32"))
    assert (got[0], got[1]) == tile and (got[2] >= 256) == round_full and (got[4] > 1) == split, got


@pytest.mark.parametrize("end", [1, 2])
@pytest.mark.parametrize("case,tile,round_full,split", GATED)
def test_gated(plans, case, tile, round_full, split, end):
    rows, in_dim, width, group, fmt, _, _ = case
    got = plans("forward", end, rows, in_dim, width, group, FMT[fmt], 0)
    assert (got[0], got[1]) == tile and (got[2] >= 256) == round_full and (got[4] > 1) == split, got


@pytest.mark.parametrize("case,shape,input_split,weights_split", GRADIENTS)
def test_gradients(plans, case, shape, input_split, weights_split):
    got = plans("gradients", *case)
    assert got[0] == shape and (got[3] > 1) == input_split and (got[5] > 1) == weights_split, got
    of = [(1, *c[0][:3]) for c in LINEAR] + [(2, *c[0][:3]) for c in GATED]
    assert case in of
