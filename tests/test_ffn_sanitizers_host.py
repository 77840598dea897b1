"""The host side of the feed-forward calls (csrc_ffn/eco_ffn_api.cpp) under the address and undefined-behaviour sanitizers; plans and launchers are the built library's."""
import os
import subprocess

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PACKAGE = os.path.join(ROOT, "paper_2601_22101_amd")
SAN = ["-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all"]


def test_feed_forward_calls_under_asan_and_ubsan(tmp_path):
    if torch.cuda.is_available():
        pytest.skip("the pointers are none")
    if not os.path.exists(os.path.join(PACKAGE, "libeco.so")):
        from paper_2601_22101_amd import build
        build.build()
    run = lambda cmd, **kw: subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=300, **kw)      # noqa: E731
    client, exe = str(tmp_path / "client.o"), str(tmp_path / "abi_ffn_san")
    r = run(["gcc", "-std=c99", "-Wall", "-Wextra", "-Werror", *SAN, "-I", os.path.join(ROOT, "include"), "-c", os.path.join(ROOT, "tests", "native", "abi_ffn_san.c"), "-o", client])
    assert r.returncode == 0, r.stdout
    r = run(["g++", "-std=c++17", *SAN, "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", os.path.join(PACKAGE, "csrc_ffn", "eco_ffn_api.cpp"), client, "-L", PACKAGE, "-l:libeco.so",
             "-Wl,-rpath," + PACKAGE, "-L/opt/rocm/lib", "-lamdhip64", "-Wl,-rpath,/opt/rocm/lib", "-o", exe])
    assert r.returncode == 0, r.stdout[-3000:]
    r = run([exe], env={**os.environ, "ASAN_OPTIONS": "detect_leaks=0:abort_on_error=0:halt_on_error=1"})      # (leaks at exit are the HIP runtime's)
    assert r.returncode == 0 and r.stdout.strip().endswith("ok"), r.stdout[-3000:]
    assert "runtime error" not in r.stdout and "AddressSanitizer" not in r.stdout
