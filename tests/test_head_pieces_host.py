"""How the backward pass of the losses at the output projection cuts the vocabulary into pieces: tests/native/head_pieces_host.cpp against the built library."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PACKAGE = os.path.join(ROOT, "paper_2601_22101_amd")


def test_pieces_of_the_vocabulary_cost_the_least(tmp_path):
    if not os.path.exists(os.path.join(PACKAGE, "libeco.so")):
        from paper_2601_22101_amd import build
        build.build()
    exe = str(tmp_path / "head_pieces_host")
    cmd = ["g++", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I", os.path.join(PACKAGE, "csrc"),
           os.path.join(ROOT, "tests", "native", "head_pieces_host.cpp"), "-L", PACKAGE, "-l:libeco.so", "-Wl,-rpath," + PACKAGE, "-Wl,--allow-shlib-undefined", "-o", exe]
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, r.stdout
    out = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=120,
                         env={**os.environ, "LD_LIBRARY_PATH": "/opt/rocm/lib:" + os.environ.get("LD_LIBRARY_PATH", "")})
    assert out.returncode == 0 and "pieces ok" in out.stdout, out.stdout
