"""bench.py replays a profile's traffic of the step only on the sources that it was taken on: the step's own, not those of the losses beside it."""
import os
import shutil
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)

import bench          # noqa: E402


def test_the_hash_is_of_the_steps_sources(tmp_path, monkeypatch):
    csrc = tmp_path / "paper_2601_22101_amd" / "csrc"
    shutil.copytree(os.path.join(ROOT, "paper_2601_22101_amd", "csrc"), csrc)
    here = bench.kernel_source_hash()
    monkeypatch.setattr(bench, "ROOT", str(tmp_path))
    assert bench.kernel_source_hash() == here
    for name in sorted(os.listdir(csrc)):
        before = (csrc / name).read_bytes()
        (csrc / name).write_bytes(before + b"\n")
        assert (bench.kernel_source_hash() == here) == name.startswith("eco_head"), name
        (csrc / name).write_bytes(before)
    (csrc / "eco_head_more.hip").write_text("// another kernel of the losses\n")
    assert bench.kernel_source_hash() == here
