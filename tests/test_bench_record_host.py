"""The committed record of the step's HBM traffic is one of the step's present sources, so that bench.py reports it."""
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)

import bench          # noqa: E402


def test_the_committed_traffic_is_of_the_trees_sources():
    value, source = bench.profiled_traffic("cfg4_smoe_2p1b_shaped")
    assert value is not None and bench.kernel_source_hash() in source, source


def test_only_the_step_and_the_losses_lie_beside_the_step():
    """What else is in its folder would make a change to another operator look like one to the step."""
    names = os.listdir(os.path.join(ROOT, "paper_2601_22101_amd", "csrc"))
    step = ("eco_api.cpp", "eco_device.hpp", "eco_internal.hpp", "eco_kernels_misc.hip")
    assert all(n in step or n.startswith(("eco_step_", "eco_head")) for n in names), names
