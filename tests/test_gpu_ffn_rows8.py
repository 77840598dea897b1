"""The tests that make 8-bit rows, with the check that no code is NaN."""
import pytest

import ffn_checks
import test_gpu_ffn
from test_gpu_ffn import eco, harness, test_a_layers_half, test_fewer_rows_leave_the_others_alone, test_gated, test_norm      # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def finite_codes(monkeypatch):
    monkeypatch.setattr(test_gpu_ffn, "hold_rows8", ffn_checks.hold_rows8)
