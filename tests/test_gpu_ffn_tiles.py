"""The feed-forward products at the sizes of ffn_tiles: each of the large tiles, and workgroups that go through several of them, element by element and as a whole against float64."""
import pytest

from ffn_tiles import GATED, LINEAR
from ffn_util import DTYPE
from test_gpu_ffn import harness      # noqa: F401
from test_gpu_ffn_whole import check_gated, check_linear

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("case", [c[0] for c in LINEAR], ids=lambda c: "-".join(map(str, c)))
def test_linear(harness, case):      # noqa: F811
    check_linear(harness, *case[:6], out=DTYPE[case[6]])


@pytest.mark.parametrize("case", [c[0] for c in GATED], ids=lambda c: "-".join(map(str, c)))
def test_gated(harness, case):      # noqa: F811
    check_gated(harness, *case)
