"""Forward tiles of 256 rows, which long walks of heads wider than 64 features take: each width that has a form of its own, walks that end inside a block of 32
keys, on one, and on a step of 64.  Tolerances as in test_gpu_attention_ops.py."""
import pytest

from paper_2408_04275_amd import binding as mm
from test_gpu_attention_ops import Cross, runs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [80, 96, 112, 128])
@pytest.mark.parametrize("keys", [4201, 4224, 4256])
def test_tiles_of_256_rows(d, keys):
    # 38 tiles of 128 rows for each of four key/value heads, and one that a run of a single token leaves nearly empty
    Cross(mm.BF16, 64, 4, d, runs([300, 1], [keys, 33]), seed=d + keys).verify(back=False)
