"""test_lds_waits.py's check of LDS reads that are written as inline assembly, on the kernels of cross attention."""
import os
import subprocess

import pytest

from paper_2408_04275_amd.build import CSRC, FLAGS, HIPCC
from test_lds_waits import early_uses, functions


@pytest.mark.parametrize("source", ["cross_mfma.hip", "cross_mfma_bwd.hip"])
def test_no_register_is_touched_while_a_read_fills_it(source):
    r = subprocess.run([HIPCC, *FLAGS, "-S", "--cuda-device-only", os.path.join(CSRC, source), "-o", "-"], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    reads = 0
    for name, body in functions(r.stdout):
        reads += sum(inline and text.startswith("ds_read") for text, _, inline in body)
        assert early_uses(body) == {}, name
    assert reads > 0
