"""The calls of include/mmtrain_ops.h allocate nothing, on the host either: what they plan is on the stack, and a sort that asks for a buffer of its own
would be the allocation.  Shown on the host code of the files that they are made of, which may name no allocating function.  Needs the compiler, no GPU."""
import os
import re
import subprocess

import pytest

from paper_2408_04275_amd.build import CSRC, FLAGS, HIPCC

SOURCES = ["api_ops.hip", "rope.hip", "residual_norm.hip", "grad_norm.hip", "optimizer.hip", "embed.hip", "qk_norm.hip", "api_cross.hip", "cross_plan.hip", "cross_mfma.hip",
           "cross_mfma_bwd.hip", "cross_f32.hip"]


@pytest.mark.parametrize("source", SOURCES)
def test_host_code_names_no_allocation(source, tmp_path):
    obj = str(tmp_path / "host.o")
    r = subprocess.run([HIPCC, *FLAGS, "--offload-host-only", "-c", os.path.join(CSRC, source), "-o", obj], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    names = subprocess.run(["nm", "-u", obj], capture_output=True, text=True, check=True).stdout.split()
    assert "U" in names
    # operator new and delete in all their forms, and what they rest on
    assert [n for n in names if re.match(r"_Zn[wa]|_Zd[la]|(malloc|calloc|realloc|aligned_alloc|posix_memalign)$", n)] == []
