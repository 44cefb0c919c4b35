"""fp32 cross attention against 64 bits as a whole, under the bounds of cross_precision.py, which test_cross_precision.py shows to tell lost blocks and lost bits."""
import numpy as np
import pytest
import torch

import cross_precision as cp
from paper_2408_04275_amd import binding as mm
from paper_2408_04275_amd.harness import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", list(cp.CASES))
def test_fp32_results_as_a_whole(name):
    nh, nkv, d, (cu, begin, end, Tk) = cp.CASES[name]
    x = cp.inputs(name)
    dev = {n: torch.from_numpy(a.reshape(len(a), -1)).to("cuda") for n, a in x.items()}
    out = {n: torch.full_like(dev[s], 7.0) for n, s in (("o", "q"), ("dq", "q"), ("dk", "k"), ("dv", "v"))}
    out["lse"] = torch.full((nh, int(cu[-1])), 7.0, device="cuda")
    desc, batch = mm.make_cross_attn_desc(mm.F32, nh, nkv, d), mm.CrossBatch.on_device(cu, begin, end, Tk)
    t = mm.make_cross_attn_tensors(dev["q"], dev["k"], dev["v"], out["o"], out["lse"])
    g = mm.make_cross_attn_grads(dev["do"], out["dq"], out["dk"], out["dv"])
    for back in (0, 1):
        n = mm.mmtrain_cross_attn_workspace_bytes(desc, batch, back)
        ws = torch.full((n,), 0xA5, dtype=torch.uint8, device="cuda")
        check(mm.mmtrain_cross_attn_bwd(desc, batch, t, g, ws, n) if back else mm.mmtrain_cross_attn_fwd(desc, batch, t, ws, n), "cross_attn")
        torch.cuda.synchronize()
    got = {n: a.cpu().numpy() for n, a in out.items()}
    got = {n: a if n == "lse" else a.reshape(len(a), -1, d) for n, a in got.items()}
    bound = cp.bounds(name, x)
    ref = dict(zip(("o", "lse"), cp.forward(name, x)))
    ref.update(cp.backward(name, x, got["o"], got["lse"]))
    far = {n: cp.too_far(got[n], ref[n], bound[n]) for n in bound}
    assert all(v <= 1 for v in far.values()), far
