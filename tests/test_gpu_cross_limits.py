"""Cross attention at the ends of the sizes that its documentation names.  Tolerances as in test_gpu_attention_ops.py: each result is off by its rounding to bf16
and by the roundings to bf16 of the probabilities and their gradients, half a step of the sum of the absolute values of the terms they stand in.  A score of 16
products is off by at most 24 2^-24 of the sum of their absolute values, and so a log-sum-exp; a probability, which takes both, by twice that: below 2^-18 of it."""
import numpy as np
import pytest
import torch

from paper_2408_04275_amd import binding as mm
from paper_2408_04275_amd.harness import check

pytestmark = pytest.mark.gpu
HALF = 2.0 ** -8


def test_more_than_two_to_the_27_query_tokens():
    Tq, Tk, d = (1 << 27) + 70, 9, 16
    gen = torch.Generator(device="cuda").manual_seed(1)
    q = torch.empty((Tq, d), dtype=torch.bfloat16, device="cuda")
    for a in range(0, Tq, 1 << 24):
        q[a:a + (1 << 24)] = torch.randn((min(1 << 24, Tq - a), d), generator=gen, device="cuda").to(torch.bfloat16)
    k, v = (torch.randn((Tk, d), generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2))
    ends = [slice(0, 1000), slice(Tq - 1000, Tq)]
    do = torch.zeros_like(q)
    for part in ends:                                  # rows in between have no gradient: dK and dV are sums over the two ends
        do[part] = torch.randn((1000, d), generator=gen, device="cuda").to(torch.bfloat16)
    o, dq = torch.full_like(q, 7.0), torch.full_like(q, 7.0)
    dk, dv = torch.full_like(k, 7.0), torch.full_like(k, 7.0)
    lse = torch.full((1, Tq), 7.0, device="cuda")
    desc = mm.make_cross_attn_desc(mm.BF16, 1, 1, d)
    batch = mm.CrossBatch.on_device(np.array([0, Tq]), np.array([0]), np.array([Tk]), Tk)
    t, g = mm.make_cross_attn_tensors(q, k, v, o, lse), mm.make_cross_attn_grads(do, dq, dk, dv)
    for back in (0, 1):
        n = mm.mmtrain_cross_attn_workspace_bytes(desc, batch, back)
        ws = torch.full((n,), 0xA5, dtype=torch.uint8, device="cuda")
        check(mm.mmtrain_cross_attn_bwd(desc, batch, t, g, ws, n) if back else mm.mmtrain_cross_attn_fwd(desc, batch, t, ws, n), "cross_attn")
        torch.cuda.synchronize()
    kk, vv = k.double(), v.double()
    for a in range(0, Tq, 1 << 23):                    # forward: every row
        rows = slice(a, min(a + (1 << 23), Tq))
        qq = q[rows].double()
        s, slack = qq @ kk.t() / 4.0, 2.0 ** -18 * (1 + (qq.abs() @ kk.abs().t() / 4.0).amax(1, keepdim=True))
        p = torch.softmax(s, 1)
        ref, mag = p @ vv, p @ vv.abs()
        assert torch.all((o[rows].double() - ref).abs() <= HALF * (ref.abs() + mag) + slack * mag)
        assert torch.all((lse[0, rows].double() - torch.logsumexp(s, 1)).abs() <= slack[:, 0])
    assert not torch.any(dq[1000:Tq - 1000])
    sums = {n: torch.zeros((Tk, d), dtype=torch.float64, device="cuda") for n in ("dk", "dv", "mk", "mv")}
    for rows in ends:
        qq, dd = q[rows].double(), do[rows].double()
        p = torch.exp(qq @ kk.t() / 4.0 - lse[0, rows].double()[:, None])
        ds = p * (dd @ vv.t() - (dd * o[rows].double()).sum(1, keepdim=True))
        slack = 2.0 ** -18 * (1 + (qq.abs() @ kk.abs().t() / 4.0).amax(1, keepdim=True))
        mp = p * (HALF + slack)                        # what a probability, and its gradient, may be off by
        mds = ds.abs() * (HALF + slack) + p * 2.0 ** -18 * (dd.abs() @ vv.abs().t() + (dd.abs() * o[rows].double().abs()).sum(1, keepdim=True))
        ref = ds @ kk / 4.0
        assert torch.all((dq[rows].double() - ref).abs() <= HALF * ref.abs() + mds @ kk.abs() / 4.0)
        sums["dk"] += ds.t() @ qq / 4.0
        sums["mk"] += mds.t() @ qq.abs() / 4.0
        sums["dv"] += p.t() @ dd
        sums["mv"] += mp.t() @ dd.abs()
    for got, name in ((dk, "k"), (dv, "v")):
        ref, mag = sums["d" + name], sums["m" + name]
        # (sums of 2000 rows: their additions take at most 2^-13 of the terms, a 32nd of what their roundings may take)
        assert torch.all((got.double() - ref).abs() <= HALF * ref.abs() + 1.04 * mag), name
