"""Embedding, norms of heads and cross attention at the ends of what their documentation allows: strides, heads, runs and widths, first calls that are captured.
Tolerances as in test_gpu_attention_ops.py."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from paper_2408_04275_amd import binding as mm
from paper_2408_04275_amd.harness import check, torch_dtype
from test_gpu_attention_ops import DTYPES, Cross, embed_case, qk_case, runs

pytestmark = pytest.mark.gpu


def wide_rows(c, ld):
    """c's tensors as columns of rows ld elements apart."""
    of = lambda rows: torch.zeros((rows, ld), dtype=torch_dtype(c.dtype), device="cuda")  # noqa: E731
    nq, nk = c.nh * c.d, c.nkv * c.d
    queries, keys = of(c.Tq), of(c.Tk)
    col = lambda t, i, n: t[:, i * 4096:i * 4096 + n]  # noqa: E731
    q, do, o, dq = (col(queries, i, nq) for i in range(4))
    k, v, dk, dv = (col(keys, i, nk) for i in range(4))
    q.copy_(c.q), do.copy_(c.do), k.copy_(c.k), v.copy_(c.v)
    c.q, c.do, c.k, c.v = q, do, k, v
    c.out = {"o": o, "dq": dq, "dk": dk, "dv": dv}


@DTYPES
@pytest.mark.parametrize("lq,lk", [([70, 3], [100, 66]), ([1, 1], [40, 130]), ([4, 9], [900, 60])])
def test_cross_rows_as_far_apart_as_they_may_be(dtype, lq, lk):
    """Rows just below 2^24 elements apart give what rows beside each other give."""
    ld = (1 << 24) - (8 if dtype == mm.BF16 else 4)
    for nh, nkv in ((2, 2), (6, 2)):
        c = Cross(dtype, nh, nkv, 64 if dtype == mm.BF16 else 48, runs(lq, lk), seed=len(lq) + lq[0])
        c.fwd(), c.bwd()
        want, lse = {n: t.clone() for n, t in c.out.items()}, c.lse.clone()
        wide_rows(c, ld)
        c.fwd(), c.bwd()
        torch.cuda.synchronize()
        assert torch.equal(c.lse, lse) and all(torch.equal(t, want[n]) for n, t in c.out.items())


@DTYPES
@pytest.mark.parametrize("nh,nkv", [(4096, 1), (4096, 4096), (4095, 3)])
def test_cross_as_many_heads_as_there_may_be(dtype, nh, nkv):
    Cross(dtype, nh, nkv, 16, runs([2, 1], [70, 3]), seed=nkv).verify()


@DTYPES
def test_cross_as_many_runs_as_there_may_be(dtype):
    """Runs of up to two tokens that see up to three keys of their own; every fifth sees none."""
    S = 65536
    rng = np.random.default_rng(50)
    lk = rng.integers(0, 4, S) * (np.arange(S) % 5 > 0)
    Cross(dtype, 1, 1, 16, runs(rng.integers(0, 3, S), lk, tail=1), seed=51).verify()


def test_embed_as_wide_as_it_may_be():
    for dtype in (mm.BF16, mm.F32):
        embed_case(dtype, 40, 65536, 20, 7, seed=52)
        embed_case(dtype, 40, 65536, 20, 7, main=True, accumulate=True, seed=53)


@DTYPES
def test_qk_norm_as_many_heads_as_there_may_be(dtype):
    qk_case(dtype, 65535, 1, 8, 8, "half", "layer", T=3, positions=[0, 5, 131071], main=True, seed=54)
    qk_case(dtype, 1, 65535, 16, 8, "interleaved", "rms", T=2, positions=[7, -3], seed=55)


@pytest.mark.parametrize("lq,lk", [([1] * 90, [300] * 90), ([1] * 5, [4000] * 5), ([40] * 70, [50] * 70)])
def test_cross_with_tables_and_chunks_in_a_graph(lq, lk):
    """Replayed with other tensors in the same places, eager calls with workspaces of their own in between."""
    c = Cross(mm.BF16, 4, 2, 64, runs(lq, lk), seed=56)
    space = {back: torch.full((mm.mmtrain_cross_attn_workspace_bytes(c.desc, c.batch, back),), 0xA5, dtype=torch.uint8, device="cuda") for back in (0, 1)}
    t = mm.make_cross_attn_tensors(c.q, c.k, c.v, c.out["o"], c.lse)
    g = mm.make_cross_attn_grads(c.do, c.out["dq"], c.out["dk"], c.out["dv"])
    c.fwd(), c.bwd()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        check(mm.mmtrain_cross_attn_fwd(c.desc, c.batch, t, space[0], space[0].numel()), "fwd")
        check(mm.mmtrain_cross_attn_bwd(c.desc, c.batch, t, g, space[1], space[1].numel()), "bwd")
    gen = torch.Generator(device="cuda").manual_seed(57)
    for i in range(4):
        for x in (c.q, c.k, c.v, c.do):
            x.copy_(torch.randn(x.shape, generator=gen, device="cuda"))
        c.fwd(), c.bwd()
        torch.cuda.synchronize()
        want = {n: x.clone() for n, x in c.out.items()} | {"lse": c.lse.clone()}
        for x in (*c.out.values(), c.lse):
            x.fill_(float(i))
        for s in space.values():
            s.fill_(i)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, want[n]) for n, x in (*c.out.items(), ("lse", c.lse))), i


CAPTURED = '''
import numpy as np, torch
from paper_2408_04275_amd import binding as mm
T, H, V, nq, nk, d = 5000, 256, 300, 2, 1, 64
new = lambda *s: torch.randn(s, device="cuda").to(torch.bfloat16)
embed, norms, rope = mm.make_embed_desc(mm.BF16, H, V), mm.make_qk_norm_desc(mm.BF16, nq, nk, d), mm.make_rope_desc(mm.BF16, nq + nk, d)
cross = mm.make_cross_attn_desc(mm.BF16, nq, nk, d)
pack = mm.PackedBatch.on_device(np.array([0, 4000, 5000], dtype=np.int32))
batch = mm.CrossBatch.on_device(np.array([0, 4000, 5000]), np.array([0, 600]), np.array([600, 1300]), 1300)
table, kv, dy, w = new(V, H), new(1300, 2 * d), new(T, nq * d), {"q_w": new(d), "k_w": new(d)}
ids = torch.arange(T, dtype=torch.int32, device="cuda") % V
out = {n: torch.zeros_like(dy) for n in ("o", "dq")} | {n: torch.zeros((T, H), dtype=torch.bfloat16, device="cuda") for n in ("x", "y", "dx")}
out |= {n: torch.zeros((1300, d), dtype=torch.bfloat16, device="cuda") for n in ("dk", "dv")} | {"table": torch.zeros((V, H), device="cuda")}
lse = torch.zeros((nq, T), device="cuda")
need = [mm.mmtrain_embed_workspace_bytes(embed, T), mm.mmtrain_qk_norm_rope_workspace_bytes(norms, T), *(mm.mmtrain_cross_attn_workspace_bytes(cross, batch, b) for b in (0, 1))]
ws = torch.zeros(max(need), dtype=torch.uint8, device="cuda")
n = ws.numel()
def step():
    cw = mm.make_qk_norm_weights(w)
    t = mm.make_cross_attn_tensors(out["y"][:, :nq * d], kv[:, :d], kv[:, d:], out["o"], lse)
    g = mm.make_cross_attn_grads(dy, out["dq"], out["dk"], out["dv"])
    assert [mm.mmtrain_embed_fwd(embed, T, ids, table, None, out["x"]),
            mm.mmtrain_qk_norm_rope_fwd(norms, rope, T, pack, None, cw, out["x"], H, out["y"], H),
            mm.mmtrain_cross_attn_fwd(cross, batch, t, ws, n), mm.mmtrain_cross_attn_bwd(cross, batch, t, g, ws, n),
            mm.mmtrain_qk_norm_rope_bwd(norms, rope, T, pack, None, cw, out["x"], H, out["y"], H, out["dx"], H, None, 0, ws, n),
            mm.mmtrain_embed_bwd(embed, T, ids, out["dx"], out["table"], None, mm.BWD_WGRAD_F32, ws, n)] == [mm.OK] * 6
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    step()
for i in range(3):
    dy.copy_(new(T, nq * d))
    graph.replay()
    torch.cuda.synchronize()
    got = {k: v.clone() for k, v in out.items()}
    for v in out.values():
        v.zero_()
    step()
    torch.cuda.synchronize()
    assert all(torch.equal(v, got[k]) for k, v in out.items()) and float(got["table"].abs().sum()) > 0, i
print("captured first")
'''


def test_the_first_calls_of_a_process_may_be_captured():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", CAPTURED], cwd=root, capture_output=True, text=True, timeout=100)
    assert r.returncode == 0 and "captured first" in r.stdout, r.stdout + r.stderr
