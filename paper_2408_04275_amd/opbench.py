"""Operator microbenchmarks through the C-ABI: time one operator in isolation.

    python -m paper_2408_04275_amd.opbench gemm --layout nt --m 8192 --n 22016 --k 4096 [--iters 20]
    python -m paper_2408_04275_amd.opbench attn --config 3 [--iters 20]
    python -m paper_2408_04275_amd.opbench rope --config 3 [--interleaved] [--rot 64]
    python -m paper_2408_04275_amd.opbench join --config 3 [--post rms] [--pre rms] [--gate none]
    python -m paper_2408_04275_amd.opbench clip --config 3 --layers 1 [--dtype f32]
    python -m paper_2408_04275_amd.opbench copy --mb 512          (a plain copy kernel, for counter calibration)

Prints one JSON line per run.  Meant to be run alone or under rocprofv3 (kernel trace or --pmc).
"""
import argparse
import json
import sys
import time

import numpy as np
import torch

from . import binding as mm
from . import workloads as wl
from .harness import check


def _time(fn, iters, warmup=3):
    for _ in range(warmup):
        fn()
    torch.cuda.synchronize()
    e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    e0.record()
    for _ in range(iters):
        fn()
    e1.record()
    torch.cuda.synchronize()
    return e0.elapsed_time(e1) / iters


def bench_gemm(a):
    layout = {"nt": mm.GEMM_NT, "nn": mm.GEMM_NN, "tn": mm.GEMM_TN}[a.layout]
    M, N, K = a.m, a.n, a.k
    shp_a = (K, M) if layout == mm.GEMM_TN else (M, K)
    shp_b = (N, K) if layout == mm.GEMM_NT else (K, N)
    g = torch.Generator(device="cuda").manual_seed(0)
    A = torch.randn(shp_a, device="cuda", generator=g).to(torch.bfloat16)
    B = (torch.randn(shp_b, device="cuda", generator=g) * 0.02).to(torch.bfloat16)
    Cm = torch.empty((M, N), device="cuda", dtype=torch.bfloat16)
    R = torch.randn((M, N), device="cuda", generator=g).to(torch.bfloat16) if a.residual else None

    wsb = 0 if a.no_workspace or a.residual else mm.mmtrain_gemm_workspace_bytes(layout, M, N)
    ws = torch.empty(wsb, dtype=torch.uint8, device="cuda") if wsb else None

    def run():
        check(mm.mmtrain_gemm(mm.BF16, layout, M, N, K, A, shp_a[1], B, shp_b[1], Cm, N, None, R, 0, ws, wsb), "mmtrain_gemm")

    ms = _time(run, a.iters)
    print(json.dumps({"op": "gemm", "layout": a.layout, "M": M, "N": N, "K": K, "workspace_bytes": wsb, "ms": ms,
                      "tflops": 2.0 * M * N * K / ms / 1e9}))


def bench_attn(a):
    shape = wl.SHAPES[a.config]
    seed = wl.longtail_seed() if a.config == 4 else 0
    cu, modes, _ = wl.make_segments(a.config, seed)
    T = int(cu[-1])
    desc = mm.make_desc(shape.kind, mm.BF16, shape.hidden, shape.n_heads, shape.n_kv_heads, shape.head_dim, shape.ffn_hidden)
    batch = mm.PackedBatch.on_device(cu, modes)
    g = torch.Generator(device="cuda").manual_seed(0)
    qkv = torch.randn((T, shape.nqkv), device="cuda", generator=g).to(torch.bfloat16)
    d_o = torch.randn((T, shape.nq), device="cuda", generator=g).to(torch.bfloat16)
    o = torch.empty((T, shape.nq), device="cuda", dtype=torch.bfloat16)
    d_qkv = torch.empty_like(qkv)
    lse = torch.empty((shape.n_heads, T), device="cuda", dtype=torch.float32)
    wsb = mm.mmtrain_attn_workspace_bytes(T, len(cu) - 1, shape.n_heads)
    ws = torch.empty(wsb, dtype=torch.uint8, device="cuda")
    fl = wl.model_flops(shape, cu, modes)["attn_fwd"]
    ms_f = _time(lambda: check(mm.mmtrain_attn_fwd(desc, batch, qkv, o, lse, ws, wsb), "attn_fwd"), a.iters)
    ms_b = _time(lambda: check(mm.mmtrain_attn_bwd(desc, batch, qkv, o, lse, d_o, d_qkv, ws, wsb), "attn_bwd"), a.iters)
    out = {"op": "attn", "config": a.config, "T": T, "segments": len(cu) - 1, "fwd_ms": ms_f, "bwd_ms": ms_b,
           "fwd_tflops": fl / ms_f / 1e9, "bwd_tflops": 2 * fl / ms_b / 1e9}
    if a.cu_busy:
        # one forward + backward with the per-compute-unit busy counters on: max / mean over the units that ran work
        busy = torch.zeros((3, 1024), dtype=torch.int64, device="cuda")
        mm.mmtrain_profile_attn_busy(busy)
        check(mm.mmtrain_attn_fwd(desc, batch, qkv, o, lse, ws, wsb), "attn_fwd")
        check(mm.mmtrain_attn_bwd(desc, batch, qkv, o, lse, d_o, d_qkv, ws, wsb), "attn_bwd")
        torch.cuda.synchronize()
        mm.mmtrain_profile_attn_busy(None)
        rows = busy.cpu().numpy()
        for name, r in zip(("fwd", "dq", "dkv"), rows):
            used = r[r > 0].astype(np.float64) / 100.0            # 100 MHz ticks -> microseconds
            out["cu_busy_" + name] = {"units": int(used.size), "mean_us": float(used.mean()), "max_us": float(used.max()),
                                      "max_over_mean": float(used.max() / used.mean())}
    print(json.dumps(out))


def bench_adam(a):
    """One AdamW step over n fp32 master weights (+ bf16 working copy, gradient cleared): bytes moved per second."""
    n = a.mparams * 1_000_000
    g = torch.Generator(device="cuda").manual_seed(0)
    w = torch.randn(n, device="cuda", generator=g)
    gr = torch.randn(n, device="cuda", generator=g)
    m = torch.zeros(n, device="cuda")
    v = torch.zeros(n, device="cuda")
    out = torch.empty(n, device="cuda", dtype=torch.bfloat16)
    desc = mm.make_adam_desc(1e-4, 0.9, 0.95, 1e-8, 0.1, 1.0, 1, zero_grad=True)
    ms = _time(lambda: check(mm.mmtrain_adam_step(desc, n, w, gr, m, v, out, mm.BF16), "adam"), a.iters)
    nbytes = n * (16 + 12 + 2 + 4)
    print(json.dumps({"op": "adam", "n": n, "ms": ms, "GB_per_s": nbytes / ms / 1e6, "bytes_per_element": 34,
                      "frac_of_8TBps": nbytes / ms / 1e6 / 8000.0}))


def _segments(config):
    return wl.make_segments(config, wl.longtail_seed() if config == 4 else 0)[0]


def bench_rope(a):
    """Query and key heads of a workload's packed qkv: positions applied in place, and their gradient."""
    shape, cu = wl.SHAPES[a.config], _segments(a.config)
    T, heads = int(cu[-1]), shape.n_heads + shape.n_kv_heads
    batch = mm.PackedBatch.on_device(cu)
    desc = mm.make_rope_desc(mm.BF16, heads, shape.head_dim, a.rot, mm.ROPE_INTERLEAVED if a.interleaved else mm.ROPE_HALF)
    qkv = torch.randn((T, shape.nqkv), device="cuda").to(torch.bfloat16)
    out = {"op": "rope", "config": a.config, "T": T, "heads": heads, "head_dim": shape.head_dim, "rot_dim": desc.rot_dim, "interleaved": a.interleaved}
    for name, flags in (("fwd", 0), ("gradient", mm.ROPE_GRADIENT)):
        ms = _time(lambda: check(mm.mmtrain_rope(desc, T, batch, None, qkv, shape.nqkv, qkv, shape.nqkv, flags), "rope"), a.iters)
        out[name + "_ms"], out[name + "_GBps"] = ms, 4 * T * heads * desc.rot_dim / ms / 1e6
    print(json.dumps(out))


def bench_join(a):
    """The join of a workload's branch with its residual stream, forward and backward with every gradient."""
    shape, cu = wl.SHAPES[a.config], _segments(a.config)
    T, H = int(cu[-1]), shape.hidden
    norms = {"none": mm.NORM_NONE, "rms": mm.NORM_RMS, "layer": mm.NORM_LAYER}
    gates = {"none": mm.GATE_NONE, "channel": mm.GATE_CHANNEL, "segment": mm.GATE_SEGMENT}
    desc = mm.make_residual_norm_desc(mm.BF16, H, norms[a.post], norms[a.pre], gates[a.gate])
    batch = mm.PackedBatch.on_device(cu)
    names = [n + "_w" for n in ("post", "pre") if getattr(a, n) != "none"] + [n + "_b" for n in ("post", "pre") if getattr(a, n) == "layer"]
    w = {k: torch.ones(H, device="cuda", dtype=torch.bfloat16) for k in names}
    if a.gate != "none":
        w["gate"] = torch.ones((len(cu) - 1, H) if a.gate == "segment" else (H,), device="cuda", dtype=torch.bfloat16)
    x, b, dy, dh, y, h, dx, db = (torch.randn((T, H), device="cuda").to(torch.bfloat16) for _ in range(8))
    keep = {k: torch.empty(T, device="cuda") for k in mm.RESIDUAL_NORM_STATS}
    st = mm.make_residual_norm_stats(keep)
    grads = {k: torch.empty_like(v) for k, v in w.items()}
    wsb = mm.mmtrain_residual_norm_workspace_bytes(desc, T)
    ws = torch.empty(wsb, dtype=torch.uint8, device="cuda")
    cw, cg, pre = mm.make_residual_norm_weights(w), mm.make_residual_norm_grads(grads), a.pre != "none"
    ms_f = _time(lambda: check(mm.mmtrain_residual_norm_fwd(desc, T, batch, cw, x, b, y, h if pre else None, st), "join fwd"), a.iters)
    ms_b = _time(lambda: check(mm.mmtrain_residual_norm_bwd(desc, T, batch, cw, y, b, st, dy, dh if pre else None, dx, db, cg, 0, ws, wsb), "join bwd"), a.iters)
    bytes_f = 2 * T * H * (4 if pre else 3)
    bytes_b = 2 * T * H * (2 + 1 + 2 * pre + (a.post != "none" or a.gate != "none"))
    print(json.dumps({"op": "join", "config": a.config, "T": T, "hidden": H, "post": a.post, "pre": a.pre, "gate": a.gate, "fwd_ms": ms_f, "bwd_ms": ms_b,
                      "fwd_GBps": bytes_f / ms_f / 1e6, "bwd_GBps": bytes_b / ms_b / 1e6}))


def bench_clip(a):
    """Norm of the gradients of a workload's layers, their clipping in place and, from fp32, the clipped optimizer step instead."""
    dtype = torch.float32 if a.dtype == "f32" else torch.bfloat16
    sizes = [int(np.prod(s)) for s in wl.weight_shapes(wl.SHAPES[a.config]).values()] * a.layers
    at = np.concatenate([[0], np.cumsum([-(-n // 8) * 8 for n in sizes])])
    n = int(at[-1])
    flat = torch.randn(n, device="cuda").to(dtype)
    tensors = mm.make_grad_tensors([flat[int(p):int(p) + k] for p, k in zip(at, sizes)])
    wsb = mm.mmtrain_grad_norm_workspace_bytes(len(sizes))
    ws = torch.empty(wsb, dtype=torch.uint8, device="cuda")
    result = torch.zeros(2, dtype=torch.float64, device="cuda")
    ms_n = _time(lambda: check(mm.mmtrain_grad_norm(tensors, 1.0, result, ws, wsb), "grad_norm"), a.iters)
    result.view(torch.float32)[3] = 0.9999          # clipping in place over and over would run out of something to clip
    ms_c = _time(lambda: check(mm.mmtrain_grad_clip(tensors, result), "grad_clip"), a.iters)
    out = {"op": "clip", "config": a.config, "tensors": len(sizes), "n": n, "dtype": a.dtype, "norm_ms": ms_n, "clip_ms": ms_c,
           "norm_GBps": n * flat.element_size() / ms_n / 1e6, "clip_GBps": 2 * n * flat.element_size() / ms_c / 1e6}
    if a.dtype == "f32":
        w, m, v = (torch.zeros(n, device="cuda") for _ in range(3))
        p = torch.empty(n, device="cuda", dtype=torch.bfloat16)
        desc = mm.make_adam_desc(1e-4, 0.9, 0.95, 1e-8, 0.1, 1.0, 1)
        out["adam_ms"] = _time(lambda: check(mm.mmtrain_adam_step_clipped(desc, n, w, flat, m, v, p, mm.BF16, result), "adam"), a.iters)
    print(json.dumps(out))


def bench_copy(a):
    n = a.mb * (1 << 20)
    src = torch.empty(n, dtype=torch.uint8, device="cuda").fill_(1)
    dst = torch.empty_like(src)
    ms = _time(lambda: dst.copy_(src), a.iters)
    print(json.dumps({"op": "copy", "bytes_read": n, "bytes_written": n, "ms": ms, "GBps": 2 * n / ms / 1e6}))


def main(argv=None):
    ap = argparse.ArgumentParser()
    sub = ap.add_subparsers(dest="op", required=True)
    g = sub.add_parser("gemm")
    g.add_argument("--layout", default="nt", choices=["nt", "nn", "tn"])
    g.add_argument("--m", type=int, default=8192)
    g.add_argument("--n", type=int, default=22016)
    g.add_argument("--k", type=int, default=4096)
    g.add_argument("--residual", action="store_true")
    g.add_argument("--no-workspace", action="store_true", help="no scratch: the product is never cut along K")
    g.add_argument("--iters", type=int, default=20)
    t = sub.add_parser("attn")
    t.add_argument("--config", type=int, default=3)
    t.add_argument("--iters", type=int, default=20)
    t.add_argument("--cu-busy", action="store_true", help="also report the attention kernels' load balance over the compute units")
    ad = sub.add_parser("adam")
    ad.add_argument("--mparams", type=int, default=202, help="millions of parameters (202 = one 7B layer)")
    ad.add_argument("--iters", type=int, default=20)
    r = sub.add_parser("rope")
    r.add_argument("--config", type=int, default=3)
    r.add_argument("--rot", type=int, default=None, help="rotated features of a head (default: all)")
    r.add_argument("--interleaved", action="store_true")
    r.add_argument("--iters", type=int, default=20)
    j = sub.add_parser("join")
    j.add_argument("--config", type=int, default=3)
    j.add_argument("--post", default="rms", choices=["none", "rms", "layer"])
    j.add_argument("--pre", default="rms", choices=["none", "rms", "layer"])
    j.add_argument("--gate", default="none", choices=["none", "channel", "segment"])
    j.add_argument("--iters", type=int, default=20)
    cl = sub.add_parser("clip")
    cl.add_argument("--config", type=int, default=3)
    cl.add_argument("--layers", type=int, default=1)
    cl.add_argument("--dtype", default="f32", choices=["f32", "bf16"])
    cl.add_argument("--iters", type=int, default=20)
    c = sub.add_parser("copy")
    c.add_argument("--mb", type=int, default=512)
    c.add_argument("--iters", type=int, default=10)
    a = ap.parse_args(argv)
    mm.load_library()
    {"gemm": bench_gemm, "attn": bench_attn, "copy": bench_copy, "adam": bench_adam, "rope": bench_rope, "join": bench_join, "clip": bench_clip}[a.op](a)


if __name__ == "__main__":
    main()
