"""The operators of include/mmtrain_ops.h on the CPU: their oracle against independent definitions, and what the entry points refuse
(all argument checks run before any HIP call)."""
import os
import re
import subprocess
import sys

import numpy as np
import pytest
import torch

from oracle import operators_oracle as oo
from paper_2408_04275_amd import binding as mm

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x100000         # a 256-aligned address that no error path touches
NAN, INF = float("nan"), float("inf")


def test_header_and_binding_name_the_same_calls():
    text = open(os.path.join(ROOT, "include", "mmtrain_ops.h")).read()
    names = re.findall(r"MMTRAIN_API\s+[\w\s\*]+?\b(mmtrain_\w+)\s*\(", text)
    assert set(names) == set(mm.OPS_EXPORTS) and len(names) == len(mm.OPS_EXPORTS)
    for n in names:
        assert getattr(mm.load_library(), n) is not None


# ---- the oracle ------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_oracle_rope_is_a_complex_rotation_that_only_sees_distances(layout):
    rng = np.random.default_rng(0)
    theta = oo.rope_frequencies(12, 100.0)
    q, k = rng.standard_normal((1, 1, 16)), rng.standard_normal((1, 1, 16))
    score = lambda p, r: float(np.sum(oo.rope(q, [p], theta, layout)[0] * oo.rope(k, [r], theta, layout)[0]))  # noqa: E731
    assert np.isclose(score(5, 2), score(103, 100), rtol=1e-12) and not np.isclose(score(5, 2), score(6, 2))
    y, _ = oo.rope(q, [7], theta, layout, 1.5)
    z = q[0, 0, :6] + 1j * q[0, 0, 6:12] if layout == "half" else q[0, 0, 0:12:2] + 1j * q[0, 0, 1:12:2]
    z = 1.5 * z * np.exp(7j * theta)
    got = y[0, 0, :6] + 1j * y[0, 0, 6:12] if layout == "half" else y[0, 0, 0:12:2] + 1j * y[0, 0, 1:12:2]
    assert np.allclose(got, z, rtol=1e-13) and np.array_equal(y[..., 12:], q[..., 12:])


def test_oracle_rope_gradient_is_the_transpose():
    rng = np.random.default_rng(1)
    theta = oo.rope_frequencies(8, 10000.0)
    x, dy, pos = rng.standard_normal((4, 2, 10)), rng.standard_normal((4, 2, 10)), [0, 3, 1000, -5]
    for layout in ("half", "interleaved"):
        y, _ = oo.rope(x, pos, theta, layout, 1.25)
        dx, _ = oo.rope(dy, pos, theta, layout, 1.25, gradient=True)
        assert np.isclose(np.sum(y * dy), np.sum(x * dx), rtol=1e-13)


def test_oracle_rope_scaling_ends():
    plain = oo.rope_frequencies(64, 10000.0)
    assert np.allclose(oo.rope_frequencies(64, 10000.0, "linear", 4.0), plain / 4)
    for scaling in ("wavelength", "ramp"):
        f = oo.rope_frequencies(64, 10000.0, scaling, 8.0, 1.0, 32.0, 4096.0)
        turns = 4096.0 * plain / (2 * np.pi)
        assert np.all((f <= plain * (1 + 1e-15)) & (f >= plain / 8 * (1 - 1e-15)))
        assert np.allclose(f[turns > 40], plain[turns > 40]) and np.allclose(f[turns < 0.7], plain[turns < 0.7] / 8)
        assert np.all(np.diff(f) < 0)


def torch_norm(v, w, name, kind, eps):
    if kind == "none":
        return v
    if kind == "layer":
        return torch.nn.functional.layer_norm(v, (v.shape[1],), w[name + "_w"], w[name + "_b"], eps)
    return v * torch.rsqrt(v.square().mean(1, keepdim=True) + eps) * w[name + "_w"]


def make_params(rng, H, post, pre, gate, S=0):
    w = {}
    for n, kind in (("post", post), ("pre", pre)):
        if kind != "none":
            w[n + "_w"] = 1 + 0.2 * rng.standard_normal(H)
        if kind == "layer":
            w[n + "_b"] = 0.2 * rng.standard_normal(H)
    if gate != "none":
        w["gate"] = rng.standard_normal((S, H) if gate == "segment" else H)
    return w


KINDS = [("rms", "rms", "none"), ("layer", "layer", "segment"), ("none", "layer", "channel"), ("rms", "none", "channel"),
         ("none", "none", "segment"), ("layer", "rms", "none"), ("rms", "layer", "channel"), ("none", "rms", "none")]


@pytest.mark.parametrize("post,pre,gate", KINDS)
def test_oracle_join_matches_autograd(post, pre, gate):
    rng = np.random.default_rng(2)
    T, H, cu = 9, 16, np.array([0, 4, 4, 9])
    w = make_params(rng, H, post, pre, gate, 3)
    x, b, dy, dh = (rng.standard_normal((T, H)) for _ in range(4))
    seg = cu if gate == "segment" else None
    fwd, _ = oo.join_fwd(x, b, w, post, pre, 1e-5, 1e-3, 0.7, 0.4, seg)
    tw = {k: torch.tensor(v, requires_grad=True) for k, v in w.items()}
    tx, tb = torch.tensor(x, requires_grad=True), torch.tensor(b, requires_grad=True)
    n = torch_norm(tb, tw, "post", post, 1e-5)
    if gate != "none":
        n = n * (tw["gate"] if gate == "channel" else torch.repeat_interleave(tw["gate"], torch.tensor(np.diff(cu)), 0))
    y = 0.7 * tx + 0.4 * n
    h = torch_norm(y, tw, "pre", pre, 1e-3)
    loss = (y * torch.tensor(dy)).sum() + ((h * torch.tensor(dh)).sum() if pre != "none" else 0.0)
    loss.backward()
    assert np.allclose(fwd["y"], y.detach().numpy(), rtol=1e-12, atol=1e-13)
    if pre != "none":
        assert np.allclose(fwd["h"], h.detach().numpy(), rtol=1e-12, atol=1e-13)
    back, mag = oo.join_bwd(fwd["y"], b, w, fwd, dy, dh if pre != "none" else None, post, pre, 0.7, 0.4, seg)
    for k, ref in {"dx": tx.grad, "d_branch": tb.grad, **{k: t.grad for k, t in tw.items()}}.items():
        assert np.allclose(back[k], ref.numpy(), rtol=1e-10, atol=1e-12), k
        assert np.all(mag[k] >= np.abs(back[k]) * (1 - 1e-12)), k


def test_oracle_join_matches_differences():
    rng = np.random.default_rng(3)
    T, H, eps = 5, 8, 1e-6
    w = make_params(rng, H, "layer", "rms", "channel")
    x, b, dy, dh = (rng.standard_normal((T, H)) for _ in range(4))
    kw = dict(post="layer", pre="rms", alpha=0.9, beta=1.1)

    def loss(x, b, w):
        f, _ = oo.join_fwd(x, b, w, **kw)
        return np.sum(f["y"] * dy) + np.sum(f["h"] * dh)

    fwd, _ = oo.join_fwd(x, b, w, **kw)
    back, _ = oo.join_bwd(fwd["y"], b, w, fwd, dy, dh, **kw)
    for name, a in (("dx", x), ("d_branch", b), *w.items()):
        for i in np.ndindex(a.shape):
            at = a[i]
            a[i] = at + eps
            up = loss(x, b, w)
            a[i] = at - eps
            down = loss(x, b, w)
            a[i] = at
            assert np.isclose(back[name][i], (up - down) / (2 * eps), rtol=1e-6, atol=1e-7), (name, i)


def test_oracle_grad_norm():
    assert oo.grad_norm([[3.0], [4.0]], 10.0) == (25.0, 5.0, 1.0)
    assert oo.grad_norm([[3.0], [4.0]], 1.0) == (25.0, 5.0, 0.2)
    assert oo.grad_norm([], 1.0, 16.0) == (16.0, 4.0, 0.25)
    assert np.isnan(oo.grad_norm([[INF]], 1.0)[2]) and np.isnan(oo.grad_norm([[NAN]], 1.0)[2])
    assert oo.grad_norm([[0.0]], 0.0)[2] == 1.0 and oo.grad_norm([[2.0]], 0.0)[2] == 0.0


# ---- refusals --------------------------------------------------------------------------------------------------------
def pack(cu, T=None):
    return mm.PackedBatch(np.asarray(cu, dtype=np.int32), cu_dev=FAKE, total_tokens=T)


def rope(desc=None, T=16, batch=None, positions=FAKE, x=FAKE, ldx=512, y=FAKE + 4096, ldy=512, flags=0, **kw):
    desc = mm.make_rope_desc(**dict(dict(dtype=mm.BF16, n_heads=4, head_dim=128), **kw)) if desc is None else desc
    return mm.mmtrain_rope(desc, T, batch, positions, x, ldx, y, ldy, flags, stream=0)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=2), mm.ERR_INVALID_ARG), (dict(n_heads=0), mm.ERR_INVALID_ARG), (dict(head_dim=0), mm.ERR_INVALID_ARG),
    (dict(rot_dim=130), mm.ERR_INVALID_ARG), (dict(rot_dim=0), mm.ERR_INVALID_ARG), (dict(rot_dim=3), mm.ERR_UNSUPPORTED),
    (dict(head_dim=258, n_heads=1), mm.ERR_UNSUPPORTED), (dict(n_heads=65537), mm.ERR_UNSUPPORTED), (dict(layout=2), mm.ERR_INVALID_ARG), (dict(scaling=4), mm.ERR_INVALID_ARG),
    (dict(scaling=-1), mm.ERR_INVALID_ARG), (dict(base=1.0), mm.ERR_INVALID_ARG), (dict(base=NAN), mm.ERR_INVALID_ARG),
    (dict(base=INF), mm.ERR_INVALID_ARG), (dict(magnitude=-1.0), mm.ERR_INVALID_ARG), (dict(magnitude=NAN), mm.ERR_INVALID_ARG),
    (dict(scaling=mm.ROPE_LINEAR, factor=0.5), mm.ERR_INVALID_ARG), (dict(scaling=mm.ROPE_LINEAR, factor=INF), mm.ERR_INVALID_ARG),
    (dict(scaling=mm.ROPE_WAVELENGTH, factor=2.0, low=4.0, high=1.0, orig_context=8.0), mm.ERR_INVALID_ARG),
    (dict(scaling=mm.ROPE_WAVELENGTH, factor=2.0, low=0.0, high=1.0, orig_context=8.0), mm.ERR_INVALID_ARG),
    (dict(scaling=mm.ROPE_RAMP, factor=2.0, low=1.0, high=4.0, orig_context=0.0), mm.ERR_INVALID_ARG),
    (dict(scaling=mm.ROPE_RAMP, factor=NAN, low=1.0, high=4.0, orig_context=8.0), mm.ERR_INVALID_ARG),
    (dict(T=-1), mm.ERR_INVALID_ARG), (dict(flags=2), mm.ERR_INVALID_ARG), (dict(positions=None), mm.ERR_INVALID_ARG),
    (dict(positions=FAKE + 2), mm.ERR_INVALID_ARG), (dict(batch=pack([0, 16])), mm.ERR_INVALID_ARG),
    (dict(batch=pack([0, 9]), positions=None), mm.ERR_BAD_SEGMENTS), (dict(batch=pack([0, 20, 16]), positions=None), mm.ERR_BAD_SEGMENTS),
    (dict(batch=pack([1, 16]), positions=None), mm.ERR_BAD_SEGMENTS),
    (dict(x=None), mm.ERR_INVALID_ARG), (dict(y=None), mm.ERR_INVALID_ARG), (dict(x=FAKE + 2), mm.ERR_INVALID_ARG),
    (dict(ldx=511), mm.ERR_INVALID_ARG), (dict(ldy=511), mm.ERR_INVALID_ARG), (dict(y=FAKE, ldy=1024), mm.ERR_INVALID_ARG),
])
def test_rope_refuses(kw, status):
    assert rope(**kw) == status


def test_rope_takes_no_tokens_and_refuses_a_wrong_struct():
    assert rope(T=0, x=None, y=None, positions=None) == mm.OK
    assert rope(T=0, batch=pack([0]), x=None, y=None, positions=None) == mm.OK
    d = mm.make_rope_desc(mm.BF16, 4, 128)
    d.struct_size = 8
    assert rope(desc=d) == mm.ERR_INVALID_ARG
    assert mm.mmtrain_rope(None, 1, None, FAKE, FAKE, 512, FAKE, 512, stream=0) == mm.ERR_INVALID_ARG


A = [FAKE + (i << 20) for i in range(16)]       # addresses of different tensors


def sandwich(**kw):
    return mm.make_residual_norm_desc(**dict(dict(dtype=mm.BF16, hidden=64, post_norm=mm.NORM_RMS, pre_norm=mm.NORM_RMS), **kw))


def join_fwd(desc=None, T=4, batch=None, w=("post_w", "pre_w"), x=A[0], branch=A[1], y=A[2], h=A[3], stats=None, at=FAKE, **kw):
    desc = sandwich(**kw) if desc is None else desc
    weights = w if w is None else mm.make_residual_norm_weights({k: at for k in w})
    return mm.mmtrain_residual_norm_fwd(desc, T, batch, weights, x, branch, y, h, stats, stream=0)


def join_bwd(T=4, batch=None, w=("post_w", "pre_w"), y=A[0], branch=A[1], stats=("post_rstd", "pre_rstd"), dy=A[2], dh=A[3], dx=A[4], db=A[5],
             grads=("post_w", "pre_w"), flags=0, ws=A[6], ws_bytes=1 << 40, at=A[7], **kw):
    stats = stats if stats is None else mm.make_residual_norm_stats({k: A[8] for k in stats})
    grads = grads if grads is None else mm.make_residual_norm_grads({k: at for k in grads})
    return mm.mmtrain_residual_norm_bwd(sandwich(**kw), T, batch, mm.make_residual_norm_weights({k: FAKE for k in w}), y, branch, stats, dy, dh, dx,
                                        db, grads, flags, ws, ws_bytes, stream=0)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=7), mm.ERR_INVALID_ARG), (dict(hidden=0), mm.ERR_INVALID_ARG), (dict(hidden=60), mm.ERR_UNSUPPORTED),
    (dict(hidden=8200), mm.ERR_UNSUPPORTED), (dict(post_norm=3), mm.ERR_INVALID_ARG), (dict(pre_norm=-1), mm.ERR_INVALID_ARG),
    (dict(gate=3), mm.ERR_INVALID_ARG), (dict(post_eps=0.0), mm.ERR_INVALID_ARG), (dict(pre_eps=NAN), mm.ERR_INVALID_ARG),
    (dict(residual_scale=NAN), mm.ERR_INVALID_ARG), (dict(branch_scale=INF), mm.ERR_INVALID_ARG),
    (dict(T=-1), mm.ERR_INVALID_ARG), (dict(w=None), mm.ERR_INVALID_ARG), (dict(w=("post_w",)), mm.ERR_INVALID_ARG),
    (dict(w=("post_w", "pre_w", "pre_b")), mm.ERR_INVALID_ARG), (dict(w=("post_w", "pre_w", "gate")), mm.ERR_INVALID_ARG),
    (dict(at=FAKE + 8), mm.ERR_INVALID_ARG),
    (dict(pre_norm=mm.NORM_LAYER), mm.ERR_INVALID_ARG),                                   # its bias is missing
    (dict(gate=mm.GATE_SEGMENT, w=("post_w", "pre_w", "gate")), mm.ERR_INVALID_ARG),      # its segments are missing
    (dict(gate=mm.GATE_SEGMENT, w=("post_w", "pre_w", "gate"), batch=pack([0, 3])), mm.ERR_BAD_SEGMENTS),
    (dict(gate=mm.GATE_SEGMENT, w=("post_w", "pre_w", "gate"), batch=pack([0, 5, 4])), mm.ERR_BAD_SEGMENTS),
])
def test_join_refuses(kw, status):
    assert join_fwd(**kw) == status
    if kw.get("w", 0) is not None and "at" not in kw:
        assert join_bwd(**kw) == status


@pytest.mark.parametrize("kw", [
    dict(x=None), dict(branch=None), dict(y=None), dict(h=None), dict(x=A[0] + 8), dict(h=A[0]), dict(h=A[1]), dict(h=A[2]), dict(y=A[1]),
    dict(branch=A[0]), dict(pre_norm=mm.NORM_NONE, w=("post_w",)), dict(branch=None, y=None),
    dict(branch=None, y=None, post_norm=mm.NORM_NONE, pre_norm=mm.NORM_NONE, w=(), h=None),
    dict(stats=mm.make_residual_norm_stats({"pre_rstd": A[4] + 4}))])
def test_join_forward_refuses(kw):
    assert join_fwd(**kw) == mm.ERR_INVALID_ARG


@pytest.mark.parametrize("kw,status", [
    (dict(flags=4), mm.ERR_INVALID_ARG), (dict(y=None), mm.ERR_INVALID_ARG), (dict(branch=None), mm.ERR_INVALID_ARG), (dict(dh=None), mm.ERR_INVALID_ARG),
    (dict(stats=None), mm.ERR_INVALID_ARG), (dict(stats=("post_rstd",)), mm.ERR_INVALID_ARG), (dict(stats=("pre_rstd",)), mm.ERR_INVALID_ARG),
    (dict(grads=("pre_b",)), mm.ERR_INVALID_ARG), (dict(grads=("gate",)), mm.ERR_INVALID_ARG), (dict(at=A[7] + 8), mm.ERR_INVALID_ARG),
    (dict(dx=A[0]), mm.ERR_INVALID_ARG), (dict(dx=A[1]), mm.ERR_INVALID_ARG), (dict(dx=A[3]), mm.ERR_INVALID_ARG), (dict(dx=A[5]), mm.ERR_INVALID_ARG),
    (dict(db=A[0]), mm.ERR_INVALID_ARG), (dict(db=A[1]), mm.ERR_INVALID_ARG), (dict(db=A[2]), mm.ERR_INVALID_ARG), (dict(dx=A[4] + 2), mm.ERR_INVALID_ARG),
    (dict(ws=A[6] + 16), mm.ERR_INVALID_ARG), (dict(ws=None), mm.ERR_WORKSPACE), (dict(ws_bytes=64), mm.ERR_WORKSPACE),
    (dict(pre_norm=mm.NORM_NONE, w=("post_w",), grads=None), mm.ERR_INVALID_ARG),         # dh without the norm that has it
    (dict(pre_norm=mm.NORM_NONE, w=("post_w",), grads=None, dh=None, dy=None), mm.ERR_INVALID_ARG),
    (dict(post_norm=mm.NORM_NONE, w=("pre_w",), grads=None, branch=None), mm.ERR_INVALID_ARG),   # d_branch without a branch
])
def test_join_backward_refuses(kw, status):
    assert join_bwd(**kw) == status


def test_join_refuses_more_rows_than_it_counts():
    for T in ((1 << 30) + 1, (1 << 31) - 1):
        assert join_fwd(T=T) == mm.ERR_UNSUPPORTED
        assert join_bwd(T=T) == mm.ERR_UNSUPPORTED


def test_join_refuses_more_segments_than_it_has_gates_for():
    n = (1 << 20) + 1
    cu = np.zeros(n + 1, dtype=np.int32)
    cu[-1] = 4
    assert join_fwd(gate=mm.GATE_SEGMENT, w=("post_w", "pre_w", "gate"), batch=pack(cu)) == mm.ERR_UNSUPPORTED
    assert join_bwd(gate=mm.GATE_SEGMENT, w=("post_w", "pre_w", "gate"), batch=pack(cu)) == mm.ERR_UNSUPPORTED


def test_join_takes_no_tokens():
    assert join_fwd(T=0, x=None, branch=None, y=None, h=None) == mm.OK
    assert join_bwd(T=0, y=None, branch=None, stats=None, dy=None, dh=None, dx=None, db=None, grads=None, ws=None) == mm.OK


@pytest.mark.parametrize("gate", [mm.GATE_NONE, mm.GATE_CHANNEL, mm.GATE_SEGMENT])
def test_join_workspace_never_falls(gate):
    for H in (64, 1024, 1032, 2048, 4096, 8192):
        desc = mm.make_residual_norm_desc(mm.BF16, H, mm.NORM_LAYER, mm.NORM_RMS, gate)
        sizes = [mm.mmtrain_residual_norm_workspace_bytes(desc, T) for T in list(range(0, 3000)) + list(range(3000, 40000, 97))]
        assert sizes[0] > 0 and all(b >= a for a, b in zip(sizes, sizes[1:]))
    assert mm.mmtrain_residual_norm_workspace_bytes(sandwich(hidden=60), 4) == 0 and mm.mmtrain_residual_norm_workspace_bytes(sandwich(), -1) == 0


def tensors(*entries):
    return (mm.GradTensor * len(entries))(*[mm.GradTensor(*e) for e in entries])


GOOD = (A[0], None, 100, mm.F32, mm.F32)


@pytest.mark.parametrize("entry,status", [
    ((None, None, 1, mm.F32, mm.F32), mm.ERR_INVALID_ARG), ((A[1] + 4, None, 1, mm.F32, mm.F32), mm.ERR_INVALID_ARG),
    ((A[1], None, -1, mm.F32, mm.F32), mm.ERR_INVALID_ARG), ((A[1], None, 1, 2, mm.F32), mm.ERR_INVALID_ARG),
    ((A[1], None, (1 << 36) + 1, mm.BF16, mm.F32), mm.ERR_UNSUPPORTED)])
def test_grad_lists_refuse(entry, status):
    assert mm.mmtrain_grad_norm(tensors(GOOD, entry), 1.0, A[3], A[4], 1 << 30, stream=0) == status
    assert mm.mmtrain_grad_clip(tensors(GOOD, entry), A[3], stream=0) == status


def test_grad_norm_refuses():
    norm = lambda t=tensors(GOOD), m=1.0, r=A[3], w=A[4], n=1 << 30, f=0: mm.mmtrain_grad_norm(t, m, r, w, n, f, stream=0)  # noqa: E731
    assert norm(m=-1.0) == norm(m=NAN) == norm(r=None) == norm(r=A[3] + 8) == norm(w=A[4] + 16) == norm(f=2) == mm.ERR_INVALID_ARG
    assert norm(w=None) == norm(n=8) == mm.ERR_WORKSPACE
    assert mm.load_library().mmtrain_grad_norm(None, 3, 1.0, 0, A[3], A[4], 1 << 30, None) == mm.ERR_INVALID_ARG
    assert mm.load_library().mmtrain_grad_norm(tensors(GOOD), -1, 1.0, 0, A[3], A[4], 1 << 30, None) == mm.ERR_INVALID_ARG
    sizes = [mm.mmtrain_grad_norm_workspace_bytes(n) for n in range(0, 2000)]
    assert all(b >= a > 0 for a, b in zip(sizes, sizes[1:])) and mm.mmtrain_grad_norm_workspace_bytes(-1) == 0


def test_grad_clip_refuses_what_two_tensors_share():
    clip = lambda *e, r=A[3]: mm.mmtrain_grad_clip(tensors(*e), r, stream=0)  # noqa: E731
    f = mm.F32
    assert clip(GOOD, r=None) == clip(GOOD, r=A[3] + 4) == mm.ERR_INVALID_ARG
    assert clip(GOOD, GOOD) == mm.ERR_INVALID_ARG                                              # the same tensor twice
    assert clip(GOOD, (A[0] + 384, None, 4, f, f)) == mm.ERR_INVALID_ARG                       # its last quad
    assert clip(GOOD, (A[1], A[0] + 16, 4, f, f)) == mm.ERR_INVALID_ARG                        # an output in another's gradient
    assert clip((A[0], A[0] + 16, 100, f, f)) == mm.ERR_INVALID_ARG                            # ... and in its own, shifted
    assert clip((A[0], A[2], 100, f, f), (A[1], A[2], 100, f, f)) == mm.ERR_INVALID_ARG        # the same output
    assert clip((A[0], A[0], 100, f, mm.BF16)) == mm.ERR_INVALID_ARG                           # in place in another type
    assert clip((A[0], A[2] + 2, 100, f, f)) == clip((A[0], A[2], 100, f, 9)) == mm.ERR_INVALID_ARG
    assert mm.mmtrain_grad_clip(None, A[3], stream=0) == mm.OK and clip((None, None, 0, f, f)) == mm.OK


def test_grad_clip_finds_one_overlap_in_lists_of_any_order():
    # lists below and above what is sorted at a time, in address order and shuffled; the pair that overlaps stands anywhere
    rng = np.random.default_rng(4)
    for n in (2, 3, 500, 4096, 4097, 9000):
        for shuffled in (False, True):
            for kind in range(4):
                at = FAKE + 4096 * np.arange(3 * n)
                if shuffled:
                    rng.shuffle(at)
                grads, outs = [int(a) for a in at[:n]], [int(a) if i % 2 else None for i, a in enumerate(at[n:2 * n])]
                p, q = (int(i) for i in rng.choice(n, 2, replace=False))
                if kind == 0:                   # a gradient that another tensor clips in place
                    grads[p], outs[p] = grads[q] + 4080, None
                elif kind == 1:                 # an output in another's gradient, from its last 16 bytes
                    outs[p] = grads[q] + 4080
                elif kind == 2:                 # two outputs
                    outs[p] = int(at[2 * n])
                    outs[q] = outs[p] + 16
                else:                           # a range that holds another one, which is written
                    outs[p], outs[q] = int(at[2 * n]) + 1024, None
                    grads[q] = int(at[2 * n])
                e = [(g, o, 1024, mm.F32, mm.F32) for g, o in zip(grads, outs)]
                if kind == 3:
                    e[p] = (grads[p], outs[p], 8, mm.F32, mm.F32)
                assert mm.mmtrain_grad_clip(tensors(*e), A[3], stream=0) == mm.ERR_INVALID_ARG, (n, shuffled, kind)


NO_MEMORY = """
import resource
import numpy as np
from paper_2408_04275_amd import binding as mm
n = 1 << 21
t = np.zeros(n, dtype=[("grad", "u8"), ("out", "u8"), ("n", "i8"), ("dtype", "i4"), ("out_dtype", "i4")])
t["grad"] = 0x100000 + 16 * np.arange(n)
t["n"] = 4
lib = mm.load_library()
t["grad"][-1] = t["grad"][-2]
shuffled = t.copy()
shuffled["grad"][:-1] = shuffled["grad"][:-1][::-1]
shuffled["grad"][1] = shuffled["grad"][0]
used = int(open("/proc/self/statm").read().split()[0]) * resource.getpagesize()
resource.setrlimit(resource.RLIMIT_AS, (used + (8 << 20), resource.getrlimit(resource.RLIMIT_AS)[1]))
print([lib.mmtrain_grad_clip(a.ctypes.data, n, 0x100000, None) for a in (t, shuffled)])
"""


def test_grad_clip_allocates_no_host_memory():
    # a list of two million tensors with 8 MB left to the process: less than a list of their ranges would take
    r = subprocess.run([sys.executable, "-c", NO_MEMORY], cwd=ROOT, capture_output=True, text=True, timeout=120)
    assert r.stdout.strip() == str([mm.ERR_INVALID_ARG] * 2), r.stdout + r.stderr


def test_clipped_adam_refuses():
    step = lambda r, d=mm.make_adam_desc(1e-3), n=4: mm.mmtrain_adam_step_clipped(d, n, A[0], A[1], A[2], A[3], A[4], mm.BF16, r, stream=0)  # noqa: E731
    assert step(None) == step(A[5] + 8) == mm.ERR_INVALID_ARG
    assert step(A[5], mm.make_adam_desc(-1.0)) == step(A[5], n=-1) == mm.ERR_INVALID_ARG
    assert step(A[5], n=0) == mm.OK


def test_binding_refuses_lists_that_do_not_fit():
    g = torch.zeros(8)
    for bad in (lambda: mm.make_grad_tensors([g], [g, g]), lambda: mm.make_grad_tensors([g], [torch.zeros(7)]),
                lambda: mm.make_grad_tensors([g.half()]), lambda: mm.make_grad_tensors([torch.zeros(4, 4).t()])):
        with pytest.raises(ValueError):
            bad()
    t = mm.make_grad_tensors([g, g.bfloat16()], [None, torch.zeros(8)])
    assert (t[0].out, t[0].out_dtype, t[1].dtype, t[1].out_dtype, t[1].n) == (None, mm.F32, mm.BF16, mm.F32, 8)


def test_binding_finds_the_current_stream_with_public_calls_alone(monkeypatch):
    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream", raising=False)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: type("Stream", (), {"cuda_stream": 77}))
    assert mm._stream(None) == 77 and mm._stream(5) == 5
