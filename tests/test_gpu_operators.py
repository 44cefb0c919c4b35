"""The operators of include/mmtrain_ops.h on the GPU, against oracle/operators_oracle.py in 64 bits.

Tolerances.  An output is off by its rounding, finfo(dtype).eps / 2 of its value, and by the rounding errors of the fp32 evaluation.
The latter are at most k 2^-24 times the sum of the absolute values of the terms (the oracle's `mag`), k counting the roundings that
one term passes through:
  rotary: the turn is rounded to fp32 within half a turn (2^-26 of a turn, 2 pi 2^-26 rad = 1.6 x 2^-24), sine and cosine within 2 units in
    the last place (2 x 2^-24) and scaled (1), a product and a sum (2): k = 7, taken as 16.  Behind them stands the fp64 angle: the frequency's
    and the product's relative errors (4 x 2^-53) times the angle itself.
  join: a row's sums: up to 32 additions per thread and 10 to join the threads, twice where a mean is subtracted, about 10 more for the
    elementwise steps: k = 64 for a norm, twice that for backward through two norms: 128.
  sums over tokens: on top of that at most T / blocks + 512 / 32 + 32 additions: 128 more, for a summand that is itself off by 128: 256.
  gradient norm: fp64 sums (n 2^-53, negligible), one rounding of norm and factor each; a clipped gradient: those and its product, k = 3."""
import numpy as np
import pytest
import torch

from oracle import operators_oracle as oo
from paper_2408_04275_amd import binding as mm
from paper_2408_04275_amd.harness import check, torch_dtype
from test_operators import make_params

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
LAYOUTS = {"half": mm.ROPE_HALF, "interleaved": mm.ROPE_INTERLEAVED}
SCALINGS = {"plain": mm.ROPE_PLAIN, "linear": mm.ROPE_LINEAR, "wavelength": mm.ROPE_WAVELENGTH, "ramp": mm.ROPE_RAMP}
NORMS = {"none": mm.NORM_NONE, "rms": mm.NORM_RMS, "layer": mm.NORM_LAYER}
GATES = {"none": mm.GATE_NONE, "channel": mm.GATE_CHANNEL, "segment": mm.GATE_SEGMENT}


def dev(a, dtype):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to("cuda", torch_dtype(dtype))


def host(t):
    return t.detach().double().cpu().numpy()


def close(name, got, ref, mag, k, dtype, more=0.0):
    """got: a device tensor; ref and mag from the oracle; dtype: the type it was rounded to."""
    got = host(got).reshape(np.shape(ref))
    half = torch.finfo(torch_dtype(dtype)).eps / 2
    tol = half * np.abs(ref) + k * U * mag * (1 + half) + more + 1e-37
    bad = ~(np.abs(got - ref) <= tol)
    assert not bad.any(), f"{name}: {bad.sum()} of {bad.size} off, worst {np.max(np.abs(got - ref) / tol):.2f} x the tolerance"


# ---- rotary positions ------------------------------------------------------------------------------------------------
def rope_case(dtype, heads, d, rot, layout, scaling="plain", T=5, cu=None, positions=None, gradient=False, in_place=False, other=0, pad=0,
              magnitude=0.0, base=10000.0, seed=0):
    rng = np.random.default_rng(seed)
    theta = oo.rope_frequencies(rot, base, scaling, 4.0, 1.0, 32.0, 4096.0)
    m = magnitude or (0.1 * np.log(4.0) + 1.0 if scaling == "ramp" else 1.0)
    ldx = heads * d + other
    x = dev(rng.standard_normal((T, ldx)), dtype)
    before = x.clone()
    pos = oo.segment_positions(cu) if cu is not None else np.asarray(positions)
    ref, mag = oo.rope(host(x)[:, :heads * d].reshape(T, heads, d), pos, theta, layout, m, gradient)
    desc = mm.make_rope_desc(dtype, heads, d, rot, LAYOUTS[layout], base, SCALINGS[scaling], 4.0, 1.0, 32.0, 4096.0, magnitude)
    batch = mm.PackedBatch.on_device(cu) if cu is not None else None
    p = None if cu is not None else torch.tensor(pos, dtype=torch.int32, device="cuda")
    ldy = ldx if in_place else heads * d + pad
    y = x if in_place else torch.full((T, ldy), 7.0, dtype=x.dtype, device="cuda")
    check(mm.mmtrain_rope(desc, T, batch, p, x, ldx, y, ldy, mm.ROPE_GRADIENT if gradient else 0), "mmtrain_rope")
    torch.cuda.synchronize()
    half = np.zeros(d)
    half[:rot] = np.concatenate([theta, theta]) if layout == "half" else np.repeat(theta, 2)
    angle = np.abs(np.asarray(pos, np.float64))[:, None, None] * half
    # (magnitudes are rounded to fp32 too)
    close("y", y[:, :heads * d], ref.reshape(T, -1), mag.reshape(T, -1), 17, dtype, (8 * 2.0 ** -53 * angle * mag).reshape(T, -1))
    rest = host(y)[:, heads * d:]
    assert np.array_equal(rest, host(before)[:, heads * d:] if in_place else np.full_like(rest, 7.0))         # what stands behind is left alone
    keep = host(y)[:, :heads * d].reshape(T, heads, d)[..., rot:]
    assert np.array_equal(keep, host(before)[:, :heads * d].reshape(T, heads, d)[..., rot:])
    if not in_place:
        assert torch.equal(x, before)


WIDTHS = [(4, 128, 128), (3, 64, 64), (5, 80, 80), (2, 80, 40), (7, 80, 20), (1, 128, 64), (40, 96, 24), (3, 20, 10), (3, 7, 2), (2, 7, 6), (1, 256, 256),
          (2, 200, 198), (33, 16, 16), (1, 2, 2)]


@pytest.mark.parametrize("dtype", [mm.BF16, mm.F32])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("heads,d,rot", WIDTHS)
def test_rope_widths(dtype, layout, heads, d, rot):
    cu = np.array([0, 1, 1, 70, 131], dtype=np.int32)
    rope_case(dtype, heads, d, rot, layout, T=131, cu=cu, seed=1)
    rope_case(dtype, heads, d, rot, layout, T=131, cu=cu, in_place=True, gradient=True, other=2 * d, seed=2)
    rope_case(dtype, heads, d, rot, layout, T=9, positions=np.arange(9) * 1000, other=1, pad=3, seed=3)      # rows that are not aligned


@pytest.mark.parametrize("scaling", list(SCALINGS))
@pytest.mark.parametrize("gradient", [False, True])
def test_rope_scaling(scaling, gradient):
    pos = [0, 1, 4095, 4096, 131071, 2 ** 20 + 1]
    for layout in LAYOUTS:
        rope_case(mm.F32, 3, 128, 128, layout, scaling, T=6, positions=pos, gradient=gradient, seed=4)
        rope_case(mm.BF16, 3, 128, 64, layout, scaling, T=6, positions=pos, gradient=gradient, magnitude=1.5, base=500000.0, seed=5)


@pytest.mark.parametrize("T", [1, 2, 3, 63, 257, 1031, 4111])
def test_rope_lengths(T):
    cu = np.array([0, T // 3, T // 3, T], dtype=np.int32)
    rope_case(mm.BF16, 12, 128, 128, "half", T=T, cu=cu, seed=6)
    rope_case(mm.F32, 5, 80, 40, "interleaved", T=T, positions=np.arange(T)[::-1] * 7, in_place=True, seed=7)


def test_rope_far_and_negative_positions():
    pos = [2 ** 31 - 1, -2 ** 31, -1, 2 ** 30 + 7, 0]
    for layout in LAYOUTS:
        rope_case(mm.F32, 2, 64, 64, layout, positions=pos, seed=8)


def test_rope_many_segments():
    cu = np.concatenate([[0], np.repeat(np.arange(1, 400), 2), [1201]]).astype(np.int32)     # an empty segment behind each
    rope_case(mm.BF16, 2, 64, 64, "half", T=1201, cu=cu, seed=9)


def test_rope_rows_past_32_bits():
    # the last row of a view whose elements stand past 2^31
    T, ld = 3, (1 << 30) + 8
    x = torch.zeros(2 * ld + 256, dtype=torch.bfloat16, device="cuda")
    rng = np.random.default_rng(10)
    rows = dev(rng.standard_normal((T, 256)), mm.BF16)
    for t in range(T):
        x[t * ld:t * ld + 256] = rows[t]
    desc = mm.make_rope_desc(mm.BF16, 2, 128)
    pos = torch.tensor([1, 2, 3], dtype=torch.int32, device="cuda")
    check(mm.mmtrain_rope(desc, T, None, pos, x, ld, x, ld), "mmtrain_rope")
    out = torch.empty_like(rows)
    check(mm.mmtrain_rope(desc, T, None, pos, rows, 256, out, 256), "mmtrain_rope")
    assert all(torch.equal(x[t * ld:t * ld + 256], out[t]) for t in range(T))


@pytest.mark.parametrize("T", [(1 << 20) + 5, (1 << 24) + 5])
def test_rope_of_more_tokens_than_a_grid_has_workgroups(T):
    # a token a workgroup, and more than 2^32 threads
    x = torch.zeros((T, 1024), dtype=torch.bfloat16, device="cuda")
    at = torch.tensor([0, 1, (1 << 20) - 1, 1 << 20, T // 2, T - 2, T - 1], device="cuda")
    rows = torch.randn((7, 1024), device="cuda").bfloat16()
    x[at] = rows
    desc = mm.make_rope_desc(mm.BF16, 512, 2)
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    check(mm.mmtrain_rope(desc, T, None, pos, x, 1024, x, 1024), "mmtrain_rope")
    out = torch.empty_like(rows)
    check(mm.mmtrain_rope(desc, 7, None, at.int(), rows, 1024, out, 1024), "mmtrain_rope")
    assert torch.equal(x[at], out)
    x[at] = 0
    assert not any(bool(p.any()) for p in x.split(1 << 20))


def test_rope_special_values_stay_in_their_pair():
    x = torch.zeros((1, 16), dtype=torch.float32, device="cuda")
    x[0, 3], x[0, 6] = float("inf"), float("nan")
    y = torch.empty_like(x)
    check(mm.mmtrain_rope(mm.make_rope_desc(mm.F32, 1, 16), 1, None, torch.ones(1, dtype=torch.int32, device="cuda"), x, 16, y, 16), "mmtrain_rope")
    touched = {3, 11, 6, 14}
    assert all(bool(torch.isfinite(y[0, i])) == (i not in touched) for i in range(16))


# ---- the join of branch and residual stream ----------------------------------------------------------------------------
def join_case(dtype, T, H, post, pre, gate, cu=None, flags=0, offset=0.0, seed=0, alias=False, no_dy=False, wanted=None, branch=True,
              alpha=0.75, beta=0.5):
    rng = np.random.default_rng(seed)
    S = 0 if cu is None else len(cu) - 1
    wd = {k: dev(v, dtype) for k, v in make_params(rng, H, post, pre, gate, S).items()}
    w = {k: host(v) for k, v in wd.items()}
    x, b, dy, dh = (dev(rng.standard_normal((T, H)) * s + o, dtype) for s, o in ((1, offset), (2, offset), (1, 0), (1, 0)))
    desc = mm.make_residual_norm_desc(dtype, H, NORMS[post], NORMS[pre], GATES[gate], 1e-5, 1e-4, alpha, beta)
    batch = mm.PackedBatch.on_device(cu) if cu is not None else None
    weights = mm.make_residual_norm_weights(wd)
    seg = cu if gate == "segment" else None
    kinds = dict(post=post, pre=pre)
    # forward
    ref, mag = oo.join_fwd(host(x), host(b) if branch else None, w, post_eps=np.float32(1e-5), pre_eps=np.float32(1e-4), alpha=alpha, beta=beta, cu=seg, **kinds)
    x0, y, h = x.clone(), x if alias else torch.empty_like(x), torch.empty_like(x)
    st = {k: torch.full((T,), 9.0, device="cuda") for k in mm.RESIDUAL_NORM_STATS}
    check(mm.mmtrain_residual_norm_fwd(desc, T, batch, weights, x, b if branch else None, y if branch else None, h if pre != "none" else None,
                                       mm.make_residual_norm_stats(st)), "fwd")
    if branch:
        close("y", y, ref["y"], mag["y"], 64, dtype)
    if pre != "none":
        close("h", h, ref["h"], mag["h"], 128, dtype)
    # statistics: the mean's error is k U of the mean absolute value; 1 / deviation's follows from the variance's
    stats = {}
    for n, v in (("post", host(b)), ("pre", ref["y"] if branch else host(x0))):
        if kinds[n] == "none":
            continue
        scale = np.sqrt((v ** 2).mean(1))
        if kinds[n] == "layer":
            close(n + "_mean", st[n + "_mean"], ref[n + "_mean"], scale, 64, mm.F32)
        rel = 64 * U * (1 + scale * ref[n + "_rstd"])
        assert np.all(np.abs(host(st[n + "_rstd"]) - ref[n + "_rstd"]) <= rel * ref[n + "_rstd"]), n
        stats[n + "_mean"], stats[n + "_rstd"] = host(st[n + "_mean"]), host(st[n + "_rstd"])
    for k in st:
        if k not in stats or kinds[k.split("_")[0]] != "layer" and k.endswith("mean"):
            assert torch.all(st[k] == 9.0), k                           # what the description does not have is not written
    # backward, from what forward has stored
    names = list(w) if wanted is None else wanted
    grad_dtype = mm.F32 if flags & mm.BWD_WGRAD_F32 else dtype
    g = {k: dev(rng.standard_normal(w[k].shape), grad_dtype) for k in names}
    g0 = {k: host(v) for k, v in g.items()}
    v = y if branch else x
    dyt = None if no_dy else dy
    ref, mag = oo.join_bwd(host(v), host(b) if branch else None, w, stats, None if no_dy else host(dy), host(dh) if pre != "none" else None, alpha=alpha,
                           beta=beta, cu=seg, **kinds)
    dx = dyt if alias and dyt is not None else torch.empty_like(x)
    db = (dh if alias and pre != "none" else torch.empty_like(x)) if branch else None
    wsb = mm.mmtrain_residual_norm_workspace_bytes(desc, T)
    ws = torch.full((wsb,), 255, dtype=torch.uint8, device="cuda")                        # NaN all over
    check(mm.mmtrain_residual_norm_bwd(desc, T, batch, weights, v, b if branch else None, mm.make_residual_norm_stats(st), dyt,
                                       dh if pre != "none" else None, dx, db, mm.make_residual_norm_grads(g), flags, ws, wsb), "bwd")
    torch.cuda.synchronize()
    close("dx", dx, ref["dx"], mag["dx"], 128, dtype)
    if branch:
        close("d_branch", db, ref["d_branch"], mag["d_branch"], 128, dtype)
    for k in names:
        r, m = ref[k], mag[k]
        if flags & mm.BWD_ACCUMULATE_WGRAD:
            r, m = r + g0[k], m + np.abs(g0[k])
        close("d" + k, g[k], r, m, 256, grad_dtype)


FORMS = [("rms", "rms", "none"), ("layer", "layer", "segment"), ("none", "layer", "channel"), ("rms", "none", "channel"), ("none", "rms", "segment"),
         ("layer", "rms", "none"), ("none", "none", "segment"), ("none", "none", "none"), ("layer", "none", "none"), ("none", "rms", "none")]
RAGGED = np.array([0, 1, 1, 70, 199, 200, 200, 643], dtype=np.int32)
MAIN = mm.BWD_ACCUMULATE_WGRAD | mm.BWD_WGRAD_F32


@pytest.mark.parametrize("dtype", [mm.BF16, mm.F32])
@pytest.mark.parametrize("post,pre,gate", FORMS)
def test_join_forms(dtype, post, pre, gate):
    cu = RAGGED if gate == "segment" else None
    join_case(dtype, 643, 256, post, pre, gate, cu, seed=1)
    join_case(dtype, 643, 1032, post, pre, gate, cu, flags=MAIN, seed=2, alias=True)


@pytest.mark.parametrize("H", [8, 16, 504, 512, 520, 1024, 1280, 2040, 2048, 2056, 4096, 4104, 5120, 8184, 8192])
@pytest.mark.parametrize("post,pre,gate", [("rms", "rms", "none"), ("layer", "layer", "segment")])
def test_join_widths(H, post, pre, gate):
    cu = np.array([0, 5, 5, 36, 37], dtype=np.int32) if gate == "segment" else None
    join_case(mm.BF16, 37, H, post, pre, gate, cu, seed=3)
    join_case(mm.F32, 37, H, post, pre, gate, cu, flags=mm.BWD_ACCUMULATE_WGRAD, seed=4)


@pytest.mark.parametrize("T", [1, 2, 3, 5, 255, 513, 1031, 2307])
@pytest.mark.parametrize("post,pre,gate", [("rms", "rms", "channel"), ("layer", "layer", "segment")])
def test_join_lengths(T, post, pre, gate):
    cu = np.array([0, T // 2, T // 2, T], dtype=np.int32) if gate == "segment" else None
    join_case(mm.BF16, T, 1024, post, pre, gate, cu, seed=5)
    join_case(mm.F32, T, 136, post, pre, gate, cu, flags=MAIN, seed=6)


@pytest.mark.parametrize("H", [64, 1280, 4096])
def test_join_a_gate_for_every_token_and_for_all(H):
    for cu in (np.arange(0, 601), np.array([0, 600]), np.array([0, 0, 0, 600, 600, 600]), np.array([0, 599, 600])):
        join_case(mm.BF16, 600, H, "none", "rms", "segment", cu.astype(np.int32), seed=7)
        join_case(mm.F32, 600, H, "rms", "none", "segment", cu.astype(np.int32), flags=mm.BWD_ACCUMULATE_WGRAD, seed=8)


def test_join_many_segments_and_many_rows():
    cu = np.zeros(70001, dtype=np.int32)
    cu[30000:] = 40                             # nearly all of them empty, more than a grid's second dimension takes
    cu[69990:] = 333
    join_case(mm.BF16, 333, 64, "layer", "rms", "segment", cu, seed=19)
    join_case(mm.F32, 333, 64, "none", "none", "segment", cu, flags=mm.BWD_ACCUMULATE_WGRAD, seed=20)
    # (a summand of a column passes through T / 256 additions more than the 2307 rows of the other tests: 60000 rows / 256 = 234)
    join_case(mm.F32, 60000, 64, "rms", "layer", "channel", wanted=[], seed=21)


def test_join_rows_past_32_bits():
    T, H = (1 << 18) + 8, 8192                  # 2^31 elements and more
    w = {"post_w": torch.randn(H, device="cuda").bfloat16(), "pre_w": torch.randn(H, device="cuda").bfloat16()}
    x, b = (torch.zeros((T, H), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for t in (x, b):
        t[-8:] = torch.randn((8, H), device="cuda")
    desc = mm.make_residual_norm_desc(mm.BF16, H, mm.NORM_RMS, mm.NORM_RMS)
    cw = mm.make_residual_norm_weights(w)
    y, h = torch.empty_like(x), torch.empty_like(x)
    st = {k: torch.empty(T, device="cuda") for k in ("post_rstd", "pre_rstd")}
    check(mm.mmtrain_residual_norm_fwd(desc, T, None, cw, x, b, y, h, mm.make_residual_norm_stats(st)), "fwd")
    few = [torch.empty((8, H), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    check(mm.mmtrain_residual_norm_fwd(desc, 8, None, cw, x[-8:], b[-8:], few[0], few[1]), "fwd")
    assert torch.equal(y[-8:], few[0]) and torch.equal(h[-8:], few[1])
    grads = {k: torch.empty(H, device="cuda") for k in w}
    wsb = mm.mmtrain_residual_norm_workspace_bytes(desc, T)
    ws = torch.empty(wsb, dtype=torch.uint8, device="cuda")
    dx, db = torch.empty_like(x), torch.empty_like(x)
    args = lambda n, v, o, p, q, s, g: mm.mmtrain_residual_norm_bwd(desc, n, None, cw, v, o, mm.make_residual_norm_stats(s), None, o, p, q,  # noqa: E731
                                                                     mm.make_residual_norm_grads(g), mm.BWD_WGRAD_F32, ws, wsb)
    check(args(T, y, b, dx, db, st, grads), "bwd")
    some = {k: torch.empty(H, device="cuda") for k in w}
    check(args(8, y[-8:], b[-8:], few[0], few[1], {k: v[-8:] for k, v in st.items()}, some), "bwd")
    assert torch.equal(dx[-8:], few[0]) and torch.equal(db[-8:], few[1])
    for k in w:                                 # the other rows' gradients are zero: the same eight summands, in another order
        assert torch.allclose(grads[k], some[k], rtol=1e-5, atol=1e-4)


@pytest.mark.parametrize("dtype", [mm.BF16, mm.F32])
def test_join_other_forms(dtype):
    for pre in ("rms", "layer"):                # the norm in front of the first block: no branch
        join_case(dtype, 77, 1024, "none", pre, "none", branch=False, seed=9)
        join_case(dtype, 77, 2560, "none", pre, "none", branch=False, flags=mm.BWD_WGRAD_F32, no_dy=True, alias=True, seed=10)
    join_case(dtype, 77, 512, "rms", "layer", "channel", no_dy=True, seed=11)
    join_case(dtype, 77, 512, "layer", "layer", "channel", wanted=[], seed=12)                      # frozen
    join_case(dtype, 77, 512, "layer", "layer", "channel", wanted=["post_b", "pre_w"], seed=13)
    join_case(dtype, 77, 512, "layer", "layer", "segment", np.array([0, 70, 77], dtype=np.int32), wanted=["post_w", "pre_b"], seed=14)
    join_case(dtype, 77, 512, "layer", "layer", "segment", np.array([0, 70, 77], dtype=np.int32), wanted=["gate"], seed=15)
    join_case(dtype, 77, 1024, "rms", "rms", "none", alpha=0.0, beta=-1.0, seed=16)


@pytest.mark.parametrize("post,pre", [("layer", "layer"), ("rms", "rms")])
def test_join_rows_far_from_zero(post, pre):
    join_case(mm.F32, 65, 1024, post, pre, "none", offset=100.0, seed=17)
    join_case(mm.BF16, 65, 4096, post, pre, "none", offset=30.0, seed=18)


def test_join_rows_of_zeros_and_specials():
    # a zero row: 1 / sqrt(eps), h = bias; a NaN stays in its row
    T, H = 5, 64
    w = {"pre_w": torch.ones(H, device="cuda"), "pre_b": torch.full((H,), 0.5, device="cuda")}
    x, b = torch.zeros((T, H), device="cuda"), torch.zeros((T, H), device="cuda")
    b[3, 7] = float("nan")
    y, h, r = torch.empty_like(x), torch.empty_like(x), torch.empty(T, device="cuda")
    check(mm.mmtrain_residual_norm_fwd(mm.make_residual_norm_desc(mm.F32, H, pre_norm=mm.NORM_LAYER), T, None, mm.make_residual_norm_weights(w), x, b, y, h,
                                       mm.make_residual_norm_stats({"pre_rstd": r})), "fwd")
    rows = [0, 1, 2, 4]
    assert torch.all(h[rows] == 0.5) and torch.all(y[rows] == 0) and torch.all(torch.isnan(h[3]))
    assert np.allclose(host(r)[rows], 1 / np.sqrt(np.float32(1e-5)), rtol=1e-6)


def test_join_no_tokens_writes_zero_gradients():
    H = 64
    for gate, cu in (("channel", None), ("segment", np.array([0, 0, 0], dtype=np.int32))):
        desc = mm.make_residual_norm_desc(mm.F32, H, mm.NORM_RMS, mm.NORM_RMS, GATES[gate])
        for flags, want in ((0, 0.0), (mm.BWD_ACCUMULATE_WGRAD, 3.0)):
            w = {k: torch.ones((2, H) if k == "gate" and cu is not None else H, device="cuda") for k in ("post_w", "pre_w", "gate")}
            g = {k: torch.full_like(v, 3.0) for k, v in w.items()}
            wsb = mm.mmtrain_residual_norm_workspace_bytes(desc, 0)
            ws = torch.full((wsb,), 255, dtype=torch.uint8, device="cuda")
            check(mm.mmtrain_residual_norm_bwd(desc, 0, mm.PackedBatch.on_device(cu) if cu is not None else None, mm.make_residual_norm_weights(w), None, None,
                                               None, None, None, None, None, mm.make_residual_norm_grads(g), flags, ws, wsb), "bwd")
            assert all(torch.all(v == want) for v in g.values())


# ---- gradient norm and clipping ------------------------------------------------------------------------------------------
def grads_of(sizes, dtypes, std=1.0, seed=0):
    rng = np.random.default_rng(seed)
    return [dev(rng.standard_normal(n) * std, dtypes[i % len(dtypes)]) for i, n in enumerate(sizes)]


def norm_of(tensors, n, max_norm, result=None, flags=0):
    result = torch.full((2,), float("nan"), dtype=torch.float64, device="cuda") if result is None else result
    wsb = mm.mmtrain_grad_norm_workspace_bytes(n)
    ws = torch.full((wsb,), 255, dtype=torch.uint8, device="cuda")
    check(mm.mmtrain_grad_norm(tensors, max_norm, result, ws, wsb, flags), "mmtrain_grad_norm")
    torch.cuda.synchronize()
    f = result.view(torch.float32)
    return result, float(result[0]), float(f[2]), float(f[3])


SIZES = [[1], [5], [4097], [100003], [0, 3, 0, 8, 16384, 16385, 7], [1 + 97 * i for i in range(300)], [8] * 129, [3000001, 1, 65536]]


@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: f"{len(s)}x{max(s)}")
@pytest.mark.parametrize("dtypes", [(mm.F32,), (mm.BF16,), (mm.F32, mm.BF16)], ids=["f32", "bf16", "mixed"])
@pytest.mark.parametrize("max_norm", [0.5, 1e9])
def test_grad_norm_and_clip(sizes, dtypes, max_norm):
    grads = grads_of(sizes, dtypes)
    q, norm, factor = oo.grad_norm([host(g) for g in grads], max_norm)
    same = mm.make_grad_tensors(grads)
    result, got_q, got_norm, got_factor = norm_of(same, len(grads), max_norm)
    assert abs(got_q - q) <= 1e-12 * q and abs(got_norm - norm) <= 2 * U * norm and abs(got_factor - factor) <= 2 * U * factor
    for out in ((mm.F32,), (mm.BF16,), None):
        outs = None if out is None else [torch.full((g.numel(),), 5.0, dtype=torch_dtype(out[0]), device="cuda") for g in grads]
        before = [g.clone() for g in grads]
        check(mm.mmtrain_grad_clip(mm.make_grad_tensors(grads, outs), result), "mmtrain_grad_clip")
        torch.cuda.synchronize()
        for i, b in enumerate(before):
            got = grads[i] if outs is None else outs[i]
            ref = host(b) * factor
            close(f"tensor {i}", got, ref, np.abs(ref), 3, mm.BF16 if got.dtype == torch.bfloat16 else mm.F32)
            assert outs is None or torch.equal(grads[i], b)


def test_grad_clip_writes_nothing_past_its_tensors():
    flat = torch.full((4096,), 2.0, device="cuda")
    views = [flat[0:5], flat[8:17], flat[1024:2049]]
    tensors = mm.make_grad_tensors(views)
    result, *_ = norm_of(tensors, 3, 1.0)
    check(mm.mmtrain_grad_clip(tensors, result), "clip")
    touched = torch.zeros(4096, dtype=torch.bool, device="cuda")
    for a, b in ((0, 5), (8, 17), (1024, 2049)):
        touched[a:b] = True
    assert torch.all(flat[~touched] == 2.0) and torch.all(flat[touched] < 1.0)


def test_grad_clip_one_gradient_into_two_places():
    g = grads_of([1000], (mm.F32,), seed=5)[0]
    outs = [torch.empty(1000, device="cuda"), torch.empty(500, device="cuda", dtype=torch.bfloat16)]
    result, *_ , factor = norm_of(mm.make_grad_tensors([g]), 1, 1.0)
    check(mm.mmtrain_grad_clip(mm.make_grad_tensors([g, g[:500]], outs), result), "clip")
    ref = host(g) * factor
    close("fp32", outs[0], ref, np.abs(ref), 3, mm.F32)
    close("bf16", outs[1], ref[:500], np.abs(ref[:500]), 3, mm.BF16)


def test_grad_tensor_past_32_bits():
    n = (1 << 31) + 21
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g[-1], g[-13], g[(1 << 31) + 1], g[0] = 3.0, 4.0, 12.0, 84.0
    tensors = mm.make_grad_tensors([g])
    result, q, norm, factor = norm_of(tensors, 1, 1.0)
    assert (q, norm) == (7225.0, 85.0)
    check(mm.mmtrain_grad_clip(tensors, result), "clip")
    for i, v in ((-1, 3.0), (-13, 4.0), ((1 << 31) + 1, 12.0), (0, 84.0)):
        assert abs(float(g[i]) - v / 85.0) <= 2.0 ** -8 * v / 85.0


def test_grad_norm_extremes():
    big = torch.full((1000,), 3e38, device="cuda")                      # squares past fp32
    result, q, norm, factor = norm_of(mm.make_grad_tensors([big[:1]]), 1, 1.0)
    assert np.isclose(norm, 3e38, rtol=1e-6) and np.isclose(factor, 1 / 3e38, rtol=1e-6)
    assert norm_of(mm.make_grad_tensors([big]), 1, 1.0)[2] == np.inf     # the norm itself is past fp32
    tiny = torch.full((1000,), 1e-30, device="cuda")                    # squares that fp32 has not
    assert np.isclose(norm_of(mm.make_grad_tensors([tiny]), 1, 1.0)[2], 1e-30 * np.sqrt(1000), rtol=1e-6)
    zero = torch.zeros(10, device="cuda")
    assert norm_of(mm.make_grad_tensors([zero]), 1, 0.0)[1:] == (0.0, 0.0, 1.0)
    assert norm_of(None, 0, 1.0)[1:] == (0.0, 0.0, 1.0)
    one = torch.ones(16, device="cuda")
    assert norm_of(mm.make_grad_tensors([one]), 1, float("inf"))[1:] == (16.0, 4.0, 1.0)
    assert norm_of(mm.make_grad_tensors([one]), 1, 4.0)[3] == 1.0 and norm_of(mm.make_grad_tensors([one]), 1, 0.0)[3] == 0.0


def test_grad_norm_past_fp32_leaves_everything_alone():
    # what the norm says and what is done agree: 1000 x 3e38^2 is a finite sum, its root no fp32 number
    g = torch.full((1000,), 3e38, device="cuda")
    result, q, norm, factor = norm_of(mm.make_grad_tensors([g]), 1, 1.0)
    assert np.isfinite(q) and norm == np.inf and np.isnan(factor)
    before = g.clone()
    check(mm.mmtrain_grad_clip(mm.make_grad_tensors([g]), result), "clip")
    assert torch.equal(g, before)


def test_grad_norm_adds_up_calls_and_ranks():
    a, b = grads_of([5000], (mm.F32,), seed=1)[0], grads_of([3001], (mm.BF16,), seed=2)[0]
    q, norm, factor = oo.grad_norm([host(a), host(b)], 1.0)
    result, *_ = norm_of(mm.make_grad_tensors([a]), 1, 1.0)
    _, got_q, got_norm, got_factor = norm_of(mm.make_grad_tensors([b]), 1, 1.0, result, mm.GRAD_NORM_ADD)
    assert np.isclose(got_q, q, rtol=1e-12) and np.isclose(got_norm, norm, rtol=2 * U) and np.isclose(got_factor, factor, rtol=2 * U)
    result[0] = 4.0 * q                                                 # as if other ranks had added theirs
    _, got_q, got_norm, _ = norm_of(None, 0, 1.0, result, mm.GRAD_NORM_ADD)
    assert np.isclose(got_norm, 2 * norm, rtol=2 * U)


@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_a_norm_that_is_not_finite_leaves_everything_alone(bad):
    g = grads_of([1000, 33], (mm.F32, mm.BF16))
    g[0][500] = bad
    before = [t.clone() for t in g]
    tensors = mm.make_grad_tensors(g)
    result, _, norm, factor = norm_of(tensors, 2, 1.0)
    assert not np.isfinite(norm) and np.isnan(factor)
    check(mm.mmtrain_grad_clip(tensors, result), "clip")
    out = [torch.zeros(t.numel(), device="cuda") for t in g]
    check(mm.mmtrain_grad_clip(mm.make_grad_tensors(g, out), result), "clip")
    for t, b, o in zip(g, before, out):
        assert torch.equal(t.view(torch.uint8), b.view(torch.uint8)) and torch.equal(torch.nan_to_num(o), torch.nan_to_num(b.float()))
    state = [torch.randn(1000, device="cuda") for _ in range(3)]
    kept, param = [t.clone() for t in state], torch.full((1000,), 8.0, dtype=torch.bfloat16, device="cuda")
    for zero in (False, True):
        check(mm.mmtrain_adam_step_clipped(mm.make_adam_desc(1e-2, zero_grad=zero), 1000, state[0], g[0], state[1], state[2], param, mm.BF16, result), "adam")
        assert all(torch.equal(a, b) for a, b in zip(state, kept)) and torch.all(param == 8.0)
        assert torch.all(g[0] == 0) if zero else torch.equal(g[0].view(torch.uint8), before[0].view(torch.uint8))


@pytest.mark.parametrize("n", [1, 5, 1027, 100001])
@pytest.mark.parametrize("zero", [False, True])
@pytest.mark.parametrize("max_norm", [0.25, 1e9])
def test_clipped_adam_is_adam_on_clipped_gradients(n, zero, max_norm):
    g = grads_of([n], (mm.F32,), seed=n)[0]
    state = [t.abs() if i == 2 else t for i, t in enumerate(grads_of([n] * 3, (mm.F32,), 0.1, seed=n + 1))]
    other = [t.clone() for t in state]
    result, _, _, factor = norm_of(mm.make_grad_tensors([g]), 1, max_norm)
    p, q = (torch.empty(n, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    # grad_scale times the factor as one fp32 number, which is what the description of the unclipped step can carry
    scale = float(np.float32(0.5) * np.float32(factor))
    check(mm.mmtrain_adam_step(mm.make_adam_desc(1e-2, weight_decay=0.1, grad_scale=scale, step=3), n, other[0], g.clone(), other[1], other[2], q, mm.BF16), "adam")
    check(mm.mmtrain_adam_step_clipped(mm.make_adam_desc(1e-2, weight_decay=0.1, grad_scale=0.5, step=3, zero_grad=zero), n, state[0], g, state[1], state[2], p,
                                       mm.BF16, result), "adam")
    assert all(torch.equal(a, b) for a, b in zip(state, other)) and torch.equal(p, q)
    assert bool(torch.all(g == 0)) == zero


@pytest.mark.parametrize("from_dtype,to_dtype", [(mm.BF16, mm.F32), (mm.F32, mm.BF16), (mm.F32, None)])
def test_grad_clip_of_more_than_the_caches_hold(from_dtype, to_dtype):
    # 384 MB and more are written: streamed
    n = (100 << 20) + 5 if to_dtype != mm.BF16 else (200 << 20) + 5
    g = torch.randn(n, device="cuda").to(torch_dtype(from_dtype))
    out = None if to_dtype is None else torch.full((n + 8,), 7.0, dtype=torch_dtype(to_dtype), device="cuda")
    before = g.clone()
    tensors = mm.make_grad_tensors([g, g[:0]], None if out is None else [out[:n], out[n:n]])
    result, _, norm, factor = norm_of(tensors, 2, 1.0)
    assert np.isclose(norm, float(torch.linalg.vector_norm(before, dtype=torch.float64)), rtol=1e-6)
    check(mm.mmtrain_grad_clip(tensors, result), "clip")
    got = g if out is None else out[:n]
    want = (before.float() * result.view(torch.float32)[3]).to(got.dtype)      # one fp32 product, one rounding
    assert torch.equal(got, want) and (out is None or torch.all(out[n:] == 7.0))


@pytest.mark.parametrize("n", [300, 9000])
def test_grad_clip_takes_lists_in_any_order(n):
    # parts of two flat buffers that share nothing, neighbours without a gap, shuffled: more than are sorted at a time, and fewer
    rng = np.random.default_rng(n)
    sizes = 8 * rng.integers(0, 6, size=n)
    at = np.concatenate([[0], np.cumsum(sizes)])
    flat = dev(rng.standard_normal(at[-1]), mm.F32)
    before, out = flat.clone(), torch.zeros_like(flat)
    order = rng.permutation(n)
    parts = [slice(int(at[i]), int(at[i + 1])) for i in order]
    elsewhere = [bool(i % 2) for i in order]
    tensors = mm.make_grad_tensors([flat[p] for p in parts], [out[p] if e else None for p, e in zip(parts, elsewhere)])
    result, *_, factor = norm_of(tensors, n, 1.0)
    check(mm.mmtrain_grad_clip(tensors, result), "clip")
    want = before * result.view(torch.float32)[3]
    for p, e in zip(parts, elsewhere):
        assert torch.equal((out if e else flat)[p], want[p]) and (not e or torch.equal(flat[p], before[p]))
