"""Embedding, norms of queries and keys, cross attention on the CPU: the oracle against independent definitions (autograd, differences), and
what the entry points refuse (all argument checks run before any HIP call)."""
import numpy as np
import pytest
import torch

from oracle import attention_ops_oracle as ao
from oracle import operators_oracle as oo
from paper_2408_04275_amd import binding as mm

FAKE = 0x100000         # a 256-aligned address that no error path touches
NAN, INF = float("nan"), float("inf")
BAD, UNSUP, SEG, WS = mm.ERR_INVALID_ARG, mm.ERR_UNSUPPORTED, mm.ERR_BAD_SEGMENTS, mm.ERR_WORKSPACE


# ---- the oracle ------------------------------------------------------------------------------------------------------
def test_oracle_embedding():
    rng = np.random.default_rng(0)
    table, features = rng.standard_normal((5, 8)), rng.standard_normal((3, 8))
    ids = [4, -1, 0, 5, -3, 4, -4, -2 ** 31, 2 ** 31 - 1]
    y = ao.embed_fwd(ids, table, features, 2.0)
    want = [2 * table[4], features[0], 2 * table[0], 0 * table[0], features[2], 2 * table[4]] + [0 * table[0]] * 3
    assert np.array_equal(y, np.stack(want))
    dy = rng.standard_normal(y.shape)
    (dt, df), (mt, _) = ao.embed_bwd(ids, dy, 5, 3, 2.0)
    for source, grad in ((table, dt), (features, df)):                # linear: a difference is the gradient
        step = rng.standard_normal(source.shape)
        parts = [table + step if source is table else table, features + step if source is features else features]
        assert np.isclose(np.sum((ao.embed_fwd(ids, *parts, 2.0) - y) * dy), np.sum(step * grad), rtol=1e-12)
    assert np.all(mt >= np.abs(dt) - 1e-12)


@pytest.mark.parametrize("norm", ["rms", "layer"])
@pytest.mark.parametrize("layout", [None, "half", "interleaved"])
def test_oracle_qk_norm_gradients_are_those_of_autograd(norm, layout):
    rng = np.random.default_rng(1)
    T, nq, nk, d, rot = 4, 3, 2, 16, 8
    x, dy = rng.standard_normal((T, nq + nk, d)), rng.standard_normal((T, nq + nk, d))
    w = {n + k: rng.standard_normal(d) for n in ("q", "k") for k in (("_w", "_b") if norm == "layer" else ("_w",))}
    theta = oo.rope_frequencies(rot, 100.0)
    turn = None if layout is None else ([0, 5, 1, 70], theta, layout, 1.25)
    y, _ = ao.qk_norm_fwd(x, w, nq, nk, norm, 1e-3, turn)
    tx = torch.from_numpy(x).requires_grad_(True)
    tw = {k: torch.from_numpy(v).requires_grad_(True) for k, v in w.items()}
    parts = []
    for name, part in (("q", tx[:, :nq]), ("k", tx[:, nq:])):
        if norm == "layer":
            parts.append(torch.nn.functional.layer_norm(part, (d,), tw[name + "_w"], tw[name + "_b"], 1e-3))
        else:
            parts.append(part / torch.sqrt(part.pow(2).mean(-1, keepdim=True) + 1e-3) * tw[name + "_w"])
    n = torch.cat(parts, 1)
    if layout is not None:
        z = torch.polar(torch.full((T, 1, rot // 2), 1.25, dtype=torch.float64), torch.tensor(turn[0])[:, None, None] * torch.from_numpy(theta))
        pair = torch.complex(n[..., :4], n[..., 4:8]) if layout == "half" else torch.view_as_complex(n[..., :rot].reshape(T, nq + nk, 4, 2))
        pair = pair * z
        n = torch.cat([torch.cat([pair.real, pair.imag], -1) if layout == "half" else torch.view_as_real(pair).reshape(T, nq + nk, rot), n[..., rot:]], -1)
    assert np.allclose(n.detach().numpy(), y, rtol=1e-10, atol=1e-12)
    n.backward(torch.from_numpy(dy))
    out, mag = ao.qk_norm_bwd(x, dy, w, nq, nk, norm, 1e-3, turn)
    assert np.allclose(tx.grad.numpy(), out["dx"], rtol=1e-9, atol=1e-11)
    assert set(out) == {"dx", *w}
    for k, t in tw.items():
        assert np.allclose(t.grad.numpy(), out[k], rtol=1e-9, atol=1e-11) and np.all(mag[k] >= np.abs(out[k]) - 1e-9)


def test_oracle_cross_attention_is_a_masked_softmax_with_its_gradients():
    rng = np.random.default_rng(2)
    cu, begin, end, Tk = [0, 3, 4, 9, 11], [0, 2, 2, 2], [5, 2, 9, 9], 11
    nh, nk, d, scale = 4, 2, 8, 0.4
    q, k, v, do = (torch.from_numpy(rng.standard_normal(s)).requires_grad_(True) for s in ((11, nh, d), (Tk, nk, d), (Tk, nk, d), (11, nh, d)))
    seen = torch.zeros(11, Tk, dtype=torch.bool)
    for s in range(4):
        seen[cu[s]:cu[s + 1], begin[s]:end[s]] = True
    scores = torch.einsum("thd,jhd->htj", q, k.repeat_interleave(2, 1)) * scale
    scores = scores.masked_fill(~seen, -INF)
    p = torch.softmax(scores, -1).masked_fill(~seen.any(1)[None, :, None], 0.0)
    o = torch.einsum("htj,jhd->thd", p, v.repeat_interleave(2, 1))
    arrays = [t.detach().numpy() for t in (q, k, v)]
    (ro, rl), (mag, stored, _) = ao.cross_fwd(*arrays, cu, begin, end, scale)
    assert np.allclose(ro, o.detach().numpy(), atol=1e-12) and np.allclose(rl, torch.logsumexp(scores, -1).detach().numpy())
    assert np.all(rl[:, 3] == -np.inf) and np.all(stored >= np.abs(ro) - 1e-12) and np.all(mag >= stored)
    # by hand, so that the row without keys has a gradient of zero instead of NaN
    live = [t for t in range(11) if t != 3]
    o = torch.einsum("htj,jhd->thd", torch.softmax(scores[:, live], -1), v.repeat_interleave(2, 1))
    g = torch.autograd.grad(o, (q, k, v), do.detach()[live])
    out, _, _ = ao.cross_bwd(*arrays, ro, rl, do.detach().numpy(), cu, begin, end, scale)
    for name, t in zip(("dq", "dk", "dv"), g):
        assert np.allclose(out[name], t.numpy(), atol=1e-11), name
    # and against a difference
    step = rng.standard_normal(arrays[1].shape)
    f = lambda e: np.sum(ao.cross_fwd(arrays[0], arrays[1] + e * step, arrays[2], cu, begin, end, scale)[0][0] * do.detach().numpy())  # noqa: E731
    assert np.isclose((f(1e-5) - f(-1e-5)) / 2e-5, np.sum(out["dk"] * step), rtol=1e-7)


# ---- refusals --------------------------------------------------------------------------------------------------------
def embed_calls(status, T=4, ids=FAKE, table=FAKE, features=FAKE, y=2 * FAKE, dy=FAKE, d_table=2 * FAKE, d_features=3 * FAKE, flags=0, ws=4 * FAKE, wsb=1 << 30,
                both=True, fwd=True, **kw):
    d = mm.make_embed_desc(**{**dict(dtype=mm.BF16, hidden=64, vocab=100, n_features=7, scale=1.0), **kw})
    if "struct_size" in kw:
        d.struct_size = kw["struct_size"]
    if fwd:
        assert mm.mmtrain_embed_fwd(d, T, ids, table, features, y, 0) == status
    if both or not fwd:
        assert mm.mmtrain_embed_bwd(d, T, ids, dy, d_table, d_features, flags, ws, wsb, 0) == status


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=7), BAD), (dict(hidden=0), BAD), (dict(hidden=-8), BAD), (dict(vocab=0), BAD), (dict(n_features=-1), BAD), (dict(scale=NAN), BAD),
    (dict(scale=INF), BAD), (dict(hidden=60), UNSUP), (dict(hidden=65544), UNSUP), (dict(vocab=(1 << 30) + 1), UNSUP), (dict(vocab=2 ** 31 - 1, n_features=2 ** 31 - 1), UNSUP),
    (dict(T=-1), BAD), (dict(T=(1 << 30) + 1), UNSUP), (dict(ids=None), BAD), (dict(ids=FAKE + 2), BAD)])
def test_embed_refuses(kw, status):
    embed_calls(status, **kw)
    if not set(kw) & {"T", "ids"}:
        d = mm.make_embed_desc(**{**dict(dtype=mm.BF16, hidden=64, vocab=100), **kw})
        assert mm.mmtrain_embed_workspace_bytes(d, 4) == 0


def test_embed_refuses_tensors():
    for kw in (dict(table=None), dict(features=None), dict(y=None), dict(table=FAKE + 8), dict(y=FAKE), dict(n_features=0)):
        embed_calls(BAD, both=False, **kw)
    for kw in (dict(dy=None), dict(dy=FAKE + 4), dict(d_table=FAKE), dict(d_features=2 * FAKE), dict(flags=4), dict(n_features=0), dict(ws=4 * FAKE + 128)):
        embed_calls(BAD, fwd=False, **kw)
    for kw in (dict(ws=None), dict(wsb=16)):
        embed_calls(WS, fwd=False, **kw)
    d = mm.make_embed_desc(mm.BF16, 64, 100, 7)
    d.struct_size = 4
    assert mm.mmtrain_embed_fwd(d, 4, FAKE, FAKE, FAKE, 2 * FAKE, 0) == BAD and mm.mmtrain_embed_fwd(None, 4, FAKE, FAKE, FAKE, 2 * FAKE, 0) == BAD
    d.struct_size += 20
    assert mm.mmtrain_embed_fwd(d, 0, None, None, None, None, 0) == mm.OK
    assert mm.mmtrain_embed_bwd(d, 4, FAKE, FAKE, None, None, 0, FAKE, 1 << 30, 0) == mm.OK             # nothing asked for
    sizes = [mm.mmtrain_embed_workspace_bytes(d, T) for T in (0, 1, 7, 100, 5000, 16384, 16385, 20000, 100000, 1 << 20, 1 << 26)]
    assert sizes == sorted(sizes) and sizes[0] > 0 and mm.mmtrain_embed_workspace_bytes(d, -1) == 0


QK = dict(dtype=mm.BF16, n_q_heads=4, n_k_heads=2, head_dim=64, norm=mm.NORM_RMS, eps=1e-6)
W_RMS = mm.QkNormWeights(FAKE, None, FAKE, None)


def qk_fwd(desc=None, rope=None, T=4, batch=None, positions=FAKE, weights=W_RMS, x=FAKE, ld_x=512, y=2 * FAKE, ld_y=384, **kw):
    d = mm.make_qk_norm_desc(**{**QK, **kw}) if desc is None else desc
    return mm.mmtrain_qk_norm_rope_fwd(d, rope, T, batch, positions, weights, x, ld_x, y, ld_y, 0)


def qk_bwd(rope=None, T=4, batch=None, positions=FAKE, weights=W_RMS, x=FAKE, ld_x=512, dy=2 * FAKE, ld_dy=384, dx=3 * FAKE, ld_dx=384,
           grads=mm.QkNormGrads(FAKE, None, FAKE, None), flags=0, ws=4 * FAKE, wsb=1 << 30, **kw):
    return mm.mmtrain_qk_norm_rope_bwd(mm.make_qk_norm_desc(**{**QK, **kw}), rope, T, batch, positions, weights, x, ld_x, dy, ld_dy, dx, ld_dx, grads, flags,
                                       ws, wsb, 0)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=3), BAD), (dict(n_q_heads=-1), BAD), (dict(n_q_heads=0, n_k_heads=0), BAD), (dict(head_dim=0), BAD), (dict(norm=mm.NORM_NONE), BAD), (dict(norm=3), BAD),
    (dict(eps=0.0), BAD), (dict(eps=NAN), BAD), (dict(head_dim=60), UNSUP), (dict(head_dim=264), UNSUP), (dict(n_q_heads=65537), UNSUP),
    (dict(n_q_heads=65000, n_k_heads=1000), UNSUP), (dict(T=-1), BAD), (dict(T=(1 << 30) + 1), UNSUP), (dict(weights=None), BAD),
    (dict(weights=mm.QkNormWeights(FAKE, None, None, None)), BAD), (dict(weights=mm.QkNormWeights(FAKE, FAKE, FAKE, None)), BAD),
    (dict(norm=mm.NORM_LAYER), BAD), (dict(n_q_heads=0), BAD), (dict(weights=mm.QkNormWeights(FAKE + 8, None, FAKE, None)), BAD), (dict(x=None), BAD), (dict(x=FAKE + 8), BAD),
    (dict(ld_x=376), BAD), (dict(ld_x=388), UNSUP),
    (dict(rope=mm.make_rope_desc(mm.F32, 6, 64)), BAD), (dict(rope=mm.make_rope_desc(mm.BF16, 5, 64)), BAD), (dict(rope=mm.make_rope_desc(mm.BF16, 6, 128)), BAD),
    (dict(rope=mm.make_rope_desc(mm.BF16, 6, 64, 30)), UNSUP), (dict(rope=mm.make_rope_desc(mm.BF16, 6, 64, 31)), UNSUP), (dict(rope=mm.make_rope_desc(mm.BF16, 6, 64, base=1.0)), BAD),
    (dict(rope=mm.make_rope_desc(mm.BF16, 6, 64), positions=None), BAD), (dict(rope=mm.make_rope_desc(mm.BF16, 6, 64), positions=FAKE + 2), BAD),
    (dict(rope=mm.make_rope_desc(mm.BF16, 6, 64), batch=mm.PackedBatch(np.array([0, 4]), cu_dev=FAKE)), BAD),
    (dict(rope=mm.make_rope_desc(mm.BF16, 6, 64), positions=None, batch=mm.PackedBatch(np.array([0, 5]), cu_dev=FAKE)), SEG)])
def test_qk_norm_refuses(kw, status):
    assert qk_fwd(**kw) == status
    assert qk_bwd(**kw) == status


def test_qk_norm_refuses_tensors():
    for kw in (dict(y=None), dict(y=FAKE), dict(y=2 * FAKE + 4), dict(ld_y=376)):
        assert qk_fwd(**kw) == BAD, kw
    assert qk_fwd(ld_y=388) == UNSUP and qk_fwd(T=0, x=None, y=None) == mm.OK
    for kw in (dict(dy=None), dict(dy=2 * FAKE + 8), dict(ld_dy=300), dict(ld_dx=300), dict(dx=FAKE, ld_dx=512), dict(dx=2 * FAKE, ld_dx=392), dict(flags=4),
               dict(grads=mm.QkNormGrads(FAKE, FAKE, None, None)), dict(grads=mm.QkNormGrads(FAKE + 4, None, None, None)), dict(ws=FAKE + 128)):
        assert qk_bwd(**kw) == BAD, kw
    assert qk_bwd(ld_dx=388) == UNSUP and qk_bwd(ws=None) == WS and qk_bwd(wsb=256) == WS
    assert qk_bwd(dx=None, grads=None, ws=None) == mm.OK and qk_bwd(T=0, x=None, dy=None, dx=None, grads=None, ws=None) == mm.OK
    only_k = dict(n_q_heads=0, weights=mm.QkNormWeights(None, None, FAKE, None))
    assert qk_bwd(grads=mm.QkNormGrads(FAKE, None, None, None), **only_k) == BAD
    d = mm.make_qk_norm_desc(**QK)
    sizes = [mm.mmtrain_qk_norm_rope_workspace_bytes(d, T) for T in (0, 1, 5, 1000, 1025, 10000, 1 << 24)]
    assert sizes == sorted(sizes) and sizes[0] > 0 and mm.mmtrain_qk_norm_rope_workspace_bytes(d, -1) == 0
    d.struct_size = 8
    assert qk_fwd(desc=d) == BAD and mm.mmtrain_qk_norm_rope_workspace_bytes(d, 4) == 0 and mm.mmtrain_qk_norm_rope_workspace_bytes(None, 4) == 0


CROSS = dict(dtype=mm.BF16, n_heads=4, n_kv_heads=2, head_dim=64)


def cross_batch(cu=(0, 3, 5), begin=(0, 4), end=(4, 9), Tk=9, q_tokens=None, dev=FAKE):
    return mm.CrossBatch(np.array(cu), np.array(begin), np.array(end), Tk, dev, dev, dev, q_tokens)


def cross_status(batch=None, tensors=None, grads=None, ws=5 * FAKE, wsb=1 << 40, no_batch=False, struct_size=None, **kw):
    """(forward, backward)"""
    d = mm.make_cross_attn_desc(**{**CROSS, **kw})
    if struct_size is not None:
        d.struct_size = struct_size
    b = None if no_batch else cross_batch() if batch is None else batch
    t = mm.CrossAttnTensors(**{**dict(q=FAKE, ld_q=256, k=2 * FAKE, ld_k=128, v=3 * FAKE, ld_v=128, o=4 * FAKE, ld_o=256, lse=FAKE), **(tensors or {})})
    g = mm.CrossAttnGrads(**{**dict(d_o=6 * FAKE, ld_do=256, d_q=7 * FAKE, ld_dq=256, d_k=8 * FAKE, ld_dk=128, d_v=9 * FAKE, ld_dv=128), **(grads or {})})
    return mm.mmtrain_cross_attn_fwd(d, b, t, ws, wsb, 0), mm.mmtrain_cross_attn_bwd(d, b, t, g, ws, wsb, 0)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=2), BAD), (dict(n_heads=0), BAD), (dict(n_kv_heads=0), BAD), (dict(head_dim=-16), BAD), (dict(softmax_scale=-1.0), BAD), (dict(softmax_scale=NAN), BAD),
    (dict(softmax_scale=INF), BAD), (dict(struct_size=8), BAD), (dict(head_dim=72), UNSUP), (dict(head_dim=144), UNSUP), (dict(n_kv_heads=3), UNSUP),
    (dict(n_heads=8192, n_kv_heads=8192), UNSUP), (dict(no_batch=True), BAD),
    (dict(batch=cross_batch(cu=(1, 3, 5))), SEG), (dict(batch=cross_batch(cu=(0, 6, 5))), SEG), (dict(batch=cross_batch(q_tokens=6)), SEG),
    (dict(batch=cross_batch(begin=(-1, 4))), SEG), (dict(batch=cross_batch(begin=(5, 4))), SEG), (dict(batch=cross_batch(end=(4, 10))), SEG),
    (dict(batch=cross_batch(dev=None)), BAD),
    (dict(tensors=dict(q=None)), BAD), (dict(tensors=dict(k=FAKE + 8)), BAD), (dict(tensors=dict(v=None)), BAD), (dict(tensors=dict(o=None)), BAD),
    (dict(tensors=dict(ld_q=248)), BAD), (dict(tensors=dict(ld_k=120)), BAD), (dict(tensors=dict(ld_q=260)), UNSUP), (dict(tensors=dict(ld_v=1 << 24)), UNSUP),
    (dict(tensors=dict(lse=FAKE + 4)), BAD), (dict(ws=None), WS), (dict(wsb=8), WS), (dict(ws=5 * FAKE + 64), BAD)])
def test_cross_attention_refuses(kw, status):
    assert cross_status(**kw) == (status, status)
    if not set(kw) & {"tensors", "ws", "wsb", "struct_size", "no_batch"}:
        b = kw.pop("batch", None) or cross_batch()
        assert mm.mmtrain_cross_attn_workspace_bytes(mm.make_cross_attn_desc(**{**CROSS, **kw}), b, 0) == 0


def test_cross_attention_refuses_more():
    assert cross_status(tensors=dict(o=FAKE))[0] == BAD
    for g in (dict(d_o=None), dict(d_o=FAKE + 2), dict(d_k=None), dict(d_v=None), dict(ld_dq=8), dict(d_q=FAKE), dict(d_k=2 * FAKE), dict(d_v=8 * FAKE), dict(d_q=6 * FAKE)):
        assert cross_status(grads=g)[1] == BAD, g
    assert cross_status(grads=dict(ld_dk=132))[1] == UNSUP
    assert cross_status(tensors=dict(lse=None))[1] == BAD
    # the runs that see a key have to follow one another where keys get gradients; a run that sees nothing may stand anywhere
    swapped = cross_batch(begin=(4, 0), end=(9, 4))
    assert cross_status(batch=swapped)[1] == SEG
    assert cross_status(batch=cross_batch(begin=(0, 2), end=(9, 8)))[1] == SEG
    many = mm.CrossBatch(np.zeros(65538), np.zeros(65537), np.zeros(65537), 0, FAKE, FAKE, FAKE)
    assert cross_status(batch=many) == (UNSUP, UNSUP)
    assert mm.mmtrain_cross_attn_bwd(mm.make_cross_attn_desc(**CROSS), cross_batch(), mm.CrossAttnTensors(), None, FAKE, 1 << 30, 0) == BAD
    assert mm.mmtrain_cross_attn_fwd(mm.make_cross_attn_desc(**CROSS), cross_batch(), None, FAKE, 1 << 30, 0) == BAD
    # nothing to do
    empty = mm.CrossBatch(np.array([0]), np.zeros(0), np.zeros(0), 0)
    nothing = mm.CrossAttnTensors()
    assert mm.mmtrain_cross_attn_fwd(mm.make_cross_attn_desc(**CROSS), empty, nothing, FAKE, 1 << 30, 0) == mm.OK
    assert mm.mmtrain_cross_attn_bwd(mm.make_cross_attn_desc(**CROSS), empty, nothing, mm.CrossAttnGrads(), FAKE, 1 << 30, 0) == mm.OK
    d = mm.make_cross_attn_desc(**CROSS)
    assert mm.mmtrain_cross_attn_workspace_bytes(d, cross_batch(), 1) > 0 and mm.mmtrain_cross_attn_workspace_bytes(None, cross_batch(), 1) == 0
    assert mm.mmtrain_cross_attn_workspace_bytes(d, empty, 0) > 0


@pytest.mark.parametrize("dtype,tokens,kv_tokens,nh,nkv,S,status", [
    (mm.BF16, 1 << 22, 9, 64, 64, 1, UNSUP), (mm.BF16, (1 << 22) - 64, 9, 64, 64, 1, mm.OK), (mm.F32, 1 << 21, 9, 64, 64, 1, UNSUP), (mm.F32, (1 << 21) - 64, 9, 64, 64, 1, mm.OK),
    (mm.BF16, 8, 1 << 30, 1, 1, 1, UNSUP), (mm.BF16, 8, (1 << 30) - 1024, 1, 1, 1, mm.OK), (mm.F32, 8, 1 << 27, 1, 1, 1, UNSUP), (mm.BF16, 65536, 9, 128, 128, 65536, UNSUP),
    (mm.BF16, 65536, 9, 32, 32, 65536, mm.OK)])
def test_cross_attention_calls_that_no_launch_holds(dtype, tokens, kv_tokens, nh, nkv, S, status):
    """2^32 threads; the workspace's size is 0 where a call would be refused."""
    b = mm.CrossBatch(np.linspace(0, tokens, S + 1).astype(np.int64), np.zeros(S, np.int64), np.full(S, 9), kv_tokens, FAKE, FAKE, FAKE)
    d = mm.make_cross_attn_desc(dtype, nh, nkv, 16)
    for back in (0, 1):
        assert (mm.mmtrain_cross_attn_workspace_bytes(d, b, back) > 0) == (status == mm.OK)
    if status != mm.OK:
        t = mm.CrossAttnTensors(q=FAKE, ld_q=nh * 16, k=2 * FAKE, ld_k=nkv * 16, v=3 * FAKE, ld_v=nkv * 16, o=4 * FAKE, ld_o=nh * 16, lse=FAKE)
        g = mm.CrossAttnGrads(d_o=6 * FAKE, ld_do=nh * 16, d_q=7 * FAKE, ld_dq=nh * 16, d_k=8 * FAKE, ld_dk=nkv * 16, d_v=9 * FAKE, ld_dv=nkv * 16)
        assert mm.mmtrain_cross_attn_fwd(d, b, t, 5 * FAKE, 1 << 40, 0) == status and mm.mmtrain_cross_attn_bwd(d, b, t, g, 5 * FAKE, 1 << 40, 0) == status
