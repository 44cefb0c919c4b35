"""Embedding, norms of queries and keys with rotation, and cross attention on the GPU, against oracle/attention_ops_oracle.py in 64 bits.

Tolerances.  An output is off by its rounding, finfo(dtype).eps / 2 of its value, and by the rounding errors of the fp32 evaluation: at most
k 2^-24 times the sum of the absolute values of the terms (the oracle's `mag`), k counting the roundings that one term passes through:
  embedding: forward a product and nothing else, k = 1.  A row's gradient: additions of the tokens of a chunk, then of the chunks' sums: up to
    16 + T / 2048 and 2048, in the cases here at most T and never more than the tokens of that row.
  norms of heads: a head's sum, 16 additions in a thread and 6 across threads, twice where a mean is subtracted, the root and its reciprocal (3),
    product with gain and bias (3), rotation (7, see test_gpu_operators.py): k = 64; backward a second pair of sums and the products in front of
    them: 128.  Gains' gradients: on top of that the tokens and heads that a thread adds up, and the partial sums: 128 + 64 + T heads / 256.
  cross attention: a score: d products and additions, the scale and the exponent's (8); d + 16 in all, which the oracle's mag carries to
    every result; sums over keys (or tokens and heads) of n terms: n additions.  k = d + n + 64.
  In bf16 the probabilities and their gradients are operands of matrix products and rounded to bf16: half a step, 2^-8, of the oracle's `stored`.
The tolerances on single elements add up all errors with the same sign.  Those of bf16 are independent and mostly cancel: a result whose errors
come from up to three roundings has an l2 error of sqrt(3) eps / 2 / sqrt(3) at most, the roundings being spread evenly over half a step: below
eps / 2 of its norm."""
import numpy as np
import pytest
import torch

from oracle import attention_ops_oracle as ao
from oracle import operators_oracle as oo
from paper_2408_04275_amd import binding as mm
from paper_2408_04275_amd.harness import check, torch_dtype
from test_gpu_operators import LAYOUTS, SCALINGS, U, close, dev, host

pytestmark = pytest.mark.gpu

HALF = {mm.BF16: 2.0 ** -8, mm.F32: 2.0 ** -24}
NORMS = {"rms": mm.NORM_RMS, "layer": mm.NORM_LAYER}


# A probability below fp32's (and bf16's) smallest normal number, 2^-126, may come out as zero.  It is then off by less than 2^-126, and a result by
# that times what it multiplies: in the cases here |dP - D| < 2^9 (64 to 128 terms of at most 4 x 4, twice) times softmax_scale |q| or |k| < 2^7 at
# most, for each of the result's fewer than k terms.
UNDERFLOW = 2.0 ** -126 * 2.0 ** 16


def near(name, got, ref, mag, k, stored, dtype, out_dtype=None):
    """Every element by its own bound, and the whole by its norm."""
    bf16 = dtype == mm.BF16
    close(name, got, ref, mag, k, dtype if out_dtype is None else out_dtype, (HALF[mm.BF16] * 1.01 * stored if bf16 else 0.0) + k * UNDERFLOW)
    got = host(got).reshape(np.shape(ref))
    norm = np.linalg.norm(ref)
    if bf16 and norm > 0:
        assert np.linalg.norm(got - ref) <= HALF[mm.BF16] * norm, f"{name}: l2 error {np.linalg.norm(got - ref) / norm:.2e}"


# ---- embedding -------------------------------------------------------------------------------------------------------
def embed_case(dtype, T, H, vocab, features, ids=None, scale=1.5, main=None, accumulate=False, seed=0, want=("table", "features")):
    rng = np.random.default_rng(seed)
    if ids is None:
        ids = rng.integers(-features - 2, vocab + 2, T)
        ids[rng.random(T) < 0.3] = rng.integers(0, vocab)              # one id often
    ids = np.asarray(ids, np.int64)
    dids = torch.from_numpy(ids.astype(np.int32)).to("cuda") if T else torch.empty(1, dtype=torch.int32, device="cuda")
    desc = mm.make_embed_desc(dtype, H, vocab, features, scale)
    table, feats = dev(rng.standard_normal((vocab, H)), dtype), dev(rng.standard_normal((features, H)), dtype) if features else None
    y = torch.full((T + 1, H), 7.0, dtype=torch_dtype(dtype), device="cuda")
    check(mm.mmtrain_embed_fwd(desc, T, dids, table, feats, y), "embed_fwd")
    ref = ao.embed_fwd(ids, host(table), None if feats is None else host(feats), np.float32(scale))
    close("y", y[:T], ref, np.abs(ref), 1, dtype)
    assert torch.all(y[T] == 7.0)
    dy = dev(rng.standard_normal((T, H)), dtype)
    gdt = mm.F32 if main or dtype == mm.F32 else mm.BF16
    before = dev(rng.standard_normal((vocab, H)), gdt)
    d_table = before.clone() if "table" in want else None
    d_feats = torch.full((features, H), float("nan"), dtype=torch_dtype(dtype), device="cuda") if features and "features" in want else None
    wsb = mm.mmtrain_embed_workspace_bytes(desc, T)
    ws = torch.full((wsb,), 0xA5, dtype=torch.uint8, device="cuda")
    flags = (mm.BWD_WGRAD_F32 if main else 0) | (mm.BWD_ACCUMULATE_WGRAD if accumulate else 0)
    args = lambda: mm.mmtrain_embed_bwd(desc, T, dids, dy, d_table, d_feats, flags, ws, wsb)  # noqa: E731
    check(args(), "embed_bwd")
    torch.cuda.synchronize()
    (rt, rf), (mt, mf) = ao.embed_bwd(ids, host(dy), vocab, features, np.float32(scale))
    count = np.bincount(ao.embed_source(ids, vocab, features) + 1, minlength=vocab + features + 1)[1:]
    if d_table is not None:
        add = host(before) if accumulate else 0.0
        close("d_table", d_table, rt + add, mt + np.abs(add), count[:vocab, None] + 3, gdt)
        if accumulate:                                                 # rows that nobody names keep their bits
            idle = torch.from_numpy(count[:vocab] == 0).to("cuda")
            assert torch.equal(d_table[idle], before[idle])
    if d_feats is not None:
        close("d_features", d_feats, rf, mf, count[vocab:, None] + 1, dtype)
    first = [t.clone() for t in (d_table, d_feats) if t is not None]
    if d_table is not None:
        d_table.copy_(before)
    ws.fill_(0x5A)
    check(args(), "embed_bwd")
    assert all(torch.equal(a, b) for a, b in zip(first, [t for t in (d_table, d_feats) if t is not None]))      # repeats bit for bit


@pytest.mark.parametrize("dtype", [mm.BF16, mm.F32])
@pytest.mark.parametrize("T", [1, 2, 31, 64, 257, 1031, 4100])
def test_embed_lengths(dtype, T):
    embed_case(dtype, T, 64, 50, 9, seed=T)
    embed_case(dtype, T, 40, 3000, 100, main=True, accumulate=True, seed=T + 1)


@pytest.mark.parametrize("H", [8, 16, 24, 1024, 1280, 2056, 4096, 8192, 8200])
def test_embed_widths(H):
    embed_case(mm.BF16, 77, H, 20, 30, seed=H)
    embed_case(mm.BF16, 77, H, 20, 30, main=True, accumulate=True, seed=H)
    embed_case(mm.F32, 50, H, 20, 30, accumulate=True, seed=H)


def test_embed_every_token_the_same():
    for T in (3, 300, 5000):
        embed_case(mm.BF16, T, 64, 10, 0, ids=np.full(T, 7), main=True)
        embed_case(mm.F32, T, 64, 10, 2, ids=np.full(T, -2))


def test_embed_nobody_and_only_padding():
    embed_case(mm.BF16, 40, 64, 10, 3, ids=np.full(40, 10))
    embed_case(mm.BF16, 40, 64, 10, 0, ids=np.array([-1, 10, 2 ** 31 - 1, -2 ** 31] * 10), accumulate=True)
    embed_case(mm.BF16, 0, 64, 10, 3, ids=[])
    embed_case(mm.F32, 0, 64, 10, 3, ids=[], accumulate=True)


def test_embed_one_gradient_at_a_time():
    embed_case(mm.BF16, 500, 64, 40, 30, want=("table",))
    embed_case(mm.BF16, 500, 64, 40, 30, want=("features",))


@pytest.mark.parametrize("T,vocab,features", [(16384, 700, 0), (16385, 131072, 5000), (40000, 300, 20), (70001, 1, 1), (66000, 1 << 24, 3)])
def test_embed_long(T, vocab, features):
    """Long packs, one-row and large vocabularies, by sums that are exact: gradients are small whole numbers."""
    rng = np.random.default_rng(T)
    H = 16
    ids = np.where(rng.random(T) < 0.2, vocab // 2, rng.integers(-features - 1, vocab, T, dtype=np.int64)) if vocab > 1 else rng.integers(-2, 2, T)
    desc = mm.make_embed_desc(mm.BF16, H, vocab, features, 1.0)
    dy = torch.from_numpy(rng.integers(-3, 4, (T, H)).astype(np.float32)).to("cuda", torch.bfloat16)
    d_table = torch.zeros((vocab, H), device="cuda")
    d_feats = torch.zeros((features, H), dtype=torch.bfloat16, device="cuda") if features else None
    wsb = mm.mmtrain_embed_workspace_bytes(desc, T)
    ws = torch.full((wsb,), 0xA5, dtype=torch.uint8, device="cuda")
    dids = torch.from_numpy(ids.astype(np.int32)).to("cuda")
    check(mm.mmtrain_embed_bwd(desc, T, dids, dy, d_table, d_feats, mm.BWD_WGRAD_F32 | mm.BWD_ACCUMULATE_WGRAD, ws, wsb), "embed_bwd")
    src = torch.from_numpy(ao.embed_source(ids, vocab, features)).to("cuda")
    want = torch.zeros((vocab + features + 1, H), device="cuda").index_add_(0, torch.where(src < 0, vocab + features, src), dy.float())
    assert torch.equal(d_table, want[:vocab])
    if features:
        assert torch.equal(d_feats, want[vocab:-1].to(torch.bfloat16))


def test_embed_tables_past_32_bits():
    # a row whose elements stand past 2^31, read and written
    V, H = 300000, 8192
    table = torch.zeros((V, H), dtype=torch.bfloat16, device="cuda")
    rng = np.random.default_rng(3)
    ids = torch.tensor([V - 1, 5, V - 2, V - 1], dtype=torch.int32, device="cuda")
    rows = dev(rng.standard_normal((3, H)), mm.BF16)
    table[V - 1], table[5], table[V - 2] = rows[0], rows[1], rows[2]
    desc = mm.make_embed_desc(mm.BF16, H, V, 0, 1.0)
    y = torch.empty((4, H), dtype=torch.bfloat16, device="cuda")
    check(mm.mmtrain_embed_fwd(desc, 4, ids, table, None, y), "embed_fwd")
    assert torch.equal(y, rows[[0, 1, 2, 0]])
    wsb = mm.mmtrain_embed_workspace_bytes(desc, 4)
    ws = torch.empty(wsb, dtype=torch.uint8, device="cuda")
    table.fill_(3.0)
    check(mm.mmtrain_embed_bwd(desc, 4, ids, y, table, None, 0, ws, wsb), "embed_bwd")
    assert torch.equal(table[5], rows[1]) and torch.equal(table[V - 2], rows[2]) and torch.equal(table[V - 1], (2 * rows[0].float()).to(torch.bfloat16))
    assert float(table.abs().amax(1).gt(0).sum()) == 3


# ---- norms of queries and keys ------------------------------------------------------------------------------------------
def qk_case(dtype, nq, nk, d, rot=0, layout="half", norm="rms", scaling="plain", T=5, cu=None, positions=None, other=0, pad=0, in_place=False, main=False,
            accumulate=False, want=None, seed=0, eps=1e-6, want_dx=True):
    rng = np.random.default_rng(seed)
    n = nq + nk
    ldx, ldy = n * d + other, n * d + pad
    x = dev(rng.standard_normal((T, ldx)) * 1.5 + 0.2, dtype)
    before = x.clone()
    names = [k + s for k, h in (("q", nq), ("k", nk)) if h for s in (("_w", "_b") if norm == "layer" else ("_w",))]
    w = {k: dev(rng.standard_normal(d) * 0.2 + (1.0 if k.endswith("_w") else 0.0), dtype) for k in names}
    desc = mm.make_qk_norm_desc(dtype, nq, nk, d, NORMS[norm], eps)
    rope = turn = batch = p = None
    if rot:
        theta = oo.rope_frequencies(rot, 10000.0, scaling, 4.0, 1.0, 32.0, 4096.0)
        rope = mm.make_rope_desc(dtype, n, d, rot, LAYOUTS[layout], 10000.0, SCALINGS[scaling], 4.0, 1.0, 32.0, 4096.0, 1.25)
        pos = oo.segment_positions(cu) if cu is not None else np.asarray(positions)
        turn = (pos, theta, layout, 1.25)
        batch = mm.PackedBatch.on_device(cu) if cu is not None else None
        p = None if cu is not None else torch.tensor(pos, dtype=torch.int32, device="cuda")
    heads = lambda t: host(t)[:, :n * d].reshape(T, n, d)  # noqa: E731
    hw = {k: host(t) for k, t in w.items()}
    eps32 = float(np.float32(eps))
    ref, mag = ao.qk_norm_fwd(heads(x), hw, nq, nk, norm, eps32, turn)
    y = x.clone() if in_place else torch.full((T, ldy), 7.0, dtype=x.dtype, device="cuda")
    src, ld = (y, ldx) if in_place else (x, ldy)
    cw = mm.make_qk_norm_weights(w)
    check(mm.mmtrain_qk_norm_rope_fwd(desc, rope, T, batch, p, cw, src, ldx, y, ld), "qk_norm_rope_fwd")
    torch.cuda.synchronize()
    close("y", y[:, :n * d], ref.reshape(T, -1), mag.reshape(T, -1), 64, dtype)
    rest = host(y)[:, n * d:]
    assert np.array_equal(rest, host(before)[:, n * d:] if in_place else np.full_like(rest, 7.0))
    assert torch.equal(x, before)
    # backward
    dy = dev(rng.standard_normal((T, ldy)), dtype)
    gdt = mm.F32 if main or dtype == mm.F32 else mm.BF16
    start = {k: dev(rng.standard_normal(d), gdt) for k in (names if want is None else want)}
    grads = {k: t.clone() for k, t in start.items()}
    rout, rmag = ao.qk_norm_bwd(heads(x), heads(dy), hw, nq, nk, norm, eps32, turn)
    wsb = mm.mmtrain_qk_norm_rope_workspace_bytes(desc, T)
    ws = torch.full((wsb,), 0xA5, dtype=torch.uint8, device="cuda")
    flags = (mm.BWD_WGRAD_F32 if main else 0) | (mm.BWD_ACCUMULATE_WGRAD if accumulate else 0)
    dx = None if not want_dx else dy.clone() if in_place else torch.full((T, ldx), 7.0, dtype=x.dtype, device="cuda")
    g_in, ldd = (dx, ldy) if in_place else (dy, ldx)
    run = lambda: mm.mmtrain_qk_norm_rope_bwd(desc, rope, T, batch, p, cw, x, ldx, g_in, ldy, dx, ldd, mm.make_qk_norm_grads(grads), flags, ws, wsb)  # noqa: E731
    check(run(), "qk_norm_rope_bwd")
    torch.cuda.synchronize()
    if dx is not None:
        close("dx", dx[:, :n * d], rout["dx"].reshape(T, -1), rmag["dx"].reshape(T, -1), 128, dtype)
        rest = host(dx)[:, n * d:]
        assert np.array_equal(rest, host(dy)[:, n * d:] if in_place else np.full_like(rest, 7.0))
    for k in grads:
        add = host(start[k]) if accumulate else 0.0
        close(k, grads[k], rout[k] + add, rmag[k] + np.abs(add), 128 + 64 + T * n / 256, gdt)
    if not in_place:
        first = {k: t.clone() for k, t in grads.items()}
        for k in grads:
            grads[k].copy_(start[k])
        ws.fill_(0x5A)
        check(run(), "qk_norm_rope_bwd")
        assert all(torch.equal(first[k], grads[k]) for k in grads)


HEADS = [(4, 2, 64, 64), (3, 1, 128, 128), (2, 2, 80, 80), (5, 2, 80, 40), (1, 1, 128, 32), (2, 1, 96, 24), (3, 2, 8, 8), (2, 0, 256, 252), (0, 3, 256, 256), (1, 1, 24, 4), (33, 7, 16, 12),
         (2, 1, 200, 0), (4, 4, 64, 0), (1, 1, 8, 0), (0, 1, 256, 12)]


@pytest.mark.parametrize("dtype", [mm.BF16, mm.F32])
@pytest.mark.parametrize("norm", ["rms", "layer"])
@pytest.mark.parametrize("nq,nk,d,rot", HEADS)
def test_qk_norm_heads(dtype, norm, nq, nk, d, rot):
    cu = np.array([0, 1, 1, 40, 67], dtype=np.int32)
    for layout in ("half", "interleaved") if rot else ("half",):
        qk_case(dtype, nq, nk, d, rot, layout, norm, T=67, cu=cu, other=2 * d, pad=8, seed=1)
    qk_case(dtype, nq, nk, d, rot, "half", norm, T=9, positions=np.arange(9) * 1000, in_place=True, main=True, accumulate=True, seed=2)


@pytest.mark.parametrize("T", [1, 2, 3, 17, 513, 1031, 4111])
def test_qk_norm_lengths(T):
    cu = np.array([0, T // 3, T // 3, T], dtype=np.int32)
    qk_case(mm.BF16, 8, 2, 128, 128, "half", T=T, cu=cu, main=True, seed=3)
    qk_case(mm.F32, 3, 3, 80, 40, "interleaved", "layer", T=T, positions=np.arange(T)[::-1] * 3, accumulate=True, seed=4)


@pytest.mark.parametrize("scaling", list(SCALINGS))
def test_qk_norm_scaling(scaling):
    pos = [0, 1, 4095, 4096, 131071, 2 ** 20 + 1]
    for layout in LAYOUTS:
        qk_case(mm.F32, 2, 1, 128, 64, layout, "rms", scaling, T=6, positions=pos, seed=5)


def test_qk_norm_some_gradients():
    qk_case(mm.BF16, 4, 2, 64, 64, "half", "layer", T=40, positions=np.arange(40), want=["k_w", "q_b"], main=True, seed=6)
    qk_case(mm.BF16, 4, 2, 64, 64, "half", "layer", T=40, positions=np.arange(40), want=[], seed=7)
    qk_case(mm.BF16, 4, 2, 64, 64, "half", "layer", T=40, positions=np.arange(40), want_dx=False, seed=8)


def test_qk_norm_many_segments_and_long_packs():
    cu = np.concatenate([[0], np.repeat(np.arange(1, 400), 2), [1201]]).astype(np.int32)
    qk_case(mm.BF16, 2, 1, 64, 64, "half", T=1201, cu=cu, seed=9)
    qk_case(mm.F32, 1, 1, 16, 16, "half", T=30011, positions=np.arange(30011), main=True, seed=10)


def test_qk_norm_large_and_tiny_rows():
    """A head of zeros, and heads near the ends of the type's range: sums of squares of 1e15 and of 1e-15 with its epsilon."""
    d, T = 64, 4
    x = torch.zeros((T, 2 * d), device="cuda")
    rng = np.random.default_rng(11)
    base = torch.from_numpy(rng.standard_normal((T, 2 * d)).astype(np.float32)).to("cuda")
    x[1], x[2], x[3] = base[1] * 1e15, base[2] * 1e-15, base[3]
    w = {"q_w": torch.ones(d, device="cuda"), "k_w": torch.ones(d, device="cuda")}
    y = torch.empty_like(x)
    desc = mm.make_qk_norm_desc(mm.F32, 1, 1, d, mm.NORM_RMS, 1e-6)
    check(mm.mmtrain_qk_norm_rope_fwd(desc, None, T, None, None, mm.make_qk_norm_weights(w), x, 2 * d, y, 2 * d), "qk_norm_rope_fwd")
    ref, mag = ao.qk_norm_fwd(host(x).reshape(T, 2, d), {k: host(t) for k, t in w.items()}, 1, 1, "rms", float(np.float32(1e-6)))
    close("y", y, ref.reshape(T, -1), mag.reshape(T, -1), 64, mm.F32)


def test_qk_norm_rows_past_32_bits():
    T, ld, d = 3, (1 << 30) + 8, 64
    x = torch.zeros(2 * ld + 256, dtype=torch.bfloat16, device="cuda")
    rows = dev(np.random.default_rng(12).standard_normal((T, 2 * d)), mm.BF16)
    for t in range(T):
        x[t * ld:t * ld + 2 * d] = rows[t]
    ones = {k: torch.ones(d, dtype=torch.bfloat16, device="cuda") for k in ("q_w", "k_w")}
    w = mm.make_qk_norm_weights(ones)
    desc, pos = mm.make_qk_norm_desc(mm.BF16, 1, 1, d), torch.tensor([1, 2, 3], dtype=torch.int32, device="cuda")
    rope = mm.make_rope_desc(mm.BF16, 2, d)
    check(mm.mmtrain_qk_norm_rope_fwd(desc, rope, T, None, pos, w, x, ld, x, ld), "qk_norm_rope_fwd")
    out = torch.empty_like(rows)
    check(mm.mmtrain_qk_norm_rope_fwd(desc, rope, T, None, pos, w, rows, 2 * d, out, 2 * d), "qk_norm_rope_fwd")
    assert all(torch.equal(x[t * ld:t * ld + 2 * d], out[t]) for t in range(T))


# ---- cross attention ------------------------------------------------------------------------------------------------------
def runs(lq, lk, pattern="own", group=4, tail=0):
    """cu, begin, end, key rows.  own: run s sees piece s; shared: `group` runs see a piece; previous: the pieces so far of the group."""
    cu, ck = np.concatenate([[0], np.cumsum(lq)]).astype(np.int32), np.concatenate([[0], np.cumsum(lk)]).astype(np.int32)
    s = np.arange(len(lq))
    if pattern == "own":
        begin, end = ck[s], ck[s + 1]
    elif pattern == "shared":
        begin, end = ck[s // group], ck[s // group + 1]
    else:
        begin, end = ck[s // group * group], ck[s + 1]
    return cu, begin.astype(np.int32), end.astype(np.int32), int(ck[-1]) + tail


def flat(a):
    return a.reshape(len(a), a.shape[1] * a.shape[2])


class Cross:
    """Tensors of a case, in rows wider than they have to be, and its calls."""

    def __init__(self, dtype, nh, nkv, d, shape, scale=0.0, pad=0, std=1.0, seed=0, packed=True):
        self.dtype, self.nh, self.nkv, self.d = dtype, nh, nkv, d
        self.cu, self.begin, self.end, self.Tk = shape
        self.Tq = int(self.cu[-1])
        rng = np.random.default_rng(seed)
        dt = torch_dtype(dtype)
        nq, nk = nh * d, nkv * d
        wide = lambda rows, n, s=1.0: dev(rng.standard_normal((rows, n + pad)) * s, dtype)[:, :n]  # noqa: E731
        self.q, self.do = wide(self.Tq, nq, std), wide(self.Tq, nq)
        if packed:
            kv = wide(self.Tk, 2 * nk)
            self.k, self.v = kv[:, :nk], kv[:, nk:]
        else:
            self.k, self.v = wide(self.Tk, nk), wide(self.Tk, nk)
        full = lambda rows, n: torch.full((rows + 1, n + pad), 7.0, dtype=dt, device="cuda")  # noqa: E731
        self.buf = {n: full(r, c) for n, r, c in (("o", self.Tq, nq), ("dq", self.Tq, nq), ("dk", self.Tk, nk), ("dv", self.Tk, nk))}
        self.out = {n: b[:-1, :b.shape[1] - pad] for n, b in self.buf.items()}
        self.pad = pad
        self.lse = torch.full((nh, self.Tq), 7.0, device="cuda")
        self.desc = mm.make_cross_attn_desc(dtype, nh, nkv, d, scale)
        self.scale = float(np.float32(scale)) or 1.0 / np.sqrt(d)
        self.batch = mm.CrossBatch.on_device(self.cu, self.begin, self.end, self.Tk)
        self.ws = None

    def workspace(self, back):
        n = mm.mmtrain_cross_attn_workspace_bytes(self.desc, self.batch, back)
        self.ws = torch.full((n,), 0xA5, dtype=torch.uint8, device="cuda")
        return self.ws, n

    def fwd(self, lse=True):
        t = mm.make_cross_attn_tensors(self.q, self.k, self.v, self.out["o"], self.lse if lse else None)
        check(mm.mmtrain_cross_attn_fwd(self.desc, self.batch, t, *self.workspace(0)), "cross_attn_fwd")
        return self.out["o"], self.lse

    def bwd(self, want=("dq", "dk", "dv")):
        t = mm.make_cross_attn_tensors(self.q, self.k, self.v, self.out["o"], self.lse)
        g = mm.make_cross_attn_grads(self.do, *[self.out[n] if n in want else None for n in ("dq", "dk", "dv")])
        check(mm.mmtrain_cross_attn_bwd(self.desc, self.batch, t, g, *self.workspace(1)), "cross_attn_bwd")
        return self.out

    def heads(self, t, n):
        return host(t).reshape(len(t), n, self.d) if len(t) else np.zeros((0, n, self.d))

    def verify(self, back=True):
        nh, nkv, d = self.nh, self.nkv, self.d
        longest = int(max((self.end - self.begin).max(), 1)) if len(self.begin) else 1
        o, lse = self.fwd()
        torch.cuda.synchronize()
        q, k, v = self.heads(self.q, nh), self.heads(self.k, nkv), self.heads(self.v, nkv)
        (ro, rl), (mag, stored, mlse) = ao.cross_fwd(q, k, v, self.cu, self.begin, self.end, self.scale)
        near("o", o, flat(ro), flat(mag), d + longest + 64, flat(stored), self.dtype)
        blind = np.isneginf(rl)
        got = host(lse)
        assert np.array_equal(np.isneginf(got), blind)
        rl[blind], got[blind] = 0.0, 0.0
        close("lse", torch.from_numpy(got), rl, mlse, d + longest + 64, mm.F32)
        if back:
            out = self.bwd()
            torch.cuda.synchronize()
            ref, mag, stored = ao.cross_bwd(q, k, v, self.heads(o, nh), host(lse), self.heads(self.do, nh), self.cu, self.begin, self.end, self.scale)
            terms = d + max(longest, self.Tq * nh // nkv) + 64
            for n in ("dq", "dk", "dv"):
                near(n, out[n], flat(ref[n]), flat(mag[n]), terms, flat(stored[n]), self.dtype)
        for n, b in self.buf.items():                                  # nothing behind the rows and columns is touched
            assert torch.all(b[-1] == 7.0) and (not self.pad or torch.all(b[:, b.shape[1] - self.pad:] == 7.0)), n
        return self


RAGGED = runs([5, 1, 40, 0, 33, 64, 7, 130], [70, 3, 0, 20, 129, 64, 1, 200])
DTYPES = pytest.mark.parametrize("dtype", [mm.BF16, mm.F32])


@DTYPES
@pytest.mark.parametrize("d", [16, 32, 48, 64, 80, 96, 112, 128])
def test_cross_head_widths(dtype, d):
    Cross(dtype, 4, 2, d, RAGGED, std=2.0, seed=d).verify()


@DTYPES
@pytest.mark.parametrize("nh,nkv", [(1, 1), (6, 6), (6, 2), (5, 1), (16, 2), (24, 1)])
@pytest.mark.parametrize("d", [64, 128])
def test_cross_heads(dtype, nh, nkv, d):
    Cross(dtype, nh, nkv, d, RAGGED, seed=nh, pad=8, packed=False).verify()


@DTYPES
@pytest.mark.parametrize("pattern", ["own", "shared", "previous"])
def test_cross_ranges(dtype, pattern):
    rng = np.random.default_rng(20)
    for S, longest in ((3, 300), (9, 100), (70, 9), (150, 40)):
        shape = runs(rng.integers(0, longest, S), rng.integers(0, 150, S), pattern, tail=3)
        Cross(dtype, 4, 2, 64, shape, seed=S).verify()
    Cross(dtype, 2, 2, 128, runs(rng.integers(1, 90, 12), rng.integers(1, 150, 12), pattern, tail=130), seed=21).verify()


@DTYPES
@pytest.mark.parametrize("lq,lk", [(1, 1), (1, 2), (2, 1), (31, 33), (32, 32), (33, 31), (64, 64), (65, 63), (127, 129), (128, 128), (129, 127), (256, 65), (257, 1), (1, 257), (300, 700)])
def test_cross_sizes(dtype, lq, lk):
    for d in (64, 80, 128):
        Cross(dtype, 3, 3, d, runs([lq], [lk]), seed=lq + lk).verify()
    Cross(dtype, 4, 1, 128, runs([lq, 3, lq], [lk, 5, lk]), seed=lq * lk).verify()


@DTYPES
def test_cross_nothing_to_see(dtype):
    c = Cross(dtype, 4, 2, 64, runs([3, 40, 2], [0, 0, 0], tail=50)).verify()
    assert torch.all(c.out["o"] == 0) and torch.all(c.out["dk"] == 0) and torch.all(c.out["dq"] == 0)
    Cross(dtype, 4, 2, 64, (np.array([0, 5], np.int32), np.array([0], np.int32), np.array([0], np.int32), 0)).verify()
    Cross(dtype, 4, 2, 64, runs([0, 0], [30, 5])).verify()
    Cross(dtype, 4, 2, 64, (np.array([0], np.int32), np.zeros(0, np.int32), np.zeros(0, np.int32), 70)).verify()


@DTYPES
def test_cross_single_tokens(dtype):
    rng = np.random.default_rng(22)
    for nh, nkv, d, S, longest in ((8, 8, 64, 3, 50), (8, 1, 128, 5, 3000), (64, 8, 128, 2, 1500), (4, 2, 80, 90, 70), (6, 2, 64, 1, 9000), (40, 1, 64, 2, 700)):
        Cross(dtype, nh, nkv, d, runs([1] * S, rng.integers(0, longest, S)), std=2.0, seed=S).verify(back=d != 128)
    Cross(dtype, 8, 2, 64, runs([1, 2, 1, 3], [1000, 2000, 1, 1500], "shared", 2), seed=23).verify()


@DTYPES
def test_cross_forward_takes_ranges_in_any_order(dtype):
    cu, begin, end, Tk = runs([3, 50, 1, 20, 9], [100, 40, 300, 7, 65])
    at = [3, 0, 4, 1, 2]
    Cross(dtype, 4, 2, 64, (cu, begin[at], end[at], Tk), seed=24).verify(back=False)
    Cross(dtype, 4, 2, 64, (np.arange(6, dtype=np.int32), begin[at], end[at], Tk), seed=25).verify(back=False)
    # a run that sees nothing may name any place, also where keys get gradients
    begin, end = begin.copy(), end.copy()
    begin[2] = end[2] = 2
    Cross(dtype, 4, 2, 64, (cu, begin, end, Tk), seed=26).verify()


@DTYPES
def test_cross_what_is_not_seen_does_not_reach(dtype):
    """Infinities and NaN in keys and values that a run does not see, in queries and gradients of other runs, and behind the rows."""
    for lq in ([20, 40, 9], [1, 1, 1], [300, 150, 200]):
        for lk in ([90, 33, 70], [200, 1, 31]):
            for d in (64, 128):
                shape = runs(lq, lk, tail=40)
                c = Cross(dtype, 4, 2, d, shape, seed=27)
                c.fwd(), c.bwd()
                want = {n: t.clone() for n, t in c.out.items()}
                lse = c.lse.clone()
                a, b, lo, hi = int(c.cu[1]), int(c.cu[2]), int(c.begin[1]), int(c.end[1])
                for bad in (float("nan"), float("inf")):
                    for t, r0, r1 in ((c.q, a, b), (c.do, a, b), (c.k, lo, hi), (c.v, lo, hi)):
                        t[r0:r1] = bad
                    c.k[int(c.end[2]):] = bad
                    c.v[int(c.end[2]):] = bad
                    c.fwd(), c.bwd()
                    for n, t in c.out.items():
                        r0, r1 = (a, b) if n in ("o", "dq") else (lo, hi)
                        live = torch.ones(len(t), dtype=torch.bool, device="cuda")
                        live[r0:r1] = False
                        assert torch.equal(t[live], want[n][live]), (n, bad, lq, lk, d)
                    live = torch.ones(c.Tq, dtype=torch.bool, device="cuda")
                    live[a:b] = False
                    assert torch.equal(c.lse[:, live], lse[:, live])


@DTYPES
def test_cross_large_scores(dtype):
    """Scores of several hundred, which only the largest keys of a row survive, and rows of equal scores."""
    c = Cross(dtype, 4, 2, 64, runs([70, 1, 33], [100, 300, 65]), std=40.0, seed=28)
    c.q[3] = 0.0
    c.verify()
    Cross(dtype, 4, 2, 64, runs([40], [90]), scale=0.5, std=3.0, seed=29).verify()


@DTYPES
def test_cross_some_gradients(dtype):
    for lq in ([20, 40, 9], [1, 1, 1]):
        c = Cross(dtype, 4, 2, 64, runs(lq, [90, 33, 70]), seed=30)
        c.fwd(), c.bwd()
        want = {n: t.clone() for n, t in c.out.items()}
        for names in (("dq",), ("dk", "dv")):
            for n in ("dq", "dk", "dv"):
                c.out[n].fill_(3.0)
            c.bwd(names)
            for n in ("dq", "dk", "dv"):
                assert torch.equal(c.out[n], want[n] if n in names else torch.full_like(want[n], 3.0))
        c.fwd(lse=False)
        assert torch.equal(c.out["o"], want["o"])


def test_cross_repeats_bit_for_bit():
    for dtype, nh, nkv, d, shape in ((mm.BF16, 16, 2, 128, runs([700, 300], [500, 900])), (mm.BF16, 8, 8, 64, runs([1] * 4, [3000] * 4)),
                                     (mm.F32, 4, 2, 64, runs([70, 300], [500, 90]))):
        c = Cross(dtype, nh, nkv, d, shape, seed=31)
        c.fwd(), c.bwd()
        first = {n: t.clone() for n, t in c.out.items()}
        for t in c.out.values():
            t.fill_(1.0)
        c.fwd(), c.bwd()
        assert all(torch.equal(first[n], t) for n, t in c.out.items())


def test_cross_keys_past_32_bits():
    # keys of the second run stand past 2^31 elements; strides of 2^20
    nh, nkv, d, ld, Tk = 4, 2, 64, 1 << 20, 2300
    big = torch.zeros(Tk * ld, dtype=torch.bfloat16, device="cuda").view(Tk, ld)
    rng = np.random.default_rng(32)
    kv = dev(rng.standard_normal((Tk, 256)), mm.BF16)
    big[:, :256] = kv
    for lq in ([3, 40], [1, 1]):
        cu, begin, end = np.concatenate([[0], np.cumsum(lq)]), np.array([0, 2060]), np.array([2100, 2300])
        c = Cross(mm.BF16, nh, nkv, d, (cu.astype(np.int32), begin.astype(np.int32), end.astype(np.int32), Tk), seed=33)
        c.k, c.v = kv[:, :128], kv[:, 128:]
        c.fwd(), c.bwd()
        want, lse = {n: t.clone() for n, t in c.out.items()}, c.lse.clone()
        c.k, c.v = big[:, :128], big[:, 128:256]
        c.out["dk"], c.out["dv"] = big[:, 512:640], big[:, 1024:1152]
        c.fwd(), c.bwd()
        assert torch.equal(c.lse, lse) and all(torch.equal(t, want[n]) for n, t in c.out.items())


def test_cross_dispatch_from_two_streams_and_a_graph():
    """Two calls at once with a workspace each, and a captured forward and backward pass, replayed."""
    cs = [Cross(mm.BF16, 8, 2, 128, runs([200, 1, 90], [700, 300, 65]), seed=34), Cross(mm.BF16, 8, 2, 128, runs([1] * 7, [900] * 7), seed=35)]
    want = []
    for c in cs:
        c.fwd(), c.bwd()
        want.append({n: t.clone() for n, t in c.out.items()})
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cs]
    keep = []
    for c, st in zip(cs, streams):
        with torch.cuda.stream(st):
            for t in c.out.values():
                t.fill_(1.0)
            c.fwd()
            keep.append(c.ws)
            c.bwd()
            keep.append(c.ws)
    torch.cuda.synchronize()
    for c, w in zip(cs, want):
        assert all(torch.equal(t, w[n]) for n, t in c.out.items())
    c = cs[0]
    nf, nb = (mm.mmtrain_cross_attn_workspace_bytes(c.desc, c.batch, b) for b in (0, 1))
    wf, wb = (torch.full((n,), 0xA5, dtype=torch.uint8, device="cuda") for n in (nf, nb))
    t = mm.make_cross_attn_tensors(c.q, c.k, c.v, c.out["o"], c.lse)
    g = mm.make_cross_attn_grads(c.do, c.out["dq"], c.out["dk"], c.out["dv"])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        check(mm.mmtrain_cross_attn_fwd(c.desc, c.batch, t, wf, nf), "fwd")
        check(mm.mmtrain_cross_attn_bwd(c.desc, c.batch, t, g, wb, nb), "bwd")
    for i in range(3):
        for x in c.out.values():
            x.fill_(float(i))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, want[0][n]) for n, x in c.out.items()), i
        wf.fill_(i), wb.fill_(i)


# ---- cross attention: the forms that a call takes ----------------------------------------------------------------------------
@DTYPES
def test_cross_gradients_of_few_rows_and_long_walks(dtype):
    """dQ in chunks of keys: runs that have several, one or none; few keys and no keys among them; and without dQ."""
    for nh, nkv, d in ((4, 2, 64), (3, 3, 80), (4, 1, 128)):
        c = Cross(dtype, nh, nkv, d, runs([20, 1, 0, 7, 3], [1500, 60, 900, 0, 1031], tail=9), seed=40, pad=8).verify()
        first = {n: t.clone() for n, t in c.out.items()}
        for want in (("dq",), ("dk", "dv")):
            for n in ("dq", "dk", "dv"):
                c.out[n].fill_(5.0)
            c.bwd(want)
            assert all(torch.equal(c.out[n], first[n]) if n in want else torch.all(c.out[n] == 5.0) for n in ("dq", "dk", "dv"))
    S = 70
    lk = np.full(S, 3)
    lk[[0, 40, 69]] = 1300, 900, 1100
    Cross(dtype, 2, 1, 64, runs([1] * S, lk), seed=41).verify()


@DTYPES
@pytest.mark.parametrize("lq,lk,nh,nkv", [(900, 100, 8, 2), (700, 260, 4, 4), (333, 1, 6, 1)])
def test_cross_gradients_of_many_rows_and_few_keys(dtype, lq, lk, nh, nkv):
    """dK and dV of a tile from several workgroups."""
    for d in (64, 112):
        Cross(dtype, nh, nkv, d, runs([lq, 5, lq // 2], [lk, 70, lk]), seed=lq + d).verify()
    Cross(dtype, nh, nkv, 128, runs([lq, lq // 3, 64], [lk, lk, lk], "previous"), seed=lq).verify()


def test_cross_fp32_gradients_of_short_runs():
    """A wavefront for each 16 keys: pieces that end inside a workgroup's keys."""
    rng = np.random.default_rng(42)
    Cross(mm.F32, 16, 8, 64, runs(rng.integers(0, 7, 40), rng.integers(90, 160, 40), tail=70), seed=43).verify()
    Cross(mm.F32, 8, 8, 80, runs(rng.integers(1, 4, 30), rng.integers(140, 180, 30), "previous", tail=3), seed=44).verify()


@DTYPES
@pytest.mark.parametrize("S,group", [(5, 5), (63, 7), (64, 64), (65, 65), (130, 9), (200, 200), (300, 3)])
def test_cross_neighbouring_runs_with_the_same_keys(dtype, S, group):
    """As many continuations of a prompt; some have no token."""
    rng = np.random.default_rng(S)
    shape = runs(rng.integers(0, 4, S), rng.integers(0, 300, -(-S // group)), "shared", group, tail=2)
    Cross(dtype, 4, 2, 64, shape, seed=S).verify()
    cu, begin, end, Tk = shape
    begin, end = begin.copy(), end.copy()
    begin[S // 2] = end[S // 2] = 0                    # one among them sees nothing
    Cross(dtype, 2, 2, 128, (cu, begin, end, Tk), seed=S + 1).verify()
    end[0] = begin[0]                                  # ... and the first
    Cross(dtype, 2, 1, 80, (cu, begin, end, Tk), seed=S + 2).verify()


@DTYPES
@pytest.mark.parametrize("S", [255, 256, 257, 700, 1100])
def test_cross_many_runs(dtype, S):
    rng = np.random.default_rng(S)
    Cross(dtype, 2, 1, 64, runs(rng.integers(0, 4, S), rng.integers(0, 20, S), tail=200), seed=S).verify()
    Cross(dtype, 2, 2, 64, runs(rng.integers(0, 3, S), rng.integers(0, 9, S), "previous", 40), seed=S + 1).verify()


@DTYPES
def test_cross_more_tiles_than_are_sorted(dtype):
    Cross(dtype, 2, 1, 64, runs([2, 1, 3], [45000, 60000, 30001], tail=400), seed=45).verify()


def test_cross_forward_of_long_runs_of_rows_and_keys():
    """Workgroups of 256 rows."""
    Cross(mm.BF16, 64, 4, 128, runs([300, 1], [4200, 33]), seed=46).verify(back=False)


@pytest.mark.parametrize("T", [15, 16, 17, 4095, 4096, 4097, 32767, 32768, 32769])
def test_embed_where_its_order_and_chunks_change(T):
    test_embed_long(T, 5000, 70)


@pytest.mark.parametrize("T,H", [(1024, 4096), (1025, 4096), (2048, 2048), (2049, 2048), (16400, 2048)])
def test_embed_chunks_of_wide_rows(T, H):
    """Sums of small whole numbers, exact in fp32."""
    rng = np.random.default_rng(T)
    ids = torch.from_numpy(rng.integers(0, 40, T).astype(np.int32)).to("cuda")
    dy = torch.from_numpy(rng.integers(-2, 3, (T, H)).astype(np.float32)).to("cuda", torch.bfloat16)
    desc = mm.make_embed_desc(mm.BF16, H, 40, 0, 1.0)
    wsb = mm.mmtrain_embed_workspace_bytes(desc, T)
    ws, d_table = torch.full((wsb,), 0xA5, dtype=torch.uint8, device="cuda"), torch.empty((40, H), device="cuda")
    check(mm.mmtrain_embed_bwd(desc, T, ids, dy, d_table, None, mm.BWD_WGRAD_F32, ws, wsb), "embed_bwd")
    assert torch.equal(d_table, torch.zeros((40, H), device="cuda").index_add_(0, ids.long(), dy.float()))


def test_embed_and_norms_in_a_graph():
    """Captured and replayed with other tokens; eager calls with a workspace of their own in between."""
    T, H, V, nq, nk, d = 5000, 256, 300, 2, 1, 64
    gen = torch.Generator(device="cuda").manual_seed(47)
    new = lambda *s: torch.randn(s, generator=gen, device="cuda").to(torch.bfloat16)  # noqa: E731
    desc, norms, rope = mm.make_embed_desc(mm.BF16, H, V, 0, 1.0), mm.make_qk_norm_desc(mm.BF16, nq, nk, d), mm.make_rope_desc(mm.BF16, nq + nk, d)
    batch = mm.PackedBatch.on_device(np.array([0, 4000, 5000], dtype=np.int32))
    table, w = new(V, H), {"q_w": new(d), "k_w": new(d)}
    ids, dy = torch.zeros(T, dtype=torch.int32, device="cuda"), new(T, H)
    out = {"x": torch.empty_like(dy), "y": torch.zeros_like(dy), "dx": torch.zeros_like(dy), "table": torch.empty((V, H), device="cuda"),
           "q_w": torch.empty(d, device="cuda"), "k_w": torch.empty(d, device="cuda")}
    wsb = max(mm.mmtrain_embed_workspace_bytes(desc, T), mm.mmtrain_qk_norm_rope_workspace_bytes(norms, T))
    spaces = [torch.full((wsb,), 0xA5, dtype=torch.uint8, device="cuda") for _ in range(2)]

    def call(ws):
        cw = mm.make_qk_norm_weights(w)
        check(mm.mmtrain_embed_fwd(desc, T, ids, table, None, out["x"]), "embed_fwd")
        check(mm.mmtrain_qk_norm_rope_fwd(norms, rope, T, batch, None, cw, out["x"], H, out["y"], H), "fwd")
        check(mm.mmtrain_qk_norm_rope_bwd(norms, rope, T, batch, None, cw, out["x"], H, dy, H, out["dx"], H, mm.make_qk_norm_grads({k: out[k] for k in w}), mm.BWD_WGRAD_F32,
                                          ws, wsb), "bwd")
        check(mm.mmtrain_embed_bwd(desc, T, ids, out["dx"], out["table"], None, mm.BWD_WGRAD_F32, ws, wsb), "embed_bwd")
    call(spaces[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(spaces[0])
    for i in range(4):
        ids.copy_(torch.randint(-1, V + 1, (T,), generator=gen, device="cuda", dtype=torch.int32))
        dy.copy_(new(T, H))
        call(spaces[1])
        torch.cuda.synchronize()
        want = {k: t.clone() for k, t in out.items()}
        for k in ("table", "q_w", "k_w", "x"):
            out[k].fill_(float(i))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(t, want[k]) for k, t in out.items()), i


def test_embed_of_more_workgroups_than_a_launch_has_along_x():
    # rows to clear, 16 to a workgroup, behind 2^20 workgroups; rows written from more than 2^28 pieces
    V = (1 << 24) + 5000
    ids = torch.tensor([V - 1, 3, V - 1, 1 << 24], dtype=torch.int32, device="cuda")
    desc = mm.make_embed_desc(mm.BF16, 8, V, 0, 1.0)
    dy, d_table = torch.ones((4, 8), dtype=torch.bfloat16, device="cuda"), torch.full((V, 8), float("nan"), dtype=torch.bfloat16, device="cuda")
    wsb = mm.mmtrain_embed_workspace_bytes(desc, 4)
    ws = torch.empty(wsb, dtype=torch.uint8, device="cuda")
    check(mm.mmtrain_embed_bwd(desc, 4, ids, dy, d_table, None, 0, ws, wsb), "embed_bwd")
    assert float(d_table.float().sum()) == 32.0 and torch.all(d_table[V - 1] == 2) and torch.all(d_table[3] == 1) and torch.all(d_table[1 << 24] == 1)
    T, H, V = 140000, 16384, 50
    ids = torch.arange(T, dtype=torch.int32, device="cuda") % V
    table, y = torch.randn((V, H), device="cuda").to(torch.bfloat16), torch.zeros((T, H), dtype=torch.bfloat16, device="cuda")
    check(mm.mmtrain_embed_fwd(mm.make_embed_desc(mm.BF16, H, V, 0, 1.0), T, ids, table, None, y), "embed_fwd")
    assert torch.equal(y.view(-1, V, H), table.expand(T // V, V, H))


@pytest.mark.parametrize("nq,nk", [(2, 1), (0, 1), (3, 0)])
def test_qk_norm_no_tokens_writes_zero_gradients(nq, nk):
    w = {k + "_w": torch.ones(64, device="cuda") for k, n in (("q", nq), ("k", nk)) if n}
    desc = mm.make_qk_norm_desc(mm.F32, nq, nk, 64)
    wsb = mm.mmtrain_qk_norm_rope_workspace_bytes(desc, 0)
    ws = torch.full((wsb,), 0xA5, dtype=torch.uint8, device="cuda")
    for flags, want in ((0, 0.0), (mm.BWD_ACCUMULATE_WGRAD, 3.0)):
        grads = {k: torch.full((64,), 3.0, device="cuda") for k in w}
        check(mm.mmtrain_qk_norm_rope_bwd(desc, None, 0, None, None, mm.make_qk_norm_weights(w), None, 512, None, 512, None, 512, mm.make_qk_norm_grads(grads), flags, ws, wsb), "bwd")
        assert all(torch.all(t == want) for t in grads.values())


@pytest.mark.parametrize("S,nh,nkv,d,longest", [(20, 32, 32, 64, 300), (90, 32, 32, 64, 70), (15, 32, 32, 128, 200), (20, 32, 32, 128, 60), (20, 32, 32, 128, 900), (40, 64, 32, 80, 90), (70, 48, 24, 96, 40)])
def test_cross_many_workgroups_of_few_rows(S, nh, nkv, d, longest):
    """Workgroups of two wavefronts and of one; some runs without tokens or keys, and walks of one block and of many."""
    rng = np.random.default_rng(S + d)
    Cross(mm.BF16, nh, nkv, d, runs(rng.integers(0, 7, S), rng.integers(0, longest, S), tail=5), std=2.0, seed=S).verify()


def test_qk_norm_features_beside_a_small_mean():
    """A feature and its head's mean are both near zero among features of 1: the mean's rounding errors, which the other features make, are all that
    is off."""
    qk_case(mm.F32, 6, 1, 248, 0, "half", "layer", T=240, other=64, main=True, seed=5365)
    qk_case(mm.F32, 2, 2, 80, 40, "interleaved", "layer", T=700, positions=np.arange(700), seed=48)
