"""What the operators at the two ends of a multimodal decoder's attention are measured on: the embedding of a pack of text tokens and
image features with its gradient, per-head norms of queries and keys with the rotation in the same pass, and attention from a pack of
text to encoder states of other lengths.

`own` false: elementary torch operations in 32 bits (64 where angles of far positions need them), rounded once; ragged segments are
gathered into padded ones, so there is no loop over them.  `own` true: the library's calls.  `exact` evaluates the definitions in 64 bits.
"""
import math

import numpy as np
import torch

own = False

NORM_EPS = 1e-6


# ---------------------------------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------------------------------
def _cross(name, dtype, segments, q_tokens, kv_tokens, heads, kv_heads, d, ranges, direction, pack_seed):
    """`segments` runs of queries, one token each where q_tokens is their number.  ranges: "own" = each sees its piece of the keys,
    "shared" = four in a row see the same piece (several continuations of one prompt), "previous" = each sees its piece and the ones
    before it in its group of four (text between images sees the images so far)."""
    return dict(name=name, what="cross", dtype=dtype, segments=segments, q_tokens=q_tokens, kv_tokens=kv_tokens, heads=heads, kv_heads=kv_heads,
                head_dim=d, ranges=ranges, direction=direction, pack_seed=pack_seed)


def _qk(name, dtype, tokens, q_heads, k_heads, other, d, rot, norm, layout, scaling, positions, direction, main, pack_seed=0):
    """`other` heads (values) stand behind the queries and keys in a row and are left alone; rot 0: no rotation; main: gain gradients
    added to fp32 buffers."""
    return dict(name=name, what="qk", dtype=dtype, tokens=tokens, q_heads=q_heads, k_heads=k_heads, other=other, head_dim=d, rot=rot, norm=norm,
                layout=layout, scaling=scaling, positions=positions, direction=direction, main=main, pack_seed=pack_seed)


def _embed(name, dtype, tokens, hidden, vocab, features, direction, main, pack_seed=0):
    """`features` rows of an encoder stand in the pack beside the text; main: the table's gradient is added to an fp32 buffer."""
    return dict(name=name, what="embed", dtype=dtype, tokens=tokens, hidden=hidden, vocab=vocab, features=features, direction=direction, main=main,
                pack_seed=pack_seed)


def listed():
    return [
        # three sequences generate a token each over the states of an image or two: latency alone
        _cross("cross_single_tokens", "bf16", 3, 3, 1733, 16, 4, 64, "own", "forward", 1),
        # sixteen sequences of the 72B heads, a token each, over long encoder states: the keys' and values' bytes
        _cross("cross_single_tokens_long", "bf16", 16, 16, 98311, 64, 8, 128, "own", "forward", 2),
        # the 7B heads' pack of 8192 text tokens in twelve samples, each of which sees its two images of 576 features
        _cross("cross_7b_forward", "bf16", 12, 8192, 13824, 32, 32, 128, "own", "forward", 3),
        # ... and back
        _cross("cross_7b_backward", "bf16", 12, 8192, 13824, 32, 32, 128, "own", "backward", 3),
        # interleaved samples of the 72B heads: 61 short runs of text, each of which sees the images so far; back
        _cross("cross_interleaved_backward", "bf16", 61, 2111, 18307, 64, 8, 128, "previous", "backward", 4),
        # the 80-wide heads' model in fp32, as numerics are debugged, back
        _cross("cross_f32_80_backward", "f32", 5, 1031, 2111, 16, 16, 80, "own", "backward", 5),
        # seven sequences generate a token each far into a stretched context: the smallest call
        _qk("qk_single_tokens", "bf16", 7, 32, 8, 8, 128, 128, "rms", "half", "wavelength", "far", "forward", False),
        # the 7B-shaped layer's packed qkv, gains' gradients added up over microbatches in fp32
        _qk("qk_7b_backward", "bf16", 8192, 32, 32, 32, 128, 128, "rms", "half", "plain", "pack", "backward", True, 6),
        # a long odd pack of the 72B heads, LayerNorm, half of each head rotated, interleaved, stretched context
        _qk("qk_72b_partial_forward", "bf16", 16411, 64, 8, 8, 128, 64, "layer", "interleaved", "ramp", "pack", "forward", False, 7),
        # a pack of text and image rows through the 7B-wide table
        _embed("embed_pack_forward", "bf16", 8192, 4096, 32768, 4608, "forward", False, 8),
        # ... and back into the fp32 main gradient of the table, of which few rows are touched
        _embed("embed_main_backward", "bf16", 8192, 4096, 32768, 4608, "backward", True, 8),
        # the whole gradient of a large vocabulary's 72B-wide bf16 table from a long odd pack
        _embed("embed_whole_backward", "bf16", 16411, 8192, 131072, 5000, "backward", False, 9),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    what = rng.choice(["cross", "cross", "cross", "qk", "qk", "embed", "embed"])
    seed = rng.randrange(1 << 20)
    if what == "cross":
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        heads, kv_heads = rng.choice([(4, 4), (16, 16), (32, 32), (12, 4), (32, 8), (64, 8)])
        d = rng.choice([64, 80, 128]) if dtype == "bf16" else rng.choice([64, 80])
        ranges = rng.choice(["own", "own", "shared", "previous"])
        if rng.random() < 0.35:
            S = _log_int(rng, 1, 48)
            c = _cross("", dtype, S, S, S * _log_int(rng, 16, 4000 if dtype == "bf16" else 1000), heads, kv_heads, d, ranges, "forward", seed)
        else:
            S = _log_int(rng, 1, 80)
            most = 8192 if dtype == "bf16" else 1200
            c = _cross("", dtype, S, max(S, _log_int(rng, 8, most)), S * _log_int(rng, 8, 1500), heads, kv_heads, d, ranges,
                       rng.choice(["forward", "backward", "backward"]), seed)
        while c["kv_tokens"] > 64 and _pairs(c) * heads * d > (3.0e10 if dtype == "bf16" else 2.5e9):
            c["kv_tokens"] //= 2
        while c["kv_tokens"] * kv_heads * d > 9.0e7:
            c["kv_tokens"] //= 2
    elif what == "qk":
        d = rng.choice([64, 80, 128])
        rot = rng.choice([d, d, d // 2, 0])
        scaling = rng.choice(["plain", "plain", "linear", "wavelength", "ramp"])
        direction = rng.choice(["forward", "backward"])
        c = _qk("", rng.choice(["bf16", "bf16", "f32"]), _log_int(rng, 1, 10000), rng.choice([4, 16, 20, 32, 64]), rng.choice([0, 4, 8, 16]),
                rng.choice([0, 4, 8]), d, rot, rng.choice(["rms", "rms", "layer"]), rng.choice(["half", "interleaved"]), scaling,
                rng.choice(["far", "pack"]), direction, direction == "backward" and rng.random() < 0.5, seed)
    else:
        T = _log_int(rng, 1, 40000)
        direction = rng.choice(["forward", "backward", "backward"])
        H = rng.choice([8 * rng.randint(8, 300), rng.choice([1024, 1280, 4096, 8192])])
        while T * H > 1.2e8:
            T //= 2
        c = _embed("", rng.choice(["bf16", "bf16", "f32"]), T, H, _log_int(rng, 300, 60000), rng.choice([0, T // 2]), direction,
                   direction == "backward" and rng.random() < 0.6, seed)
    c.pop("name")
    return c


# ---------------------------------------------------------------------------------------------------------------------
# packs: from the case alone
# ---------------------------------------------------------------------------------------------------------------------
def _split(rng, total, n, least=0):
    """`total` in n parts within a factor of about three of one another."""
    w = rng.uniform(0.5, 1.5, n)
    cuts = np.floor(np.cumsum(w) / w.sum() * (total - least * n)).astype(np.int64)
    cuts[-1] = total - least * n
    return np.diff(np.concatenate([[0], cuts])) + least


def _ranges(c):
    """cu_q and, for each run of queries, the keys that it sees; every tenth run of several tokens sees none, and the last rows of the
    keys belong to nobody where there are enough."""
    rng = np.random.default_rng(c["pack_seed"])
    S = c["segments"]
    lq = _split(rng, c["q_tokens"], S, 1)
    pieces = -(-S // 4) if c["ranges"] == "shared" else S
    lk = _split(rng, c["kv_tokens"] - (5 if c["kv_tokens"] > 100 and c["kv_tokens"] % 2 else 0), pieces)
    ck = np.concatenate([[0], np.cumsum(lk)])
    s = np.arange(S)
    if c["ranges"] == "shared":
        begin, end = ck[s // 4], ck[s // 4 + 1]
    elif c["ranges"] == "previous":
        begin, end = ck[s // 4 * 4], ck[s + 1]
    else:
        begin, end = ck[s], ck[s + 1]
    if c["q_tokens"] > S:
        end = np.where(s % 10 == 4, begin, end)
    return np.concatenate([[0], np.cumsum(lq)]).astype(np.int32), begin.astype(np.int32), end.astype(np.int32)


def _pairs(c):
    cu, begin, end = _ranges(c)
    return float(np.sum(np.diff(cu).astype(np.float64) * (end - begin)))


def _cu(c):
    """A few segments of any length, an empty one among them where there is room."""
    T = c["tokens"]
    rng = np.random.default_rng(c["pack_seed"])
    n = max(1, min(24, T // 200))
    cuts = np.sort(rng.integers(0, T + 1, size=n - 1))
    if n > 3:
        cuts[1] = cuts[0]
    return np.concatenate([[0], cuts, [T]]).astype(np.int32)


# base, factor, low, high, trained context, magnitude of the cosines and sines
SCALING = {"plain": (10000.0, 1.0, 0.0, 0.0, 0.0, 1.0), "linear": (10000.0, 4.0, 0.0, 0.0, 0.0, 1.0),
           "wavelength": (500000.0, 8.0, 1.0, 4.0, 8192.0, 1.0), "ramp": (10000.0, 4.0, 1.0, 32.0, 4096.0, 1.125)}
EMBED_SCALE = 1.5


# ---------------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------------
def _dtype(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _randn(gen, shape, dtype, std=1.0, mean=0.0):
    a = torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)
    return a.mul_(std).add_(mean).to(dtype)


def _qk_params(c):
    return [n + k for n in ("q", "k") if c[n + "_heads"] for k in (("_w", "_b") if c["norm"] == "layer" else ("_w",))]


def _ids(c, gen):
    """Text tokens by their rank's frequency (the r-th most frequent word about 1 / r of the time), scattered over the vocabulary; runs of
    image features in their order; a few padded places at the end."""
    T, V, F = c["tokens"], c["vocab"], c["features"]
    u = torch.rand(T, generator=gen, device="cuda", dtype=torch.float64)
    rank = torch.exp(u * math.log(V + 1.0)).long().sub_(1).clamp_(0, V - 1)
    ids = (rank * 7919 + 17) % V
    if F:
        run = max(1, min(576, F // 3))
        t = torch.arange(T, device="cuda")
        place = t % (2 * run)
        feature = t // (2 * run) * run + place
        ids = torch.where((place < run) & (feature < F), -1 - feature, ids)
    if T > 50:
        ids[T - T // 50:] = V
    return ids.to(torch.int32)


def _inputs(c, seed):
    gen = torch.Generator(device="cuda").manual_seed(1000003 * int(seed) + 31)
    dt = _dtype(c)
    if c["what"] == "cross":
        d = c["head_dim"]
        i = {"q": _randn(gen, (c["q_tokens"], c["heads"] * d), dt), "kv": _randn(gen, (c["kv_tokens"], 2 * c["kv_heads"] * d), dt)}
        i["cu"], i["begin"], i["end"] = (torch.from_numpy(a).cuda() for a in _ranges(c))
        if c["direction"] == "backward":
            i["do"] = _randn(gen, i["q"].shape, dt)
        return i
    if c["what"] == "qk":
        i = {"x": _randn(gen, (c["tokens"], (c["q_heads"] + c["k_heads"] + c["other"]) * c["head_dim"]), dt, 1.5, 0.1)}
        if c["positions"] == "far":
            i["pos"] = torch.randint(0, 131072, (c["tokens"],), generator=gen, device="cuda", dtype=torch.int32)
        else:
            i["cu"] = torch.from_numpy(_cu(c)).cuda()
        i["w"] = {k: _randn(gen, (c["head_dim"],), dt, 0.1, 1.0 if k.endswith("_w") else 0.0) for k in _qk_params(c)}
        if c["direction"] == "backward":
            i["dy"] = _randn(gen, (c["tokens"], (c["q_heads"] + c["k_heads"]) * c["head_dim"]), dt)
            if c["main"]:
                i["main"] = {k: _randn(gen, (c["head_dim"],), torch.float32, 3.0) for k in _qk_params(c)}
        return i
    i = {"ids": _ids(c, gen)}
    if c["direction"] == "forward":
        i["table"] = _randn(gen, (c["vocab"], c["hidden"]), dt)
        i["features"] = _randn(gen, (c["features"], c["hidden"]), dt) if c["features"] else None
    else:
        i["dy"] = _randn(gen, (c["tokens"], c["hidden"]), dt)
        if c["main"]:
            i["main"] = _randn(gen, (c["vocab"], c["hidden"]), torch.float32)
    return i


def prepare(case, seed):
    c, s = dict(case), dict(case=dict(case))
    s.update(_inputs(c, seed))
    empty = lambda *shape, dtype=_dtype(c): torch.empty(shape, dtype=dtype, device="cuda")  # noqa: E731
    if c["what"] == "cross":
        s["lengths"] = tuple(int(v) for v in (np.diff(_ranges(c)[0]).max(), (_ranges(c)[2] - _ranges(c)[1]).max()))
        s["o"], s["lse"] = torch.empty_like(s["q"]), empty(c["heads"], c["q_tokens"], dtype=torch.float32)
        if c["direction"] == "backward":                 # what a forward pass has left
            s["o"], s["lse"] = _cross_forward_plain(c, s)
            s["dq"], s["dkv"] = torch.empty_like(s["q"]), torch.empty_like(s["kv"])
    elif c["what"] == "qk":
        n = (c["q_heads"] + c["k_heads"]) * c["head_dim"]
        s["out"] = empty(c["tokens"], n)
        if c["direction"] == "backward":
            s["grads"] = s["main"] if c["main"] else {k: torch.empty_like(t) for k, t in s["w"].items()}
    elif c["direction"] == "forward":
        s["y"] = empty(c["tokens"], c["hidden"])
    else:
        s["d_table"] = s["main"] if c["main"] else empty(c["vocab"], c["hidden"])
        s["d_features"] = empty(c["features"], c["hidden"]) if c["features"] else None
    if own:                                 # descriptions and workspaces, which a user's program keeps from step to step
        s["plan"] = _plan(c, s)
    return s


# ---------------------------------------------------------------------------------------------------------------------
# the library's calls
# ---------------------------------------------------------------------------------------------------------------------
def _check(status, what):
    if status:
        raise RuntimeError(f"{what}: status {status}")


def _plan(c, s):
    from paper_2408_04275_amd import binding as mm
    p = {"mm": mm, "ws_bytes": 0}
    dtype = mm.F32 if c["dtype"] == "f32" else mm.BF16
    back = c["direction"] == "backward"
    if c["what"] == "cross":
        nk = c["kv_heads"] * c["head_dim"]
        p["desc"] = mm.make_cross_attn_desc(dtype, c["heads"], c["kv_heads"], c["head_dim"])
        cu, begin, end = _ranges(c)
        p["batch"] = mm.CrossBatch(cu, begin, end, c["kv_tokens"], s["cu"], s["begin"], s["end"])
        p["tensors"] = mm.make_cross_attn_tensors(s["q"], s["kv"][:, :nk], s["kv"][:, nk:], s["o"], s["lse"])
        if back:
            p["grads"] = mm.make_cross_attn_grads(s["do"], s["dq"], s["dkv"][:, :nk], s["dkv"][:, nk:])
        p["ws_bytes"] = mm.mmtrain_cross_attn_workspace_bytes(p["desc"], p["batch"], back)
    elif c["what"] == "qk":
        n = c["q_heads"] + c["k_heads"]
        p["desc"] = mm.make_qk_norm_desc(dtype, c["q_heads"], c["k_heads"], c["head_dim"], {"rms": mm.NORM_RMS, "layer": mm.NORM_LAYER}[c["norm"]], NORM_EPS)
        base, factor, low, high, context, magnitude = SCALING[c["scaling"]]
        p["rope"] = None if not c["rot"] else mm.make_rope_desc(
            dtype, n, c["head_dim"], c["rot"], {"half": mm.ROPE_HALF, "interleaved": mm.ROPE_INTERLEAVED}[c["layout"]], base,
            {"plain": mm.ROPE_PLAIN, "linear": mm.ROPE_LINEAR, "wavelength": mm.ROPE_WAVELENGTH, "ramp": mm.ROPE_RAMP}[c["scaling"]],
            factor, low, high, context, magnitude)
        p["batch"] = mm.PackedBatch(_cu(c), cu_dev=s["cu"]) if "cu" in s and c["rot"] else None
        p["positions"] = s.get("pos") if c["rot"] else None
        p["weights"] = mm.make_qk_norm_weights(s["w"])
        if back:
            p["grads"] = mm.make_qk_norm_grads(s["grads"])
            p["flags"] = mm.BWD_ACCUMULATE_WGRAD | mm.BWD_WGRAD_F32 if c["main"] else 0
            p["ws_bytes"] = mm.mmtrain_qk_norm_rope_workspace_bytes(p["desc"], c["tokens"])
    else:
        p["desc"] = mm.make_embed_desc(dtype, c["hidden"], c["vocab"], c["features"], EMBED_SCALE)
        if back:
            p["flags"] = mm.BWD_ACCUMULATE_WGRAD | mm.BWD_WGRAD_F32 if c["main"] else 0
            p["ws_bytes"] = mm.mmtrain_embed_workspace_bytes(p["desc"], c["tokens"])
    p["ws"] = torch.empty(max(p["ws_bytes"], 256), dtype=torch.uint8, device="cuda")
    return p


def _run_own(c, s):
    p = s["plan"]
    mm, back = p["mm"], c["direction"] == "backward"
    if c["what"] == "cross":
        if not back:
            _check(mm.mmtrain_cross_attn_fwd(p["desc"], p["batch"], p["tensors"], p["ws"], p["ws_bytes"]), "cross_attn_fwd")
            return {"o": s["o"], "lse": s["lse"]}
        _check(mm.mmtrain_cross_attn_bwd(p["desc"], p["batch"], p["tensors"], p["grads"], p["ws"], p["ws_bytes"]), "cross_attn_bwd")
        return {"dq": s["dq"], "dkv": s["dkv"]}
    if c["what"] == "qk":
        x, out = s["x"], s["out"]
        if not back:
            _check(mm.mmtrain_qk_norm_rope_fwd(p["desc"], p["rope"], c["tokens"], p["batch"], p["positions"], p["weights"], x, x.shape[1], out,
                                               out.shape[1]), "qk_norm_rope_fwd")
            return {"y": out}
        _check(mm.mmtrain_qk_norm_rope_bwd(p["desc"], p["rope"], c["tokens"], p["batch"], p["positions"], p["weights"], x, x.shape[1], s["dy"],
                                           s["dy"].shape[1], out, out.shape[1], p["grads"], p["flags"], p["ws"], p["ws_bytes"]), "qk_norm_rope_bwd")
        return {"dx": out, "grads": s["grads"]}
    if not back:
        _check(mm.mmtrain_embed_fwd(p["desc"], c["tokens"], s["ids"], s["table"], s["features"], s["y"]), "embed_fwd")
        return {"y": s["y"]}
    _check(mm.mmtrain_embed_bwd(p["desc"], c["tokens"], s["ids"], s["dy"], s["d_table"], s["d_features"], p["flags"], p["ws"], p["ws_bytes"]), "embed_bwd")
    return {"d_table": s["d_table"], **({"d_features": s["d_features"]} if c["features"] else {})}


# ---------------------------------------------------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------------------------------------------------
def _padded(first, last, longest):
    """Row numbers [S, longest] of ragged runs of rows, and which of them exist."""
    n = first[:, None] + torch.arange(longest, device="cuda")
    live = n < last[:, None]
    return torch.where(live, n, torch.zeros_like(n)), live


def _heads(x, at, n, d):
    """Rows `at` [S, L] of x [tokens, n d] in 32 bits, as [S, n, L, d]."""
    return x[at].float().view(*at.shape, n, d).permute(0, 2, 1, 3).contiguous()


def _grouped(c, x, at):
    """The same of queries, [S, kv heads, heads of a group x L, d]."""
    n, g, d = c["kv_heads"], c["heads"] // c["kv_heads"], c["head_dim"]
    return _heads(x, at, n * g, d).view(at.shape[0], n, g * at.shape[1], d)


def _cross_scores(c, s):
    """Padded places of queries and keys, queries, keys, values and scaled scores, -inf where a key is not seen."""
    n, d = c["kv_heads"], c["head_dim"]
    lq, lk = max(s["lengths"][0], 1), max(s["lengths"][1], 1)
    qa, ql = _padded(s["cu"][:-1], s["cu"][1:], lq)
    ka, kl = _padded(s["begin"], s["end"], lk)
    q, k, v = _grouped(c, s["q"], qa), _heads(s["kv"][:, :n * d], ka, n, d), _heads(s["kv"][:, n * d:], ka, n, d)
    scores = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(1.0 / math.sqrt(d))
    scores.masked_fill_(~kl[:, None, None, :], -math.inf)
    return qa, ql, ka, kl, q, k, v, scores


def _ungrouped(c, x, ql):
    """[S, kv heads, heads of a group x L, d] back to rows: the places that exist follow one another as the tokens do."""
    S, L = ql.shape
    return x.view(S, c["heads"], L, -1).permute(0, 2, 1, 3)[ql]


def _cross_forward_plain(c, s):
    qa, ql, _, _, _, _, v, scores = _cross_scores(c, s)
    top = scores.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = scores.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v) / torch.where(total > 0, total, torch.ones_like(total))
    lse = _ungrouped(c, total.log() + top, ql)[..., 0].t().contiguous()
    return _ungrouped(c, o, ql).reshape(c["q_tokens"], -1).to(_dtype(c)), lse


def _cross_backward_plain(c, s):
    qa, ql, ka, kl, q, k, v, scores = _cross_scores(c, s)
    S, L = ql.shape
    n, d, dt = c["kv_heads"], c["head_dim"], _dtype(c)
    lse = s["lse"][:, qa].permute(1, 0, 2).reshape(S, n, -1, 1)
    do, o = _grouped(c, s["do"], qa), _grouped(c, s["o"], qa)
    live = ql[:, None, :].expand(S, c["heads"] // n, L).reshape(S, 1, -1, 1)
    p = scores.sub_(lse).exp_().masked_fill_(~live | ~kl[:, None, None, :], 0.0)
    dv = torch.matmul(p.transpose(2, 3).contiguous(), do)
    ds = torch.matmul(do, v.transpose(2, 3).contiguous()).sub_((do * o).sum(-1, keepdim=True)).mul_(p).mul_(1.0 / math.sqrt(d))
    dq = torch.matmul(ds, k)
    dk = torch.matmul(ds.transpose(2, 3).contiguous(), q)
    both = torch.cat([dk, dv], 1).permute(0, 2, 1, 3)[kl].reshape(-1, 2 * n * d)       # a key that several runs see gets the sum
    dkv = torch.zeros(s["kv"].shape, device="cuda").index_add_(0, ka[kl], both)
    return {"dq": _ungrouped(c, dq, ql).reshape(c["q_tokens"], -1).to(dt), "dkv": dkv.to(dt)}


def _segment_of(cu, T):
    """Each token's segment: the number of segments that end at it or before."""
    return (torch.arange(T, device=cu.device)[:, None] >= cu[None, 1:]).sum(1).clamp_(max=cu.numel() - 2)


def _frequencies(c, device):
    """Angle per position of each rotated pair, in 64 bits."""
    base, factor, low, high, context, _ = SCALING[c["scaling"]]
    r = c["rot"]
    i = torch.arange(r // 2, device=device, dtype=torch.float64)
    theta = torch.exp(i * (-2.0 / r * math.log(base)))
    if c["scaling"] == "linear":
        return theta / factor
    if c["scaling"] == "wavelength":        # kept where a pair turns often in the trained context, stretched where it hardly turns
        keep = ((context * theta / (2 * math.pi) - low) / (high - low)).clamp(0.0, 1.0)
    elif c["scaling"] == "ramp":            # the same by the pair's index
        at = lambda turns: r * math.log(context / (2 * math.pi * turns)) / (2 * math.log(base))  # noqa: E731
        first, last = max(math.floor(at(high)), 0), min(math.ceil(at(low)), r - 1)
        keep = 1.0 - ((i - first) / max(last - first, 1e-3)).clamp(0.0, 1.0)
    else:
        return theta
    return theta * (keep + (1.0 - keep) / factor)


def _turn(c, s, x, back):
    """Positions applied to the first `rot` features of heads [T, n, d], or taken back."""
    r = c["rot"]
    if not r:
        return x
    T = c["tokens"]
    pos = s["pos"] if "pos" in s else torch.arange(T, device="cuda") - s["cu"][_segment_of(s["cu"], T)]
    angle = pos.double()[:, None, None] * _frequencies(c, pos.device)
    m = SCALING[c["scaling"]][5]
    co, si = (angle.cos() * m).float(), (angle.sin() * (-m if back else m)).float()
    t = x[..., :r]
    a, b = (t[..., :r // 2], t[..., r // 2:]) if c["layout"] == "half" else (t[..., 0::2], t[..., 1::2])
    pair = (a * co - b * si, b * co + a * si)
    return torch.cat([torch.cat(pair, dim=-1) if c["layout"] == "half" else torch.stack(pair, dim=-1).flatten(-2), x[..., r:]], -1)


def _qk_plain(c, s):
    T, nq, nk, d, dt = c["tokens"], c["q_heads"], c["k_heads"], c["head_dim"], _dtype(c)
    n = nq + nk
    x = s["x"][:, :n * d].view(T, n, d).float()
    mean = x.mean(-1, keepdim=True) if c["norm"] == "layer" else 0.0
    rstd = torch.rsqrt((x - mean).square().mean(-1, keepdim=True) + NORM_EPS)
    hat = (x - mean) * rstd
    kinds = [(k, h) for k, h in (("q", nq), ("k", nk)) if h]
    rows = lambda name: torch.cat([s["w"][k + name].float().expand(h, d) for k, h in kinds])  # noqa: E731
    if c["direction"] == "forward":
        y = hat * rows("_w") + (rows("_b") if c["norm"] == "layer" else 0.0)
        return {"y": _turn(c, s, y, False).reshape(T, n * d).to(dt)}
    g = _turn(c, s, s["dy"].view(T, n, d).float(), True)
    back = g * rows("_w")
    dx = back - hat * (back * hat).mean(-1, keepdim=True)
    if c["norm"] == "layer":
        dx = dx - back.mean(-1, keepdim=True)
    sums = {}
    for name, part in (("q", slice(0, nq)), ("k", slice(nq, n))):
        if c[name + "_heads"]:
            sums[name + "_w"] = (g[:, part] * hat[:, part]).sum((0, 1))
            if c["norm"] == "layer":
                sums[name + "_b"] = g[:, part].sum((0, 1))
    grads = {k: s["main"][k].add_(v) if c["main"] else v.to(dt) for k, v in sums.items()}
    return {"dx": (dx * rstd).reshape(T, n * d).to(dt), "grads": grads}


def _embed_plain(c, s):
    dt, ids, V, F = _dtype(c), s["ids"].long(), c["vocab"], c["features"]
    text, image = (ids >= 0) & (ids < V), (ids < 0) & (ids >= -F)
    if c["direction"] == "forward":
        y = s["table"][torch.where(text, ids, torch.zeros_like(ids))].float() * (text.float() * EMBED_SCALE)[:, None]
        if F:
            y = torch.where(image[:, None], s["features"][torch.where(image, -1 - ids, torch.zeros_like(ids))].float(), y)
        return {"y": y.to(dt)}
    dy = s["dy"].float()
    out = {}
    table = s["main"] if c["main"] else torch.zeros((V, c["hidden"]), device="cuda")
    table.index_add_(0, ids[text], dy[text] * EMBED_SCALE)
    out["d_table"] = table if c["main"] else table.to(dt)
    if F:
        out["d_features"] = torch.zeros((F, c["hidden"]), device="cuda").index_add_(0, -1 - ids[image], dy[image]).to(dt)
    return out


def run(s):
    c = s["case"]
    if own:
        return _run_own(c, s)
    if c["what"] == "cross":
        if c["direction"] == "backward":
            return _cross_backward_plain(c, s)
        o, lse = _cross_forward_plain(c, s)
        return {"o": o, "lse": lse}
    return _qk_plain(c, s) if c["what"] == "qk" else _embed_plain(c, s)


# ---------------------------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------------------------------------
def work(case):
    c, e = case, 4 if case["dtype"] == "f32" else 2
    back = c["direction"] == "backward"
    if c["what"] == "cross":
        _, begin, end = _ranges(c)
        seen = np.zeros(c["kv_tokens"] + 1)
        np.add.at(seen, begin, 1)
        np.add.at(seen, end, -1)
        keys = int((np.cumsum(seen)[:-1] > 0).sum()) * 2 * c["kv_heads"] * c["head_dim"]
        q, lse = c["q_tokens"] * c["heads"] * c["head_dim"], 4.0 * c["q_tokens"] * c["heads"]
        pairs = _pairs(c) * c["heads"] * c["head_dim"]
        if not back:
            return {"bytes": e * (2.0 * q + keys) + lse, "flops": 4.0 * pairs}
        return {"bytes": e * (4.0 * q + keys + 2 * c["kv_tokens"] * c["kv_heads"] * c["head_dim"]) + lse, "flops": 10.0 * pairs}
    if c["what"] == "qk":
        n = c["tokens"] * (c["q_heads"] + c["k_heads"]) * c["head_dim"]
        return {"bytes": e * n * (3.0 if back else 2.0) + 4 * c["tokens"], "flops": n * (16.0 if back else 8.0)}
    T, H, V, F = c["tokens"], c["hidden"], c["vocab"], c["features"]
    image = T // 2 if F else 0
    r = np.arange(V)
    p = np.log((r + 2.0) / (r + 1.0)) / math.log(V + 1.0)
    rows = float(np.sum(1.0 - (1.0 - p) ** max(T - image, 0)))          # different words
    if not back:
        return {"bytes": e * H * (rows + image + T) + 4.0 * T, "flops": 1.0 * (T - image) * H}
    return {"bytes": e * H * (T + float(F)) + (8.0 * rows * H if c["main"] else 1.0 * e * V * H) + 4.0 * T, "flops": 2.0 * T * H}


# ---------------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------------------
def _exact_cross(c, i):
    """Run by run, head by head, by autograd through a softmax."""
    cu, begin, end = _ranges(c)
    nh, nk, d = c["heads"], c["kv_heads"], c["head_dim"]
    leaf = lambda t: t.double().requires_grad_(True)  # noqa: E731
    q, kv = leaf(i["q"]), leaf(i["kv"])
    o = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    lse = torch.full((nh, c["q_tokens"]), -math.inf, dtype=torch.float64, device="cuda")
    for a, b, lo, hi in zip(cu[:-1], cu[1:], begin, end):
        if lo == hi:
            continue
        a, b, lo, hi = int(a), int(b), int(lo), int(hi)
        qs = q[a:b].view(b - a, nh, d).transpose(0, 1)
        ks, vs = (kv[lo:hi, p * nk * d:(p + 1) * nk * d].view(hi - lo, nk, d).transpose(0, 1).repeat_interleave(nh // nk, 0) for p in (0, 1))
        scores = torch.bmm(qs, ks.transpose(1, 2).contiguous()) / math.sqrt(d)
        out = torch.bmm(torch.softmax(scores, -1), vs).transpose(0, 1).reshape(b - a, nh * d)
        if c["direction"] == "backward":
            out.backward(i["do"][a:b].double())
        else:
            o[a:b], lse[:, a:b] = out.detach(), torch.logsumexp(scores.detach(), -1)
    if c["direction"] == "backward":
        return {"dq": torch.zeros_like(q) if q.grad is None else q.grad, "dkv": torch.zeros_like(kv) if kv.grad is None else kv.grad}
    return {"o": o, "lse": lse}


def _exact_turn(c, i, x):
    base, s, low, high, context, magnitude = SCALING[c["scaling"]]
    r = c["rot"]
    if not r:
        return x
    k = np.arange(r // 2)
    theta = np.power(base, -2.0 * k / r)
    if c["scaling"] == "linear":
        theta = theta / s
    elif c["scaling"] == "wavelength":
        wave = 2 * np.pi / theta
        blend = (context / wave - low) / (high - low)
        theta = np.where(wave < context / high, theta, np.where(wave > context / low, theta / s, (1 - blend) * theta / s + blend * theta))
    elif c["scaling"] == "ramp":
        index = [r * np.log(context / (2 * np.pi * t)) / (2 * np.log(base)) for t in (high, low)]
        lo, hi = max(np.floor(index[0]), 0), min(np.ceil(index[1]), r - 1)
        stretch = np.clip((k - lo) / max(hi - lo, 1e-3), 0, 1)
        theta = theta / s * stretch + theta * (1 - stretch)
    if "pos" in i:
        pos = i["pos"].cpu().numpy().astype(np.float64)
    else:
        pos = np.concatenate([np.arange(L) for L in np.diff(_cu(c))]).astype(np.float64)
    phi = torch.from_numpy(pos[:, None] * theta[None, :]).cuda()
    turn = magnitude * torch.polar(torch.ones_like(phi), phi)[:, None, :]      # a pair is a complex number
    t = x[..., :r]
    z = torch.complex(t[..., :r // 2].contiguous(), t[..., r // 2:].contiguous()) if c["layout"] == "half" else \
        torch.view_as_complex(t.reshape(*t.shape[:2], r // 2, 2).contiguous())
    z = z * turn
    t = torch.cat([z.real, z.imag], -1) if c["layout"] == "half" else torch.view_as_real(z).flatten(-2)
    return torch.cat([t, x[..., r:]], -1)


def _exact_qk(c, i):
    T, n, d = c["tokens"], c["q_heads"] + c["k_heads"], c["head_dim"]
    x = i["x"][:, :n * d].double().requires_grad_(True)
    w = {k: t.double().requires_grad_(True) for k, t in i["w"].items()}
    parts = []
    for name, heads in (("q", x.view(T, n, d)[:, :c["q_heads"]]), ("k", x.view(T, n, d)[:, c["q_heads"]:])):
        if not c[name + "_heads"]:
            continue
        if c["norm"] == "layer":
            parts.append(torch.nn.functional.layer_norm(heads, (d,), w[name + "_w"], w[name + "_b"], NORM_EPS))
        else:
            parts.append(heads * (heads.pow(2).sum(-1, keepdim=True) / d + NORM_EPS) ** -0.5 * w[name + "_w"])
    y = _exact_turn(c, i, torch.cat(parts, 1)).reshape(T, n * d)
    if c["direction"] == "forward":
        return {"y": y.detach()}
    y.backward(i["dy"].double())
    return {"dx": x.grad, "grads": {k: t.grad + (i["main"][k].double() if c["main"] else 0.0) for k, t in w.items()}}


def _exact_embed(c, i):
    ids, V, F, H = i["ids"].cpu().numpy().astype(np.int64), c["vocab"], c["features"], c["hidden"]
    row = np.where((ids >= 0) & (ids < V), ids, np.where((ids < 0) & (ids >= -F), V - 1 - ids, V + F))      # table, features, nothing
    row = torch.from_numpy(row).cuda()
    if c["direction"] == "forward":
        source = [i["table"].double() * EMBED_SCALE, i["features"].double() if F else torch.zeros((0, H), dtype=torch.float64, device="cuda"),
                  torch.zeros((1, H), dtype=torch.float64, device="cuda")]
        return {"y": torch.cat(source)[row]}
    order = torch.argsort(row, stable=True)
    found, count = torch.unique_consecutive(row[order], return_counts=True)
    last = torch.cumsum(count, 0)
    table, features = torch.zeros((V, H), dtype=torch.float64, device="cuda"), torch.zeros((F, H), dtype=torch.float64, device="cuda")
    for a in range(0, H, 512):                             # sums of runs as differences of running sums: exact to 1e-12 of the terms
        run = torch.cumsum(i["dy"][:, a:a + 512].double()[order], 0)[last - 1]
        run = torch.cat([run[:1], run[1:] - run[:-1]])
        is_text, is_image = found < V, (found >= V) & (found < V + F)
        table[found[is_text], a:a + 512] = run[is_text] * EMBED_SCALE
        features[found[is_image] - V, a:a + 512] = run[is_image]
    return {"d_table": table + i["main"].double() if c["main"] else table, **({"d_features": features} if F else {})}


def exact(case, seed):
    return {"cross": _exact_cross, "qk": _exact_qk, "embed": _exact_embed}[case["what"]](case, _inputs(case, seed))
