"""What the operators around a block's products are measured on: rotary positions, the join of a block's branch with the residual
stream (norms, gate, residual scale), and the global gradient norm with clipping.

`own` false: elementary torch operations in 32 bits (64 where angles of far positions or long sums need them), rounded once.
`own` true: the library's calls.  `exact` evaluates the definitions in 64 bits.
"""
import math

import numpy as np
import torch

own = False

NORM_EPS = 1e-5


# ---------------------------------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------------------------------
def _rotary(name, dtype, tokens, heads, other, d, rot, layout, scaling, positions, gradient, in_place, pack_seed=0):
    """heads are rotated, `other` heads (values) stand behind them in the row and are left alone; positions: "far" = one int32 per
    token, "pack" = restarting in every segment."""
    return dict(name=name, what="rotary", dtype=dtype, tokens=tokens, heads=heads, other=other, head_dim=d, rot=rot, layout=layout,
                scaling=scaling, positions=positions, gradient=gradient, in_place=in_place, pack_seed=pack_seed)


def _join(name, dtype, tokens, hidden, post, pre, gate, direction, main, pack_seed=0):
    """post, pre: "none", "rms" or "layer"; gate: "none", "channel" or "segment"; main: gradients added to fp32 buffers."""
    return dict(name=name, what="join", dtype=dtype, tokens=tokens, hidden=hidden, post=post, pre=pre, gate=gate, direction=direction,
                main=main, pack_seed=pack_seed)


def _clip(name, dtype, layers, hidden, ffn, bias, apply, sizes_seed=-1):
    """The gradients of `layers` layers (sizes_seed >= 0: tensors of any size instead).  apply: "copy" = norm, then clipped into an
    fp32 copy; "adam" = norm, then the optimizer step that clips as it reads."""
    return dict(name=name, what="clip", dtype=dtype, layers=layers, hidden=hidden, ffn=ffn, bias=bias, apply=apply, sizes_seed=sizes_seed)


def listed():
    return [
        # seven sequences generate a token each, far into a context eight times the trained one: the smallest call
        _rotary("rotary_single_tokens", "bf16", 7, 40, 8, 128, 128, "half", "wavelength", "far", False, False),
        # the 7B-shaped layer's packed d_qkv on the way back, in place: 32 query and 32 key heads in front of the values
        _rotary("rotary_qkv_gradient", "bf16", 8192, 64, 32, 128, 128, "half", "plain", "pack", True, True, 4),
        # half of each head rotated, interleaved, a stretched context: the 72B heads on a long odd pack
        _rotary("rotary_partial_interleaved", "bf16", 16411, 72, 8, 128, 64, "interleaved", "ramp", "pack", False, False, 5),
        # 80-wide fp32 heads of which 40 features rotate: chunks of 16 bytes that hold four features
        _rotary("rotary_f32_80", "f32", 4111, 32, 0, 80, 40, "half", "linear", "pack", False, False, 6),
        # three tokens through the join of a 7B-wide block: latency alone
        _join("join_single_tokens", "bf16", 3, 4096, "rms", "rms", "none", "forward", False),
        # the 7B pack: norm behind the block, residual scale, norm in front of the next
        _join("join_7b_forward", "bf16", 8192, 4096, "rms", "rms", "none", "forward", False),
        # ... and back, gains' gradients added up over microbatches in fp32
        _join("join_7b_backward", "bf16", 8192, 4096, "rms", "rms", "none", "backward", True),
        # an image encoder's block with a learned scale per channel, back, on its pack of 16 images
        _join("join_vit_scale_backward", "bf16", 9536, 1024, "none", "layer", "channel", "backward", False),
        # a gate per image (conditioned blocks) on a ragged fp32 pack of the 80-wide heads' model
        _join("join_f32_segment_gate_backward", "f32", 4111, 1280, "layer", "layer", "segment", "backward", False, 2),
        # the fp32 layer that numerics are debugged with: six small tensors
        _clip("clip_f32_small", "f32", 1, 256, 688, False, "copy"),
        # 24 encoder layers of the 80-wide heads' model, 288 bf16 tensors, clipped into the fp32 gradients that the optimizer takes
        _clip("clip_vit_288_tensors", "bf16", 24, 1280, 5120, True, "copy"),
        # a 7B-shaped layer's fp32 main gradients, clipped by the optimizer step: the largest call
        _clip("clip_7b_adam", "f32", 1, 4096, 11008, False, "adam"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    what = rng.choice(["rotary", "rotary", "join", "join", "join", "clip"])
    seed = rng.randrange(1 << 20)
    if what == "rotary":
        d = rng.choice([64, 80, 128])
        scaling = rng.choice(["plain", "plain", "linear", "wavelength", "ramp"])
        positions = rng.choice(["far", "pack"])
        c = _rotary("", rng.choice(["bf16", "bf16", "f32"]), _log_int(rng, 1, 12000), rng.choice([4, 12, 20, 40, 64]), rng.choice([0, 4, 8]), d,
                    rng.choice([d, d, d // 2, d // 4]), rng.choice(["half", "interleaved"]), scaling, positions, rng.random() < 0.4,
                    scaling != "ramp" and rng.random() < 0.5, seed)
    elif what == "join":
        post, pre, gate = rng.choice([("rms", "rms", "none"), ("none", "layer", "channel"), ("layer", "layer", "segment"), ("none", "rms", "none"),
                                      ("rms", "none", "channel"), ("none", "rms", "segment")])
        H = rng.choice([8 * rng.randint(16, 300), rng.choice([1024, 1280, 2048, 4096, 5120, 8192])])
        direction = rng.choice(["forward", "backward", "backward"])
        c = _join("", rng.choice(["bf16", "bf16", "f32"]), _log_int(rng, 1, 9000), H, post, pre, gate, direction, direction == "backward" and rng.random() < 0.5, seed)
    else:
        c = _clip("", rng.choice(["f32", "bf16"]), rng.randint(1, 300), 0, 0, False, "copy", seed)
        if c["dtype"] == "f32" and rng.random() < 0.5:
            c["apply"] = "adam"
    c.pop("name")
    return c


# ---------------------------------------------------------------------------------------------------------------------
# packs, tensor sizes, hyperparameters: from the case alone
# ---------------------------------------------------------------------------------------------------------------------
def _cu(c):
    """A few segments of any length, an empty one among them where there is room."""
    T = c["tokens"]
    rng = np.random.default_rng(c["pack_seed"])
    n = max(1, min(24, T // 200))
    cuts = np.sort(rng.integers(0, T + 1, size=n - 1))
    if n > 3:
        cuts[1] = cuts[0]
    return np.concatenate([[0], cuts, [T]]).astype(np.int32)


def _layer_sizes(c):
    H, F = c["hidden"], c["ffn"]
    if c["bias"]:
        return [H, H, 3 * H * H, 3 * H, H * H, H, H, H, F * H, F, H * F, H]
    return [H, 3 * H * H, H * H, H, 2 * F * H, H * F]


def _sizes(c):
    if c["sizes_seed"] < 0:
        return _layer_sizes(c) * c["layers"]
    rng = np.random.default_rng(c["sizes_seed"])
    n = np.exp(rng.uniform(0.0, math.log(4e6), size=c["layers"]))
    return [int(v) + 1 for v in n]


def _places(c):
    """Where each tensor starts in the flat gradient buffer (16 bytes apart at least), and the buffer's length."""
    at, places = 0, []
    for n in _sizes(c):
        places.append(at)
        at = (at + n + 7) // 8 * 8
    return places, at


# base, factor, low, high, trained context, magnitude of the cosines and sines
SCALING = {"plain": (10000.0, 1.0, 0.0, 0.0, 0.0, 1.0), "linear": (10000.0, 4.0, 0.0, 0.0, 0.0, 1.0),
           "wavelength": (500000.0, 8.0, 1.0, 4.0, 8192.0, 1.0), "ramp": (10000.0, 4.0, 1.0, 32.0, 4096.0, 1.125)}
RESIDUAL_SCALE, BRANCH_SCALE = 0.75, 0.5
MAX_NORM = 1.0
ADAM = dict(lr=3e-4, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.1, grad_scale=0.125, step=100, zero_grad=False)


# ---------------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------------
def _dtype(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _randn(gen, shape, dtype, std=1.0, mean=0.0):
    a = torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)
    return a.mul_(std).add_(mean).to(dtype)


def _join_params(c):
    """Shapes of what the join learns, by name."""
    H, s = c["hidden"], {}
    for n, w in (("post", c["post"]), ("pre", c["pre"])):
        if w != "none":
            s[n + "_w"] = (H,)
        if w == "layer":
            s[n + "_b"] = (H,)
    if c["gate"] != "none":
        s["gate"] = (H,) if c["gate"] == "channel" else (len(_cu(c)) - 1, H)
    return s


def _inputs(c, seed):
    gen = torch.Generator(device="cuda").manual_seed(1000003 * int(seed) + 29)
    dt = _dtype(c)
    if c["what"] == "rotary":
        i = {"x": _randn(gen, (c["tokens"], (c["heads"] + c["other"]) * c["head_dim"]), dt)}
        if c["positions"] == "far":
            i["pos"] = torch.randint(0, 131072, (c["tokens"],), generator=gen, device="cuda", dtype=torch.int32)
        else:
            i["cu"] = torch.from_numpy(_cu(c)).cuda()
        return i
    if c["what"] == "join":
        shape = (c["tokens"], c["hidden"])
        i = {"w": {k: _randn(gen, s, dt, 0.1, 0.5 if k == "gate" else 1.0 if k.endswith("_w") else 0.0) for k, s in _join_params(c).items()}}
        if c["gate"] == "segment":
            i["cu"] = torch.from_numpy(_cu(c)).cuda()
        names = ("x", "b") if c["direction"] == "forward" else ("y", "b", "dy", "dh")
        i.update({k: _randn(gen, shape, dt, 2.0 if k == "b" else 1.0, 0.25 if k in "xyb" else 0.0) for k in names if k != "dh" or c["pre"] != "none"})
        if c["main"]:
            i["main"] = {k: _randn(gen, s, torch.float32, 3.0) for k, s in _join_params(c).items()}
        return i
    places, total = _places(c)
    live = torch.zeros(total, dtype=torch.bool, device="cuda")
    for p, n in zip(places, _sizes(c)):
        live[p:p + n] = True
    i = {"grad": _randn(gen, (total,), torch.float32, 1e-2).mul_(live).to(dt)}
    if c["apply"] == "adam":
        i.update(master=_randn(gen, (total,), torch.float32, 0.02), m=_randn(gen, (total,), torch.float32, 1e-5),
                 v=_randn(gen, (total,), torch.float32, 1e-5).square_().add_(1e-12))
    return i


def _statistics(x, kind):
    """Mean and reciprocal deviation of each row, as a forward pass keeps them."""
    x = x.double()
    mean = x.mean(1) if kind == "layer" else torch.zeros_like(x[:, 0])
    rstd = torch.rsqrt((x - mean[:, None]).square().mean(1) + NORM_EPS)
    return mean.float(), rstd.float()


def prepare(case, seed):
    c, s = dict(case), dict(case=dict(case))
    s.update(_inputs(c, seed))
    if c["what"] == "rotary":
        s["y"] = s["x"] if c["in_place"] else torch.empty((c["tokens"], c["heads"] * c["head_dim"]), dtype=_dtype(c), device="cuda")
    elif c["what"] == "join":
        like = s["b"]
        if c["direction"] == "forward":
            s["out"] = {"y": torch.empty_like(like)}
            if c["pre"] != "none":
                s["out"]["h"] = torch.empty_like(like)
            s["out"].update({n + k: torch.empty(c["tokens"], dtype=torch.float32, device="cuda") for n in ("post", "pre") if c[n] != "none"
                             for k in (("_mean", "_rstd") if c[n] == "layer" else ("_rstd",))})
        else:
            s["out"] = {"dx": torch.empty_like(like), "db": torch.empty_like(like)}
            s["grads"] = s["main"] if c["main"] else {k: torch.empty_like(t) for k, t in s["w"].items()}
            s["stats"] = {}
            for n, t in (("post", s["b"]), ("pre", s["y"])):
                if c[n] != "none":
                    s["stats"][n + "_mean"], s["stats"][n + "_rstd"] = _statistics(t, c[n])
    else:
        s["result"] = torch.zeros(2, dtype=torch.float64, device="cuda")
        s["norm_and_factor"] = s["result"].view(torch.float32)[2:4]
        if c["apply"] == "copy":
            s["clipped"] = torch.zeros(s["grad"].numel(), dtype=torch.float32, device="cuda")
        else:
            s["param"] = torch.zeros(s["grad"].numel(), dtype=torch.bfloat16, device="cuda")
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
    p = {"mm": mm}
    dtype = mm.F32 if c["dtype"] == "f32" else mm.BF16
    if "cu" in s:
        p["batch"] = mm.PackedBatch(_cu(c), cu_dev=s["cu"])
    if c["what"] == "rotary":
        base, factor, low, high, context, magnitude = SCALING[c["scaling"]]
        p["desc"] = mm.make_rope_desc(dtype, c["heads"], c["head_dim"], c["rot"], {"half": mm.ROPE_HALF, "interleaved": mm.ROPE_INTERLEAVED}[c["layout"]],
                                      base, {"plain": mm.ROPE_PLAIN, "linear": mm.ROPE_LINEAR, "wavelength": mm.ROPE_WAVELENGTH,
                                             "ramp": mm.ROPE_RAMP}[c["scaling"]], factor, low, high, context, magnitude)
        p["flags"] = mm.ROPE_GRADIENT if c["gradient"] else 0
    elif c["what"] == "join":
        kind = {"none": mm.NORM_NONE, "rms": mm.NORM_RMS, "layer": mm.NORM_LAYER}
        gate = {"none": mm.GATE_NONE, "channel": mm.GATE_CHANNEL, "segment": mm.GATE_SEGMENT}[c["gate"]]
        p["desc"] = mm.make_residual_norm_desc(dtype, c["hidden"], kind[c["post"]], kind[c["pre"]], gate, NORM_EPS, NORM_EPS, RESIDUAL_SCALE, BRANCH_SCALE)
        p["weights"] = mm.make_residual_norm_weights(s["w"])
        if c["direction"] == "forward":
            p["stats"] = mm.make_residual_norm_stats(s["out"])
        else:
            p["stats"] = mm.make_residual_norm_stats(s["stats"])
            p["grads"] = mm.make_residual_norm_grads(s["grads"])
            p["flags"] = mm.BWD_ACCUMULATE_WGRAD | mm.BWD_WGRAD_F32 if c["main"] else 0
            p["ws_bytes"] = mm.mmtrain_residual_norm_workspace_bytes(p["desc"], c["tokens"])
            p["ws"] = torch.empty(max(p["ws_bytes"], 256), dtype=torch.uint8, device="cuda")
    else:
        places, _ = _places(c)
        views = [s["grad"][a:a + n] for a, n in zip(places, _sizes(c))]
        outs = [s["clipped"][a:a + n] for a, n in zip(places, _sizes(c))] if c["apply"] == "copy" else views
        p["tensors"] = mm.make_grad_tensors(views, outs)
        p["ws_bytes"] = mm.mmtrain_grad_norm_workspace_bytes(len(views))
        p["ws"] = torch.empty(p["ws_bytes"], dtype=torch.uint8, device="cuda")
        p["desc"] = mm.make_adam_desc(**ADAM)
    return p


def _run_own(c, s):
    p = s["plan"]
    mm, batch = p["mm"], p.get("batch")
    if c["what"] == "rotary":
        _check(mm.mmtrain_rope(p["desc"], c["tokens"], batch, s.get("pos"), s["x"], s["x"].shape[1], s["y"], s["y"].shape[1], p["flags"]), "rope")
        return s["y"]
    if c["what"] == "join":
        o = s["out"]
        if c["direction"] == "forward":
            _check(mm.mmtrain_residual_norm_fwd(p["desc"], c["tokens"], batch, p["weights"], s["x"], s["b"], o["y"], o.get("h"), p["stats"]), "residual_norm_fwd")
            return o
        _check(mm.mmtrain_residual_norm_bwd(p["desc"], c["tokens"], batch, p["weights"], s["y"], s["b"], p["stats"], s["dy"], s.get("dh"), o["dx"], o["db"],
                                            p["grads"], p["flags"], p["ws"], p["ws_bytes"]), "residual_norm_bwd")
        return {**o, "grads": s["grads"]}
    _check(mm.mmtrain_grad_norm(p["tensors"], MAX_NORM, s["result"], p["ws"], p["ws_bytes"]), "grad_norm")
    if c["apply"] == "copy":
        _check(mm.mmtrain_grad_clip(p["tensors"], s["result"]), "grad_clip")
        return {"norm_and_factor": s["norm_and_factor"], "clipped": s["clipped"]}
    _check(mm.mmtrain_adam_step_clipped(p["desc"], s["grad"].numel(), s["master"], s["grad"], s["m"], s["v"], s["param"], mm.BF16, s["result"]), "adam_step_clipped")
    return {"norm_and_factor": s["norm_and_factor"], "master": s["master"], "m": s["m"], "v": s["v"], "param": s["param"]}


# ---------------------------------------------------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------------------------------------------------
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


def _rotary_plain(c, s):
    T, d, r, n = c["tokens"], c["head_dim"], c["rot"], c["heads"]
    pos = s["pos"] if "pos" in s else torch.arange(T, device="cuda") - s["cu"][_segment_of(s["cu"], T)]
    angle = pos.double()[:, None, None] * _frequencies(c, pos.device)
    magnitude = SCALING[c["scaling"]][5]
    co, si = (angle.cos() * magnitude).float(), (angle.sin() * (-magnitude if c["gradient"] else magnitude)).float()
    heads = s["x"][:, :n * d].view(T, n, d)
    turned = heads[..., :r].float()
    a, b = (turned[..., :r // 2], turned[..., r // 2:]) if c["layout"] == "half" else (turned[..., 0::2], turned[..., 1::2])
    pair = (a * co - b * si, b * co + a * si)
    turned = torch.cat(pair, dim=-1) if c["layout"] == "half" else torch.stack(pair, dim=-1).flatten(-2)
    y = s["y"][:, :n * d].view(T, n, d)
    y[..., :r] = turned
    if not c["in_place"]:
        y[..., r:] = heads[..., r:]
    return s["y"]


def _norm_plain(x, w, name, kind):
    if kind == "none":
        return x, {}
    mean = x.mean(1, keepdim=True) if kind == "layer" else 0.0
    rstd = torch.rsqrt((x - mean).square().mean(1, keepdim=True) + NORM_EPS)
    out = (x - mean) * rstd * w[name + "_w"].float()
    if kind == "layer":
        return out + w[name + "_b"].float(), {name + "_mean": mean[:, 0], name + "_rstd": rstd[:, 0]}
    return out, {name + "_rstd": rstd[:, 0]}


def _gate_plain(c, s, seg):
    if c["gate"] == "none":
        return torch.ones((), device="cuda")
    return s["w"]["gate"].float()[seg] if c["gate"] == "segment" else s["w"]["gate"].float()


def _norm_back_plain(d_out, x, s, name, kind):
    """Gradient of the input, and of gain and bias, from the statistics that the forward pass kept."""
    mean = s["stats"][name + "_mean"][:, None] if kind == "layer" else 0.0
    rstd = s["stats"][name + "_rstd"][:, None]
    hat = (x - mean) * rstd
    back = d_out * s["w"][name + "_w"].float()
    d_in = back - hat * (back * hat).mean(1, keepdim=True)
    learned = {name + "_w": (d_out * hat).sum(0)}
    if kind == "layer":
        d_in = d_in - back.mean(1, keepdim=True)
        learned[name + "_b"] = d_out.sum(0)
    return d_in * rstd, hat, learned


def _join_plain(c, s):
    dt, seg = _dtype(c), _segment_of(s["cu"], c["tokens"]) if "cu" in s else None
    gate, b = _gate_plain(c, s, seg), s["b"].float()
    if c["direction"] == "forward":
        n, kept = _norm_plain(b, s["w"], "post", c["post"])
        y = RESIDUAL_SCALE * s["x"].float() + BRANCH_SCALE * gate * n
        h, more = _norm_plain(y, s["w"], "pre", c["pre"])
        return {"y": y.to(dt), **({"h": h.to(dt)} if c["pre"] != "none" else {}), **kept, **more}
    dy, g = s["dy"].float(), {}
    if c["pre"] != "none":
        d_in, _, learned = _norm_back_plain(s["dh"].float(), s["y"].float(), s, "pre", c["pre"])
        dy = dy + d_in
        g.update(learned)
    dn = BRANCH_SCALE * gate * dy
    db, n = dn, b
    if c["post"] != "none":
        db, hat, learned = _norm_back_plain(dn, b, s, "post", c["post"])
        g.update(learned)
        n = hat * s["w"]["post_w"].float() + (s["w"]["post_b"].float() if c["post"] == "layer" else 0.0)
    if c["gate"] != "none":
        each = BRANCH_SCALE * n * dy
        if c["gate"] == "segment":
            each = torch.matmul((seg[None, :] == torch.arange(s["w"]["gate"].shape[0], device="cuda")[:, None]).float(), each)
        g["gate"] = each if c["gate"] == "segment" else each.sum(0)
    if c["main"]:
        grads = {k: s["main"][k].add_(t) for k, t in g.items()}
    else:
        grads = {k: t.to(dt) for k, t in g.items()}
    return {"dx": (RESIDUAL_SCALE * dy).to(dt), "db": db.to(dt), "grads": grads}


def _clip_plain(c, s):
    """On the flat buffer, whose gaps are zero: nothing faster can be had from elementary operations on the tensors one by one."""
    norm = s["grad"].double().square_().sum().sqrt()
    factor = torch.where(norm > MAX_NORM, MAX_NORM / norm, torch.ones_like(norm)).float()
    told = torch.stack([norm.float(), factor])
    if c["apply"] == "copy":
        return {"norm_and_factor": told, "clipped": s["grad"].float() * factor}
    a, w, m, v = ADAM, s["master"], s["m"], s["v"]
    g = s["grad"] * (factor * a["grad_scale"])
    m.mul_(a["beta1"]).add_(g * (1 - a["beta1"]))
    v.mul_(a["beta2"]).add_(g * g * (1 - a["beta2"]))
    step = (m / (1 - a["beta1"] ** a["step"])) / ((v / (1 - a["beta2"] ** a["step"])).sqrt() + a["eps"])
    w.sub_((step + w * a["weight_decay"]) * a["lr"])
    return {"norm_and_factor": told, "master": w, "m": m, "v": v, "param": w.to(torch.bfloat16)}


def run(s):
    c = s["case"]
    if own:
        return _run_own(c, s)
    return {"rotary": _rotary_plain, "join": _join_plain, "clip": _clip_plain}[c["what"]](c, s)


# ---------------------------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------------------------------------
def work(case):
    c, e = case, 4 if case["dtype"] == "f32" else 2
    if c["what"] == "rotary":
        pairs = c["tokens"] * c["heads"] * (c["rot"] // 2)
        moved = c["tokens"] * c["heads"] * (c["rot"] if c["in_place"] else c["head_dim"])
        return {"bytes": 2.0 * e * moved + 4 * c["tokens"], "flops": 6.0 * pairs}
    if c["what"] == "join":
        n = c["tokens"] * c["hidden"]
        params = sum(int(np.prod(s)) for s in _join_params(c).values())
        norms = (c["post"] != "none") + (c["pre"] != "none")
        if c["direction"] == "forward":
            return {"bytes": e * (n * (4.0 if c["pre"] != "none" else 3.0) + params), "flops": n * (3.0 + 5 * norms)}
        read = 2 + 2 * (c["pre"] != "none") if c["post"] != "none" or c["gate"] != "none" else 1 + 2 * (c["pre"] != "none")
        return {"bytes": e * (n * (2.0 + read) + params) + params * (8 if c["main"] else e), "flops": n * (4.0 + 12 * norms)}
    n = sum(_sizes(c))
    return {"bytes": n * (e + 4.0) if c["apply"] == "copy" else n * 30.0, "flops": n * (3.0 if c["apply"] == "copy" else 18.0)}


# ---------------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------------------
def _exact_rotary(c, i):
    base, s, low, high, context, magnitude = SCALING[c["scaling"]]
    T, d, r, n = c["tokens"], c["head_dim"], c["rot"], c["heads"]
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
        cu = _cu(c)
        pos = np.concatenate([np.arange(L) for L in np.diff(cu)]).astype(np.float64)
    phi = torch.from_numpy(pos[:, None] * theta[None, :]).cuda()
    turn = magnitude * torch.polar(torch.ones_like(phi), -phi if c["gradient"] else phi)[:, None, :]      # a pair is a complex number
    x = i["x"].double()
    y = x[:, :n * d].reshape(T, n, d).clone()
    part = y[..., :r]
    z = torch.complex(part[..., :r // 2].contiguous(), part[..., r // 2:].contiguous()) if c["layout"] == "half" else \
        torch.view_as_complex(part.reshape(T, n, r // 2, 2).contiguous())
    z = z * turn
    y[..., :r] = torch.cat([z.real, z.imag], -1) if c["layout"] == "half" else torch.view_as_real(z).reshape(T, n, r)
    y = y.reshape(T, n * d)
    return torch.cat([y, x[:, n * d:]], 1) if c["in_place"] else y


def _exact_norm(x, w, name, kind):
    if kind == "none":
        return x, {}
    if kind == "layer":
        mean, var = x.mean(1), x.var(1, unbiased=False)
        return torch.nn.functional.layer_norm(x, (x.shape[1],), w[name + "_w"], w[name + "_b"], NORM_EPS), \
            {name + "_mean": mean, name + "_rstd": (var + NORM_EPS) ** -0.5}
    r = (x.pow(2).sum(1) / x.shape[1] + NORM_EPS) ** -0.5
    return x * r[:, None] * w[name + "_w"], {name + "_rstd": r}


def _exact_join(c, i):
    w = {k: t.double().requires_grad_(True) for k, t in i["w"].items()}
    b = i["b"].double().requires_grad_(True)
    n, kept = _exact_norm(b, w, "post", c["post"])
    if c["gate"] == "segment":
        n = n * torch.cat([w["gate"][k:k + 1].expand(int(L), -1) for k, L in enumerate(np.diff(_cu(c)))], 0)
    elif c["gate"] == "channel":
        n = n * w["gate"]
    if c["direction"] == "forward":
        y = RESIDUAL_SCALE * i["x"].double() + BRANCH_SCALE * n
        h, more = _exact_norm(y, w, "pre", c["pre"])
        out = {"y": y, **({"h": h} if c["pre"] != "none" else {}), **kept, **more}
        return {k: t.detach() for k, t in out.items()}
    y = i["y"].double().requires_grad_(True)
    h, _ = _exact_norm(y, w, "pre", c["pre"])
    (h * i["dh"].double()).sum().backward() if c["pre"] != "none" else None
    dy = i["dy"].double() + (y.grad if y.grad is not None else 0.0)
    (BRANCH_SCALE * n).backward(dy)
    return {"dx": RESIDUAL_SCALE * dy, "db": b.grad, "grads": {k: t.grad + (i["main"][k].double() if c["main"] else 0.0) for k, t in w.items()}}


def _exact_clip(c, i):
    g = i["grad"].double()
    norm = torch.dot(g, g) ** 0.5
    factor = min(1.0, MAX_NORM / float(norm))
    told = torch.tensor([float(norm), factor], dtype=torch.float64, device="cuda")
    if c["apply"] == "copy":
        return {"norm_and_factor": told, "clipped": g * factor}
    a = ADAM
    beta1, beta2, eps, lr, wd = (float(np.float32(a[k])) for k in ("beta1", "beta2", "eps", "lr", "weight_decay"))
    w, m, v = i["master"].double(), i["m"].double(), i["v"].double()
    g = g * (factor * a["grad_scale"])
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    w = w - lr * ((m / (1 - beta1 ** a["step"])) / ((v / (1 - beta2 ** a["step"])).sqrt() + eps) + wd * w)
    return {"norm_and_factor": told, "master": w, "m": m, "v": v, "param": w.clone()}


def exact(case, seed):
    return {"rotary": _exact_rotary, "join": _exact_join, "clip": _exact_clip}[case["what"]](case, _inputs(case, seed))
