"""Plain fp64 definitions of the operators around a block's products: rotary positions, the join of a block's branch with the
residual stream, gradient norm and clipping.

Rotary positions and the join return, beside each result, the sum of the absolute values of the terms that make it up (`mag`): what
an fp32 evaluation's rounding errors are proportional to, however much the terms cancel.
"""
import numpy as np

F64 = np.float64


# ---- rotary positions ---------------------------------------------------------------------------------------------
def rope_frequencies(rot_dim, base, scaling="plain", factor=1.0, low=0.0, high=0.0, orig_context=0.0):
    """Angle per position of each rotated pair, [rot_dim / 2]."""
    i = np.arange(rot_dim // 2, dtype=F64)
    theta = F64(base) ** (-2.0 * i / rot_dim)
    if scaling == "plain":
        return theta
    if scaling == "linear":
        return theta / factor
    if scaling == "wavelength":
        turns = orig_context * theta / (2 * np.pi)
        keep = np.clip((turns - low) / (high - low), 0.0, 1.0)
    elif scaling == "ramp":
        index = lambda n: rot_dim * np.log(orig_context / (2 * np.pi * n)) / (2 * np.log(F64(base)))  # noqa: E731
        first, last = max(np.floor(index(high)), 0.0), min(np.ceil(index(low)), rot_dim - 1.0)
        keep = 1.0 - np.clip((i - first) / max(last - first, 1e-3), 0.0, 1.0)
    else:
        raise ValueError(scaling)
    return theta * (keep + (1.0 - keep) / factor)


def segment_positions(cu):
    return np.concatenate([np.arange(b - a) for a, b in zip(cu[:-1], cu[1:])] + [np.zeros(0, int)]).astype(np.int64)


def rope(x, positions, theta, layout="half", magnitude=1.0, gradient=False):
    """x: [T, heads, head_dim]; the first 2 len(theta) features of a head are rotated.  Returns (y, mag)."""
    x = np.asarray(x, F64)
    half = len(theta)
    phi = np.asarray(positions, F64)[:, None, None] * theta
    c, s = magnitude * np.cos(phi), magnitude * np.sin(phi) * (-1.0 if gradient else 1.0)
    first, second = (slice(0, half), slice(half, 2 * half)) if layout == "half" else (slice(0, 2 * half, 2), slice(1, 2 * half, 2))
    a, b = x[..., first], x[..., second]
    y, mag = x.copy(), np.abs(x)
    y[..., first], y[..., second] = a * c - b * s, b * c + a * s
    mag[..., first] = mag[..., second] = magnitude * (np.abs(a) + np.abs(b))
    return y, mag


# ---- the join of branch and residual stream ------------------------------------------------------------------------
def norm_statistics(v, kind, eps):
    v = np.asarray(v, F64)
    mean = v.mean(1, keepdims=True) if kind == "layer" else np.zeros((len(v), 1))
    return mean, 1.0 / np.sqrt(((v - mean) ** 2).mean(1, keepdims=True) + eps)


def _rows(gate, cu):
    """A gate per token: [H] for all, or [S, H] by segment."""
    return gate if cu is None or gate is None else np.repeat(gate, np.diff(cu), axis=0)


def join_fwd(x, branch, w, post="none", pre="none", post_eps=1e-5, pre_eps=1e-5, alpha=1.0, beta=1.0, cu=None):
    """w: post_w, post_b, gate, pre_w, pre_b (those that there are); cu: the gate is by segment.  Returns (results, mags) by name."""
    x = np.asarray(x, F64)
    out, mag = {}, {}
    if branch is None:
        y, my = x, np.abs(x)
    else:
        n, mn = np.asarray(branch, F64), np.abs(branch)
        if post != "none":
            mu, r = norm_statistics(n, post, post_eps)
            mn = (mn + np.abs(mu)) * r * np.abs(w["post_w"]) + (np.abs(w["post_b"]) if post == "layer" else 0.0)
            n = (n - mu) * r * w["post_w"] + (w["post_b"] if post == "layer" else 0.0)
            out["post_mean"], out["post_rstd"] = mu[:, 0], r[:, 0]
        gate = _rows(w.get("gate"), cu)
        gate = 1.0 if gate is None else gate
        y, my = alpha * x + beta * gate * n, abs(alpha) * np.abs(x) + np.abs(beta * gate) * mn
        out["y"], mag["y"] = y, my
    if pre != "none":
        mu, r = norm_statistics(y, pre, pre_eps)
        out["pre_mean"], out["pre_rstd"] = mu[:, 0], r[:, 0]
        bias = w["pre_b"] if pre == "layer" else 0.0
        out["h"] = (y - mu) * r * w["pre_w"] + bias
        # an error of y moves h directly and through the statistics
        rms = np.sqrt((my ** 2).mean(1, keepdims=True))
        mag["h"] = r * np.abs(w["pre_w"]) * (my + rms + np.abs((y - mu) * r) * rms) + np.abs(bias)
    return out, mag


def _norm_back(d, md, v, mu, r, gain, kind):
    """Input gradient of a norm for the output gradient d (mags md), and the normalised values."""
    hat, mhat = (v - mu) * r, (np.abs(v) + np.abs(mu)) * r
    back, mback = d * gain, md * np.abs(gain)
    s1, ms1 = (back * hat).mean(1, keepdims=True), (mback * mhat).mean(1, keepdims=True)
    s0, ms0 = (back.mean(1, keepdims=True), mback.mean(1, keepdims=True)) if kind == "layer" else (0.0, 0.0)
    return r * (back - s0 - hat * s1), r * (mback + ms0 + mhat * ms1), hat, mhat


def join_bwd(y, branch, w, stats, dy, dh, post="none", pre="none", alpha=1.0, beta=1.0, cu=None):
    """stats: the forward pass's means and reciprocal deviations, [T] each.  Returns (results, mags): dx, d_branch, parameters."""
    out, mag = {}, {}
    col = lambda k: np.asarray(stats[k], F64)[:, None]  # noqa: E731
    d = np.zeros_like(np.asarray(dh if dy is None else dy, F64)) if dy is None else np.asarray(dy, F64)
    md = np.abs(d)
    if pre != "none":
        dh, y = np.asarray(dh, F64), np.asarray(y, F64)
        d_in, md_in, hat, mhat = _norm_back(dh, np.abs(dh), y, col("pre_mean") if pre == "layer" else 0.0, col("pre_rstd"), w["pre_w"], pre)
        d, md = d + d_in, md + md_in
        out["pre_w"], mag["pre_w"] = (dh * hat).sum(0), (np.abs(dh) * mhat).sum(0)
        if pre == "layer":
            out["pre_b"], mag["pre_b"] = dh.sum(0), np.abs(dh).sum(0)
    if branch is None:
        out["dx"], mag["dx"] = d, md
        return out, mag
    out["dx"], mag["dx"] = alpha * d, abs(alpha) * md
    b = np.asarray(branch, F64)
    gate = _rows(w.get("gate"), cu)
    g1 = 1.0 if gate is None else gate
    dn, mdn = beta * g1 * d, np.abs(beta * g1) * md
    n, mn, db, mdb = b, np.abs(b), dn, mdn
    if post != "none":
        db, mdb, hat, mhat = _norm_back(dn, mdn, b, col("post_mean") if post == "layer" else 0.0, col("post_rstd"), w["post_w"], post)
        out["post_w"], mag["post_w"] = (dn * hat).sum(0), (mdn * mhat).sum(0)
        n, mn = hat * w["post_w"], mhat * np.abs(w["post_w"])
        if post == "layer":
            out["post_b"], mag["post_b"] = dn.sum(0), mdn.sum(0)
            n, mn = n + w["post_b"], mn + np.abs(w["post_b"])
    out["d_branch"], mag["d_branch"] = db, mdb
    if gate is not None:
        each, meach = beta * n * d, abs(beta) * mn * md
        if cu is None:
            out["gate"], mag["gate"] = each.sum(0), meach.sum(0)
        else:
            out["gate"] = np.stack([each[p:q].sum(0) for p, q in zip(cu[:-1], cu[1:])])
            mag["gate"] = np.stack([meach[p:q].sum(0) for p, q in zip(cu[:-1], cu[1:])])
    return out, mag


# ---- gradient norm and clipping ------------------------------------------------------------------------------------
def grad_norm(grads, max_norm, start=0.0):
    """(sum of squares, norm, factor) of a list of arrays; start: a sum of squares to add to."""
    q = start + sum(float(np.sum(np.asarray(g, F64) ** 2)) for g in grads)
    norm = float(np.sqrt(q))
    if not norm <= np.finfo(np.float32).max:              # the norm is handed out in fp32
        return q, norm, float("nan")
    return q, norm, max_norm / norm if norm > max_norm else 1.0
