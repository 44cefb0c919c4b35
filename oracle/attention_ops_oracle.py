"""Plain fp64 definitions of the embedding of a pack, of per-head norms of queries and keys with their rotation, and of attention from runs of
queries to ranges of keys, each with its gradients.

Beside each result stand sums of the absolute values of the terms that make it up, to which an evaluation's rounding errors are proportional
however much the terms cancel: `mag` for roundings of fp32 arithmetic, and where an intermediate may be kept in the storage type (the
probabilities and their gradients, as operands of a matrix product) `stored` for those.
"""
import numpy as np

from oracle.operators_oracle import rope

F64 = np.float64


# ---- embedding -----------------------------------------------------------------------------------------------------
def embed_source(ids, vocab, n_features):
    """Row of [table; features] that each token starts from, -1 for none."""
    ids = np.asarray(ids, np.int64)
    return np.where((ids >= 0) & (ids < vocab), ids, np.where((ids < 0) & (ids >= -n_features), vocab - 1 - ids, -1))


def embed_fwd(ids, table, features, scale):
    table = np.asarray(table, F64)
    features = np.zeros((0, table.shape[1])) if features is None else np.asarray(features, F64)
    src = embed_source(ids, len(table), len(features))
    rows = np.concatenate([table * scale, features, np.zeros((1, table.shape[1]))])
    return rows[src]


def embed_bwd(ids, dy, vocab, n_features, scale):
    """(d_table, d_features) and their mags."""
    dy = np.asarray(dy, F64)
    src = embed_source(ids, vocab, n_features)
    out, mag = np.zeros((vocab + n_features + 1, dy.shape[1])), np.zeros((vocab + n_features + 1, dy.shape[1]))
    np.add.at(out, src, dy)
    np.add.at(mag, src, np.abs(dy))
    return (out[:vocab] * scale, out[vocab:-1]), (mag[:vocab] * abs(scale), mag[vocab:-1])


# ---- norms of queries and keys, rotation -----------------------------------------------------------------------------
def _stats(x, norm, eps):
    mean = x.mean(-1, keepdims=True) if norm == "layer" else np.zeros(x.shape[:-1] + (1,))
    return mean, 1.0 / np.sqrt(((x - mean) ** 2).mean(-1, keepdims=True) + eps)


def _mean_mag(x, norm):
    """What the mean's rounding errors are proportional to: each of its additions rounds a partial sum, which is at most the sum of the absolute values
    (the mean itself may be as small as it likes)."""
    return np.abs(x).mean(-1, keepdims=True) if norm == "layer" else 0.0


def _gains(w, name, nq, nk, d, default):
    return np.concatenate([np.broadcast_to(np.asarray(w.get(k + name, np.full(d, default)), F64), (h, d)) for k, h in (("q", nq), ("k", nk))])


def qk_norm_fwd(x, w, nq, nk, norm, eps, turn=None):
    """x: [T, nq + nk, d]; turn: (positions, theta, layout, magnitude) or None.  Returns (y, mag)."""
    x = np.asarray(x, F64)
    d = x.shape[-1]
    mean, r = _stats(x, norm, eps)
    gain, bias = _gains(w, "_w", nq, nk, d, 1.0), _gains(w, "_b", nq, nk, d, 0.0)
    y = (x - mean) * r * gain + bias
    mag = (np.abs(x) + _mean_mag(x, norm)) * r * np.abs(gain) + np.abs(bias)
    if turn is None:
        return y, mag
    pos, theta, layout, m = turn
    return rope(y, pos, theta, layout, m)[0], rope_mag(mag, theta, layout, m)


def rope_mag(mag, theta, layout, m):
    half = len(theta)
    out = mag.copy()
    first, second = (slice(0, half), slice(half, 2 * half)) if layout == "half" else (slice(0, 2 * half, 2), slice(1, 2 * half, 2))
    out[..., first] = out[..., second] = m * (mag[..., first] + mag[..., second])
    return out


def qk_norm_bwd(x, dy, w, nq, nk, norm, eps, turn=None):
    """Returns (results, mags) by name: dx, q_w, q_b, k_w, k_b (those that there are)."""
    x, g = np.asarray(x, F64), np.asarray(dy, F64)
    d = x.shape[-1]
    mg = np.abs(g)
    if turn is not None:
        pos, theta, layout, m = turn
        g, mg = rope(g, pos, theta, layout, m, gradient=True)[0], rope_mag(mg, theta, layout, m)
    mean, r = _stats(x, norm, eps)
    hat, mhat = (x - mean) * r, (np.abs(x) + _mean_mag(x, norm)) * r
    gain = _gains(w, "_w", nq, nk, d, 1.0)
    back, mback = g * gain, mg * np.abs(gain)
    s1, ms1 = (back * hat).mean(-1, keepdims=True), (mback * mhat).mean(-1, keepdims=True)
    s0, ms0 = (back.mean(-1, keepdims=True), mback.mean(-1, keepdims=True)) if norm == "layer" else (0.0, 0.0)
    out, mag = {"dx": r * (back - s0 - hat * s1)}, {"dx": r * (mback + ms0 + mhat * ms1)}
    for name, part in (("q", slice(0, nq)), ("k", slice(nq, nq + nk))):
        if part.stop > part.start:
            out[name + "_w"], mag[name + "_w"] = (g * hat)[:, part].sum((0, 1)), (mg * mhat)[:, part].sum((0, 1))
            if norm == "layer":
                out[name + "_b"], mag[name + "_b"] = g[:, part].sum((0, 1)), mg[:, part].sum((0, 1))
    return out, mag


# ---- attention from runs of queries to ranges of keys ------------------------------------------------------------------
def _runs(cu, begin, end):
    return [(int(a), int(b), int(lo), int(hi)) for a, b, lo, hi in zip(cu[:-1], cu[1:], begin, end) if b > a and hi > lo]


def cross_fwd(q, k, v, cu, begin, end, scale):
    """q: [Tq, nh, d]; k, v: [Tk, nkv, d].  Returns (o [Tq, nh, d], lse [nh, Tq]), then mag and stored for o, mag for lse."""
    q, k, v = (np.asarray(a, F64) for a in (q, k, v))
    nh, group = q.shape[1], q.shape[1] // k.shape[1]
    o, lse = np.zeros(q.shape), np.full((nh, len(q)), -np.inf)
    mag, stored, mlse = np.zeros(q.shape), np.zeros(q.shape), np.zeros((nh, len(q)))
    for a, b, lo, hi in _runs(cu, begin, end):
        for h in range(nh):
            kk, vv, qq = k[lo:hi, h // group], v[lo:hi, h // group], q[a:b, h]
            s = qq @ kk.T * scale
            ms = np.abs(qq) @ np.abs(kk).T * scale
            top = s.max(1, keepdims=True)
            e = np.exp(s - top)
            p = e / e.sum(1, keepdims=True)
            o[a:b, h], lse[h, a:b] = p @ vv, (top + np.log(e.sum(1, keepdims=True)))[:, 0]
            mean = (p * ms).sum(1, keepdims=True)                     # what the scores' errors do to the sum that divides
            stored[a:b, h] = p @ np.abs(vv)
            mag[a:b, h] = (p * (ms + mean)) @ np.abs(vv) + stored[a:b, h]
            mlse[h, a:b] = mean[:, 0] + np.abs(lse[h, a:b]) + np.log(hi - lo) + 1.0
    return (o, lse), (mag, stored, mlse)


def cross_bwd(q, k, v, o, lse, do, cu, begin, end, scale):
    """From the forward pass's o and lse as they are stored.  Returns {dq, dk, dv}, their mags, and their `stored`."""
    q, k, v, o, lse, do = (np.asarray(a, F64) for a in (q, k, v, o, lse, do))
    nh, group = q.shape[1], q.shape[1] // k.shape[1]
    out = {"dq": np.zeros(q.shape), "dk": np.zeros(k.shape), "dv": np.zeros(k.shape)}
    mag, stored = ({n: np.zeros(a.shape) for n, a in out.items()} for _ in range(2))
    for a, b, lo, hi in _runs(cu, begin, end):
        for h in range(nh):
            g = h // group
            qq, kk, vv, dd = q[a:b, h], k[lo:hi, g], v[lo:hi, g], do[a:b, h]
            s, ms = qq @ kk.T * scale, np.abs(qq) @ np.abs(kk).T * scale
            p = np.exp(s - lse[h, a:b, None])
            dp, mdp = dd @ vv.T, np.abs(dd) @ np.abs(vv).T
            D, mD = (dd * o[a:b, h]).sum(1, keepdims=True), (np.abs(dd) * np.abs(o[a:b, h])).sum(1, keepdims=True)
            ds = p * (dp - D)
            slack = ms + np.abs(lse[h, a:b, None]) + 1.0              # relative error of p in units of fp32 roundings
            mds = p * (mdp + mD) + np.abs(ds) * slack
            out["dq"][a:b, h] += scale * ds @ kk
            mag["dq"][a:b, h] += scale * mds @ np.abs(kk)
            stored["dq"][a:b, h] += scale * np.abs(ds) @ np.abs(kk)
            out["dk"][lo:hi, g] += scale * ds.T @ qq
            mag["dk"][lo:hi, g] += scale * mds.T @ np.abs(qq)
            stored["dk"][lo:hi, g] += scale * np.abs(ds).T @ np.abs(qq)
            out["dv"][lo:hi, g] += p.T @ dd
            mag["dv"][lo:hi, g] += (p * slack).T @ np.abs(dd)
            stored["dv"][lo:hi, g] += p.T @ np.abs(dd)
    return out, mag, stored
