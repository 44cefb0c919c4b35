"""How far fp32 cross attention may be off as a whole: cases, and a bound on each result's norm, for the tests on the CPU that show what it tells apart and for
those of the kernels.

A bound on single elements adds up all roundings with the same sign; over tens of thousands of keys it lets through a missing block.  Roundings are
independent instead: at most u = 2^-24 of the value that is rounded, and over k of them a root of k as large.  Of n terms x_i that are each off by e_i u, their
sum is off by u sqrt(sum e_i^2), and by its additions: a chain of c additions rounds partial sums, which grow as the root of their number, by
u sqrt(c) of the root of the sum of the x_i^2 at most.  So with
  score         e = sqrt(sum_f (scale q_f k_f)^2) sqrt(d) + 2 |s|          (a product's and a scale's rounding on top)
  probability   relative: e + |lse| + |s| + 2                              (the difference from the log-sum-exp, the exponential)
  dP, D         e = sqrt(sum_f (dO_f v_f)^2) sqrt(d), with O in v's place for D, which all keys of a row share
each result's norm is off by at most 2 u times the norm of sqrt(k) sqrt(sum over its terms (e_term^2 + x_term^2)): the 2 covers roundings larger than their
root mean square, u / sqrt(3), which is what the argument needs.  k counts the chain: keys (dQ, O: of a wavefront, a quarter of the keys at least; of a lane's own sum) or rows."""
import numpy as np

U = 2.0 ** -24


def runs(lq, lk, pattern="own", tail=0):
    """cu, begin, end, key rows.  own: run s sees piece s; previous: all pieces so far."""
    cu, ck = np.concatenate([[0], np.cumsum(lq)]).astype(np.int32), np.concatenate([[0], np.cumsum(lk)]).astype(np.int32)
    s = np.arange(len(lq))
    return cu, (ck[s] if pattern == "own" else 0 * s).astype(np.int32), ck[s + 1].astype(np.int32), int(ck[-1]) + tail


# query heads, key/value heads, head_dim, runs
CASES = {
    "more tiles than are sorted": (2, 1, 64, runs([2, 1, 3], [45000, 60000, 30001], tail=400)),
    "long walks of single tokens": (8, 2, 128, runs([1, 1, 1], [6000, 1, 9000])),
    "few rows, keys in chunks": (4, 2, 80, runs([20, 1, 0, 7, 3], [1500, 60, 900, 0, 1031], tail=9)),
    "many rows, few keys": (8, 2, 64, runs([900, 5, 450], [100, 70, 100])),
    "many rows, two keys": (6, 1, 112, runs([333, 5, 166], [2, 70, 2])),
    "rows that see earlier keys": (4, 2, 128, runs([900, 300, 64], [100, 100, 100], "previous")),
    "ragged": (4, 2, 48, runs([5, 1, 40, 0, 33, 64, 7, 130], [70, 3, 0, 20, 129, 64, 1, 200])),
    "short runs, keys to a wavefront": (8, 8, 64, runs([3, 0, 2, 6, 1, 4] * 5, [100, 150, 130, 97, 158, 91] * 5, tail=70)),
    "short runs, wide heads": (8, 8, 96, runs([1, 3, 2] * 8, [140, 171, 160] * 8, "previous", tail=3)),
    "long runs": (2, 2, 32, runs([700, 90], [900, 2500], "previous")),
}


def inputs(name, round_to=None):
    nh, nkv, d, (cu, _, _, Tk) = CASES[name]
    rng = np.random.default_rng(len(name))
    x = {n: rng.standard_normal((rows, heads, d)).astype(np.float32)
         for n, rows, heads in (("q", cu[-1], nh), ("k", Tk, nkv), ("v", Tk, nkv), ("do", cu[-1], nh))}
    return x if round_to is None else {n: round_to(a) for n, a in x.items()}


def _each(name):
    nh, nkv, _, (cu, begin, end, _) = CASES[name]
    for a, b, lo, hi in zip(cu[:-1], cu[1:], begin, end):
        if b > a and hi > lo:
            for h in range(nh):
                yield int(a), int(b), int(lo), int(hi), h, h // (nh // nkv)


def forward(name, x, skip=None, dtype=np.float64):
    """(o, lse); skip: keys that are left out.  dtype float32: an evaluation in fp32 throughout."""
    nh, _, d, _ = CASES[name]
    x = {n: a.astype(dtype) for n, a in x.items()}
    o, lse = np.zeros(x["q"].shape, dtype), np.full((nh, len(x["q"])), -np.inf, dtype)
    for a, b, lo, hi, h, g in _each(name):
        s = x["q"][a:b, h] @ x["k"][lo:hi, g].T * dtype(1.0 / np.sqrt(d))
        if skip is not None:
            s[:, max(skip.start - lo, 0):max(skip.stop - lo, 0)] = -np.inf
        top = s.max(1, keepdims=True)
        if np.any(np.isneginf(top)):
            continue
        e = np.exp(s - top)
        total = e.sum(1, keepdims=True)
        o[a:b, h], lse[h, a:b] = e @ x["v"][lo:hi, g] / total, (top + np.log(total))[:, 0]
    return o, lse


def backward(name, x, o, lse, keys=None, rows=None, dtype=np.float64):
    """{dq, dk, dv} from a forward pass's o and lse; keys, rows: those that are left out."""
    d = CASES[name][2]
    x = {n: a.astype(dtype) for n, a in x.items()}
    o, lse, scale = o.astype(dtype), lse.astype(dtype), dtype(1.0 / np.sqrt(d))
    out = {"dq": np.zeros_like(x["q"]), "dk": np.zeros_like(x["k"]), "dv": np.zeros_like(x["v"])}
    for a, b, lo, hi, h, g in _each(name):
        q, k, v, do = x["q"][a:b, h], x["k"][lo:hi, g], x["v"][lo:hi, g], x["do"][a:b, h]
        p = np.exp(q @ k.T * scale - lse[h, a:b, None])
        if keys is not None:
            p[:, max(keys.start - lo, 0):max(keys.stop - lo, 0)] = 0
        if rows is not None:
            p[max(rows.start - a, 0):max(rows.stop - a, 0)] = 0
        ds = p * (do @ v.T - (do * o[a:b, h]).sum(1, keepdims=True))
        out["dq"][a:b, h] += scale * (ds @ k)
        out["dk"][lo:hi, g] += scale * (ds.T @ q)
        out["dv"][lo:hi, g] += p.T @ do
    return out


def bounds(name, x):
    """For each of o, lse, dq, dk and dv the bound on the norm of its error."""
    nh, nkv, d, (cu, begin, end, _) = CASES[name]
    o, lse = forward(name, x)
    x = {n: a.astype(np.float64) for n, a in x.items()}
    scale = 1.0 / np.sqrt(d)
    seen = int(max((end - begin).max(), 1))
    by_keys, by_rows = seen / 4 + d + 64, int(cu[-1]) * nh // nkv + d + 64
    sq = {n: np.zeros(a.shape) for n, a in (("o", x["q"]), ("dq", x["q"]), ("dk", x["k"]), ("dv", x["v"]), ("lse", lse))}
    for a, b, lo, hi, h, g in _each(name):
        q, k, v, do = x["q"][a:b, h], x["k"][lo:hi, g], x["v"][lo:hi, g], x["do"][a:b, h]
        s = q @ k.T * scale
        L = lse[h, a:b, None]
        p = np.exp(s - L)
        es = np.sqrt((q * q) @ (k * k).T * d) * scale + 2 * np.abs(s)
        ep = es + np.abs(L) + np.abs(s) + 2
        total = ((p * es) ** 2).sum(1, keepdims=True)                 # what the scores do to the sum that divides
        sq["o"][a:b, h] += (p * ep) ** 2 @ v ** 2 + by_keys * (p ** 2 @ v ** 2) + (total + by_keys) * o[a:b, h] ** 2
        sq["lse"][h, a:b] += (total + by_keys)[:, 0] + (4 * L[:, 0]) ** 2
        D = (do * o[a:b, h]).sum(1, keepdims=True)
        ds = p * (do @ v.T - D)
        eD2 = (do * do * o[a:b, h] ** 2).sum(1, keepdims=True) * d
        eds2 = (p ** 2) * ((do * do) @ (v * v).T * d) + (ds * ep) ** 2
        sq["dq"][a:b, h] += scale ** 2 * ((eds2 + by_keys * ds ** 2) @ k ** 2 + eD2 * (p @ k) ** 2)
        sq["dk"][lo:hi, g] += scale ** 2 * ((eds2 + p ** 2 * eD2 + by_rows * ds ** 2).T @ q ** 2)
        sq["dv"][lo:hi, g] += ((p * ep) ** 2 + by_rows * p ** 2).T @ do ** 2
    return {n: 2 * U * float(np.sqrt(e[np.isfinite(e)].sum())) for n, e in sq.items()}


def too_far(got, ref, bound):
    """The error's norm in units of its bound (1 and less: within it).  Rows that see nothing have the log-sum-exp -infinity in both."""
    got, ref = np.asarray(got, np.float64), np.asarray(ref, np.float64)
    same = np.isneginf(got) & np.isneginf(ref)
    with np.errstate(invalid="ignore"):
        r = np.linalg.norm(np.where(same, 0.0, got - ref)) / bound
    return r if np.isfinite(r) else np.inf
