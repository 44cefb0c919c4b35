"""What the bounds of cross_precision.py tell apart: an evaluation in fp32 is within them, and for each case a lost block of 16 keys or rows, a missing
gradient and inputs in fewer bits are behind them."""
import numpy as np
import pytest
import torch

import cross_precision as cp


def bf16(a):
    return torch.from_numpy(a).to(torch.bfloat16).float().numpy()


@pytest.mark.parametrize("name", list(cp.CASES))
def test_the_bounds_take_fp32_and_no_mistake(name):
    _, _, _, (cu, begin, end, _) = cp.CASES[name]
    x = cp.inputs(name)
    bound = cp.bounds(name, x)
    ref = dict(zip(("o", "lse"), cp.forward(name, x)))
    # the backward pass starts from what forward stored
    stored = {n: a.astype(np.float32) for n, a in ref.items()}
    ref.update(cp.backward(name, x, stored["o"], stored["lse"]))
    far = lambda got: {n: cp.too_far(a, ref[n], bound[n]) for n, a in got.items()}  # noqa: E731
    right = dict(zip(("o", "lse"), cp.forward(name, x, dtype=np.float32)))
    right.update(cp.backward(name, x, stored["o"], stored["lse"], dtype=np.float32))
    assert all(v <= 1 for v in far(right).values()), far(right)

    def wrong(what, got):
        low = {n: v for n, v in far(got).items() if not v > 2}
        assert not low, (what, low)
    wrong("zeros", {n: np.zeros_like(a) for n, a in ref.items()})
    rounded = cp.inputs(name, bf16)
    o, lse = cp.forward(name, rounded)
    some = {"o": o, "lse": lse}
    some.update(cp.backward(name, rounded, stored["o"], stored["lse"]))
    wrong("inputs in bf16", some)
    # a block of 16 keys (or as many as there are) in the middle of the longest range, a block of 16 rows of the longest run
    s = int(np.argmax((end - begin) * (np.diff(cu) > 0)))
    first = int(begin[s] + (end[s] - begin[s]) // 32 * 16)
    keys = slice(first, min(first + 16, int(end[s])))
    if end[s] - begin[s] > 16:
        o, lse = cp.forward(name, x, keys)
        wrong("lost keys, forward", {"o": o, "lse": lse})
    wrong("lost keys, backward", cp.backward(name, x, stored["o"], stored["lse"], keys=keys))
    r = int(np.argmax(np.diff(cu) * (end > begin)))
    rows = slice(int(cu[r]), min(int(cu[r]) + 16, int(cu[r + 1])))
    wrong("lost rows", cp.backward(name, x, stored["o"], stored["lse"], rows=rows))
