"""The join of branch and residual stream on packs long enough that every workgroup walks over several rows, changes segment inside its range
and shares segments with others; tolerances as in test_gpu_operators.py, from the same counts of roundings."""
import numpy as np
import pytest
import torch

from paper_2408_04275_amd import binding as mm
from paper_2408_04275_amd.harness import check
from test_gpu_operators import MAIN, U, close, host, join_case

pytestmark = pytest.mark.gpu


def ragged(T, S, seed, step=1):
    """S segments of any length (a few of them empty), with boundaries at multiples of `step`."""
    rng = np.random.default_rng(seed)
    cuts = step * np.sort(rng.integers(0, T // step + 1, size=S - 1))
    cuts[1::9] = cuts[::9][:len(cuts[1::9])]
    return np.concatenate([[0], np.sort(cuts), [T]]).astype(np.int32)


# forward takes up to as many workgroups as the 256 compute units hold (at most 2048 threads each): so many rows that each has two or more in turn
@pytest.mark.parametrize("T,H", [(20011, 512), (10007, 1016), (6011, 1280), (5003, 2040), (2503, 4096), (2003, 4104), (2003, 5120), (1601, 8192)])
@pytest.mark.parametrize("dtype", [mm.BF16, mm.F32])
def test_join_layer_norms_and_segment_gates_over_several_rows_a_workgroup(dtype, T, H):
    join_case(dtype, T, H, "layer", "layer", "segment", ragged(T, 150, H), flags=mm.BWD_WGRAD_F32, seed=31)


@pytest.mark.parametrize("T,H", [(2003, 5120), (1601, 8192)])
def test_join_other_wide_forms_over_several_rows_a_workgroup(T, H):
    join_case(mm.BF16, T, H, "layer", "rms", "channel", flags=MAIN, seed=32)
    join_case(mm.BF16, T, H, "none", "layer", "channel", seed=33)


# Backward has one workgroup per compute unit, 2400 rows make nine or ten a workgroup and 2560 make ten: most of these segments are shared by several
# workgroups, more of them than the summing launch takes in one turn; `step` lets them begin and end where workgroups' ranges do
@pytest.mark.parametrize("flags", [0, mm.BWD_WGRAD_F32, mm.BWD_ACCUMULATE_WGRAD, MAIN])
@pytest.mark.parametrize("H", [1280, 4096])
def test_join_gate_gradients_of_segments_that_workgroups_share(H, flags):
    for T, S, step in ((2400, 40, 1), (2400, 100, 1), (2560, 60, 10)):
        join_case(mm.BF16, T, H, "layer", "layer", "segment", ragged(T, S, S + step, step), flags=flags, seed=34)
    join_case(mm.F32, 2400, H, "none", "rms", "segment", ragged(2400, 100, 5), flags=flags, seed=35)


def test_join_gradients_of_sixty_thousand_rows():
    join_case(mm.F32, 60000, 64, "rms", "layer", "channel", seed=36)
    join_case(mm.F32, 60000, 64, "layer", "layer", "segment", ragged(60000, 300, 6), flags=MAIN, seed=37)


@pytest.mark.parametrize("T,H,rows", [(400009, 64, 8), (200003, 2056, 1)])
def test_join_gradients_of_long_packs_of_one_sign(T, H, rows):
    # A thread adds up T / 256 / rows rows (`rows` of them at once in a workgroup), then the rows' threads and 256 workgroups are joined:
    # a summand passes through T / 256 / rows + rows + 40 additions and is off by 128 itself.  Summands of one sign, where nothing cancels.
    gen = torch.Generator(device="cuda").manual_seed(38)
    dh = torch.randn((T, H), generator=gen, device="cuda").abs_().add_(0.5)
    y = torch.randn((T, H), generator=gen, device="cuda").add_(0.25)
    w = {"pre_w": torch.randn(H, generator=gen, device="cuda"), "pre_b": torch.zeros(H, device="cuda")}
    mean = torch.cat([p.double().mean(1) for p in y.split(1 << 15)])
    rstd = torch.cat([(p.double().var(1, correction=0) + 1e-5).rsqrt() for p in y.split(1 << 15)])
    stats = {"pre_mean": mean.float(), "pre_rstd": rstd.float()}
    ref, mag = ({k: np.zeros(H) for k in w} for _ in range(2))
    for p, q, mu, r in zip(y.split(1 << 15), dh.split(1 << 15), stats["pre_mean"].double().split(1 << 15), stats["pre_rstd"].double().split(1 << 15)):
        p, q, mu, r = p.double(), q.double(), mu[:, None], r[:, None]
        ref["pre_w"] += host((q * (p - mu) * r).sum(0))
        mag["pre_w"] += host((q * (p.abs() + mu.abs()) * r).sum(0))
        ref["pre_b"] += host(q.sum(0))
        mag["pre_b"] += host(q.sum(0))
    desc = mm.make_residual_norm_desc(mm.F32, H, pre_norm=mm.NORM_LAYER)
    grads = {k: torch.full((H,), 9.0, device="cuda") for k in w}
    wsb = mm.mmtrain_residual_norm_workspace_bytes(desc, T)
    ws = torch.full((wsb,), 255, dtype=torch.uint8, device="cuda")
    dx = torch.empty_like(y)
    check(mm.mmtrain_residual_norm_bwd(desc, T, None, mm.make_residual_norm_weights(w), y, None, mm.make_residual_norm_stats(stats), None, dh, dx, None,
                                       mm.make_residual_norm_grads(grads), 0, ws, wsb), "bwd")
    k = 128 + T / 256 / rows + rows + 40
    for name in w:
        close(name, grads[name], ref[name], mag[name], k, mm.F32)
        print(name, float(np.max(np.abs(host(grads[name]) - ref[name]) / (U * mag[name]))), "x 2^-24 of the summands")
