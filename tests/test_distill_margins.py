"""Distillation with the teacher's logsumexp where the listed items stand far above the others: the mass off the list is below what 32 bits hold
beside the listed mass, loss and gradient are as finite as the definition's."""
import numpy as np
import pytest

import block_reference as ref
from test_distill import EPS, PAD, _case, _check, _run, _torch

gpu = pytest.mark.gpu
SHAPES = [(3, 999), (3, 100_003), (300, 2049), (300, 20_001), (2, 300_001)]


def _types(torch):
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def _far(R, V, gap, seed):
    """Logits whose listed items stand `gap` above the others under a scale of one; every eleventh item off the list masked."""
    xs, ids, values, lse, g = _case(R, V, 20, seed, rest=True, sharp=0.0)
    lse = (lse + 0.25).astype(np.float32)                      # a fifth of the mass at least: one minus a sum holds it to 2^-20 of itself
    xs[:, ::11] = -np.inf
    for r in range(R):
        at = ids[r][ids[r] != PAD].astype(np.int64)
        xs[r, at] = gap + 0.25 * np.arange(len(at), dtype=np.float32)
    return xs, ids, values, lse, g


@gpu
@pytest.mark.parametrize("R,V", SHAPES)
@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("gap", [80.0, 90.0, 200.0])
@pytest.mark.parametrize("loss_scale", [1.0, 1e6])
def test_the_mass_off_the_list_at_any_distance(R, V, kind, gap, loss_scale):
    torch, b = _torch()
    xs, ids, values, lse, g = _far(R, V, gap, V + int(gap))
    if kind == "f16":
        loss_scale = min(loss_scale, 64.0)
    g = (g * loss_scale).astype(np.float32)
    x = torch.from_numpy(xs).cuda().to(_types(torch)[kind])
    xs = x.float().cpu().numpy()
    for how in ("fused", "apart"):
        got = _run(torch, b, x, ids, values, lse, g, 1.0, -1.5, how)
        _check(*got, xs, ids, values, lse, g, 1.0, -1.5, kind)
    placed = _run(torch, b, x.clone(), ids, values, lse, g, 1.0, -1.5, in_place=True)
    _check(*placed, xs, ids, values, lse, g, 1.0, -1.5, kind)


@gpu
@pytest.mark.parametrize("V", [999, 100_003])
@pytest.mark.parametrize("scale", [0.5, 100.0])
def test_tied_listed_items_and_one_other_at_the_edge_of_32_bits(V, scale):
    """Dozens of tied listed items, one item off the list 87 below them, the rest far below that: p_r / q_r is beyond 32 bits."""
    torch, b = _torch()
    xs = np.full((3, V), -150.0, dtype=np.float32) / scale
    ids = np.tile(np.arange(100, 148, dtype=np.uint32), (3, 1))
    values = np.full((3, 48), 1.0, dtype=np.float32)
    xs[:, 100:148] = 0.0
    xs[0, 7], xs[1, 7], xs[2, 7] = -86.0 / scale, -87.2 / scale, -95.0 / scale
    lse = np.full(3, np.log(48.0) - 1.5 + 0.105, dtype=np.float32)
    g = np.float32([1.0, 1e4, 1.0])
    for how in ("fused", "apart"):
        got = _run(torch, b, torch.from_numpy(xs).cuda(), ids, values, lse, g, scale, -1.5, how)
        _check(*got, xs, ids, values, lse, g, scale, -1.5, "f32")
        assert np.isfinite(got[0]).all() and np.isfinite(got[1]).all()
        left = got[1][:, 7] / (g * scale)                     # all of -p_r lands on the one item above the rest
        p_r = 1.0 - 48.0 * np.exp(-1.5 - lse.astype(np.float64))
        assert (np.abs(left + p_r) <= 1e-5).all()


@gpu
@pytest.mark.parametrize("how", ["fused", "apart"])
def test_one_listed_item_a_hundred_above(how):
    """One listed item at 100, 999 others at 0, a tenth of the mass off the list: loss 0.9 log 0.9 + 0.1 (log 0.1 - log q_r), the others share -0.1."""
    torch, b = _torch()
    xs = np.zeros((1, 1000), dtype=np.float32)
    xs[0, 3] = 100.0
    ids, values = np.uint32([[3]]), np.float32([[1.0]])
    lse = np.float32([-1.0 - np.log(0.9)])
    loss, grad = _run(torch, b, torch.from_numpy(xs).cuda(), ids, values, lse, None, 1.0, -1.0, how)
    want = 0.9 * np.log(0.9) + 0.1 * (np.log(0.1) - (np.log(999.0) - 100.0))
    assert abs(loss[0] - want) <= EPS * 600 * want
    assert abs(np.delete(grad[0], 3).sum() + 0.1) <= 1e-5 and abs(grad[0, 3] - 0.1) <= 1e-6


@gpu
@pytest.mark.parametrize("how", ["fused", "apart"])
def test_nothing_finite_off_the_list_is_still_an_infinite_loss(how):
    torch, b = _torch()
    xs = np.full((2, 5000), -np.inf, dtype=np.float32)
    ids, values = np.uint32([[5, 4000], [0, 4999]]), np.float32([[1.0, 2.0], [1.0, 2.0]])
    for r in range(2):
        xs[r, ids[r].astype(np.int64)] = (30.0, -200.0)
    z = np.exp(-values.astype(np.float64)).sum(1)
    lse = (np.log(z) + 0.2).astype(np.float32)
    loss, grad = _run(torch, b, torch.from_numpy(xs).cuda(), ids, values, lse, None, 1.0, -1.0, how)
    _check(loss, grad, xs, ids, values, lse, None, 1.0, -1.0, "f32")
    assert (loss == np.inf).all() and np.isfinite(grad).all()


@gpu
@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("R,V", [(2, 1000), (2, 100_003), (300, 1500)])
@pytest.mark.parametrize("all_of_it", [False, True])
def test_masks_of_the_type_s_lowest_value_are_masks_off_the_list(kind, R, V, all_of_it):
    torch, b = _torch()
    xs, ids, values, lse, g = _case(R, V, 12, V, short=False, rest=True)
    lse = (lse + 0.25).astype(np.float32)
    low = torch.finfo(_types(torch)[kind]).min
    on = np.zeros((R, V), dtype=bool)
    for r in range(R):
        on[r, ids[r].astype(np.int64)] = True
    masked = ~on if all_of_it else ~on & (np.arange(V) % 3 > 0)
    x = torch.from_numpy(np.where(masked, low, xs).astype(np.float32)).cuda().to(_types(torch)[kind])
    xs = np.where(masked, -np.inf, x.float().cpu().numpy()).astype(np.float32)
    for how in ("fused", "apart"):
        loss, grad = _run(torch, b, x, ids, values, lse, g, 0.75, -1.5, how)
        _check(loss, grad, xs, ids, values, lse, g, 0.75, -1.5, kind)
        assert (grad[masked] == 0).all() and (loss == np.inf).all() == all_of_it
