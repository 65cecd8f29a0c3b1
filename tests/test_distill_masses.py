"""What the distillation's gradient is to its loss: the derivative where the teacher's masses add up to one, and by how much it differs elsewhere."""
import numpy as np
import pytest

import block_reference as ref
from test_distill import _check, _run, _torch

gpu = pytest.mark.gpu
SCALE, TEACHER = 0.75, -1.5


def _rows():
    """(logits, ids, values, teacher logsumexp, S): eight items; lists of three and of all eight; a logsumexp of the list's own, above and below."""
    rng = np.random.default_rng(4)
    x = rng.standard_normal((6, 8)) * 1.5
    ids = np.full((6, 8), ref.PAD_ID, dtype=np.uint32)
    values = np.full((6, 8), np.inf, dtype=np.float32)
    own = np.empty(6)
    for r in range(6):
        n = 3 if r < 3 else 8
        ids[r, :n] = rng.permutation(8)[:n]
        values[r, :n] = rng.random(n) * 2
        own[r] = np.log(np.exp(TEACHER * values[r, :n].astype(np.float64)).sum())
    shift = np.array([0.0, 0.4, -0.3] * 2)
    lse = (own + shift).astype(np.float32)
    total = np.exp(own - lse.astype(np.float64))
    return x.astype(np.float32), ids, values, lse, np.where(np.arange(6) == 1, 1.0, total)      # (short list, logsumexp above: p_r makes it one)


def _stated_and_derivative(x, ids, values, lse):
    _, grad, _, _ = ref.distill(x.astype(np.float64), ids, values, SCALE, TEACHER, lse)
    slope, h = np.zeros_like(grad), 1e-5
    for v in range(x.shape[1]):
        up, down = x.astype(np.float64), x.astype(np.float64)
        up[:, v] += h
        down[:, v] -= h
        slope[:, v] = (ref.distill(up, ids, values, SCALE, TEACHER, lse)[0] - ref.distill(down, ids, values, SCALE, TEACHER, lse)[0]) / (2 * h)
    return grad, slope


def test_the_gradient_exceeds_the_derivative_by_the_mass_that_lacks():
    x, ids, values, lse, S = _rows()
    grad, slope = _stated_and_derivative(x, ids, values, lse)
    q = np.exp(SCALE * x.astype(np.float64))
    q /= q.sum(1, keepdims=True)
    # the header's words: grad - derivative = scale (1 - S) q_v, nothing where the masses add up to one
    assert np.abs(grad - slope - SCALE * (1 - S)[:, None] * q).max() <= 1e-8
    assert np.abs(S[[0, 1, 3]] - 1).max() <= 1e-6 and S[2] > 1.3 and S[4] < 0.7 and S[5] > 1.3


def test_without_a_logsumexp_the_gradient_is_the_derivative():
    x, ids, values, _, _ = _rows()
    grad, slope = _stated_and_derivative(x, ids, values, None)
    assert np.abs(grad - slope).max() <= 1e-8


def test_the_header_says_so():
    import os
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "icq.h")).read()
    words = " ".join(text.replace("*", " ").split())
    assert "d loss[r] / d logits[r][v] where the teacher's masses add up to one" in words
    assert "exceeds it by grad_loss[r] scale (1 - S) q_v" in words


@gpu
@pytest.mark.parametrize("how", ["fused", "apart"])
def test_the_kernels_give_the_stated_gradient(how):
    torch, b = _torch()
    x, ids, values, lse, _ = _rows()
    for teacher in (lse, None):
        got = _run(torch, b, torch.from_numpy(x).cuda(), ids, values, teacher, None, SCALE, TEACHER, how)
        _check(*got, x, ids, values, teacher, None, SCALE, TEACHER, "f32")
