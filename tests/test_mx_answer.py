"""Scores of a few rows from the example's held weights: every element, for any number of rows and any length."""
import numpy as np
import pytest

import mx_reference as ref
from test_mx_example import _example, _np, _values

pytestmark = pytest.mark.gpu


def _check(head, x, got, weights):
    """The product's sums, as held by held, and the bias's addition: its rounding, and the product's."""
    want, size = _values(x) @ weights.T + _np(head.bias), np.abs(_values(x)) @ np.abs(weights).T + np.abs(_np(head.bias))
    assert got.shape == want.shape and (np.abs(_np(got) - want) <= (x.shape[1] + 9) * 2.0 ** -24 * size).all()


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("rows, features", [(1, 64), (8, 4096), (16, 8192), (17, 130), (40, 1000), (300, 96)])
def test_any_number_of_rows_and_any_length(rows, features, dtype):
    """The head is made for 20 rows."""
    import torch
    head = _example().MxHead(700, features, 20)
    g = torch.Generator(device="cuda").manual_seed(rows)
    head.weights.copy_(torch.randn((700, features), device="cuda", generator=g) * 0.05)
    head.bias.copy_(torch.randn((700,), device="cuda", generator=g))
    x = torch.randn((rows, features), device="cuda", generator=g).to(getattr(torch, dtype))
    head.scores(torch.randn((20, features), device="cuda", generator=g))
    _check(head, x, head.answer(x), _values(head.weights, 32))


def _head(seed, items=700, features=130, rows=20):
    """A head before its first step, and what a step takes."""
    import torch
    head = _example().MxHead(items, features, rows, max_norm=0.5)
    g = torch.Generator(device="cuda").manual_seed(seed)
    ids = torch.stack([torch.randperm(items, device="cuda", generator=g)[:10] for _ in range(rows)]).int()
    dist = torch.rand((rows, 10), device="cuda", generator=g).sort(1).values
    return head, torch.randn((rows, features), device="cuda", generator=g).bfloat16(), ids, dist


def test_a_head_that_was_never_asked_answers_from_its_weights():
    """Zeros, in memory that held other codes."""
    import torch
    sizes = [(700, 80), (700, 8)]
    full = [torch.full(s, 0x77, dtype=torch.uint8, device="cuda") for s in sizes for _ in range(8)]
    del full
    head, x, _, _ = _head(1)
    head.bias.copy_(torch.arange(700, device="cuda"))
    assert torch.equal(head.answer(x[:3]), head.bias.expand(3, 700))


def test_after_steps_weights_and_bias_of_one_version():
    head, x, ids, dist = _head(2)
    for _ in range(3):
        head.step(x, ids, dist, 4.0, 2.0)
    before = _values(head.weights, 32)
    head.hold()
    assert np.array_equal(_values(head.weights, 32), before) and np.abs(before).max() > 0
    _check(head, x, head.answer(x), before)
    assert (np.abs(_np(head.bias)) > 0).any()
