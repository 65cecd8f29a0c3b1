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
