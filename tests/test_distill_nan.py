"""A teacher's NaN is in its row's loss and in the gradient of every item, listed or not."""
import numpy as np
import pytest

from test_distill import PAD, _case, _check, _run, _torch

gpu = pytest.mark.gpu


@gpu
@pytest.mark.parametrize("R,V,topk", [(6, 300, 12), (6, 70_000, 12), (400, 2100, 12), (6, 3000, 300)])
@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("how", ["fused", "apart"])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_nan_of_the_teacher(R, V, topk, rest, how, kind):
    torch, b = _torch()
    xs, ids, values, lse, g = _case(R, V, topk, V, short=False, rest=rest)
    values[1, 3] = np.nan                                      # one score
    values[2] = np.nan                                         # all of them
    values[3, 1:], ids[3, 1:] = np.nan, PAD                    # padding: counts for nothing
    ids[4], values[4] = PAD, np.nan                            # no entry at all
    bad = [1, 2]
    if rest:
        lse[5], lse[4] = np.nan, np.nan                        # the logsumexp (of a row with entries, and of one without)
        bad.append(5)
    x = torch.from_numpy(xs).cuda().to(torch.float32 if kind == "f32" else torch.bfloat16)
    xs = x.float().cpu().numpy()
    loss, grad = _run(torch, b, x, ids, values, lse, g, 0.75, -1.5, how)
    assert np.isnan(loss[bad]).all() and np.isnan(grad[bad]).all()
    assert loss[4] == 0 and (grad[4] == 0).all()
    keep = [r for r in range(R) if r not in bad and r != 4]
    _check(loss[keep], grad[keep], xs[keep], ids[keep], values[keep], lse[keep] if rest else None, g[keep], 0.75, -1.5, kind)
