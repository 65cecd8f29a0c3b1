"""The example's head in 4 bits: the whole of a step, each call's results against plain 64-bit forms of its own operands, and its gradients."""
import os
import sys

import numpy as np
import pytest

import block_reference
import mx_reference as ref

pytestmark = pytest.mark.gpu


def _example():
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import distill_neighbours
    return distill_neighbours


def _np(t):
    return t.double().cpu().numpy()


def _values(t, block_rows=1):
    return ref.values(*ref.quantize(_np(t), block_rows, True))


def test_a_step_s_logits_loss_gradients_norm_and_update():
    import torch
    e = _example()
    V, R, F, topk, T = 700, 150, 130, 10, 4.0
    _, ids, dist = e.neighbour_lists(items=V, queries=R, topk=topk, seed=3)
    g = torch.Generator(device="cuda").manual_seed(4)
    x = torch.relu(torch.randn((R, F), device="cuda", generator=g)).bfloat16()
    head = e.MxHead(V, F, R, max_norm=0.05)
    head.weights.copy_(torch.randn((V, F), device="cuda", generator=g) * 0.05)
    head.bias.copy_(torch.randn((V,), device="cuda", generator=g) * 0.1)
    before, bias = head.weights.clone(), head.bias.clone()
    logits = head.scores(x).clone()
    want = _values(x) @ _values(before, 32).T + _np(bias)
    size = np.abs(_values(x)) @ np.abs(_values(before, 32)).T
    # the product's sums and rounding to bf16, the bias's rounding to bf16
    assert (np.abs(_np(logits) - want) <= (F + 8) * 2.0 ** -24 * size + 2.0 ** -8 * (np.abs(want) + np.abs(want - _np(bias)) + np.abs(_np(bias)))).all()
    loss = head.step(x, ids, dist, T, 2.0)
    ref_loss, ref_grad, grad_size, reach = block_reference.distill(_np(logits), ids.cpu().numpy().view(np.uint32), dist.cpu().numpy(), 1.0, -1.0 / T)
    tol = 2.0 ** -23 * (4 * reach + V / 1024 + 64)
    got = _np(head.logits)                                     # the gradient has taken their place
    assert (np.abs(_np(loss) - ref_loss) <= tol * (1 + np.abs(ref_loss))).all()
    assert (np.abs(got - ref_grad) <= 2.0 ** -8 * np.abs(ref_grad) + tol[:, None] * grad_size + 1e-37).all()
    # gradients of weights and biases from that gradient, then clipped together
    dw = _values(head.logits.t()) @ _values(x.t()).T
    dw_size = np.abs(_values(head.logits.t())) @ np.abs(_values(x.t())).T
    db = got.sum(0)
    norm = ref.norm([dw, db])
    assert abs(float(head.norm) - norm) <= 1e-5 * norm
    f = ref.factor(float(head.norm), 0.05)
    assert f < 1
    assert (np.abs(_np(head.grad) - f * dw) <= f * (R + 16) * 2.0 ** -23 * dw_size).all()
    assert (np.abs(_np(head.bias_grad) - f * db) <= f * (R + 16) * 2.0 ** -23 * np.abs(got).sum(0)).all()
    assert torch.equal(head.weights, before.add_(head.grad, alpha=-2.0)) and torch.equal(head.bias, bias.add_(head.bias_grad, alpha=-2.0))
    # a few rows answered from the held weights: the scores of the head before the update
    held = _values(before.sub_(head.grad, alpha=-2.0), 32)     # (weights as they were when they were quantised, up to their last bit)
    few = _np(head.answer(x[:3]))
    again = _values(x[:3]) @ held.T + _np(head.bias)
    assert np.median(np.abs(few - again)) <= 1e-5 * np.abs(again).max()


def test_the_example_runs_and_repeats_its_bits():
    e = _example()
    losses, _ = e.train(steps=4, items=3000, queries=200, features=130, topk=10, bits=4)
    again, _ = e.train(steps=4, items=3000, queries=200, features=130, topk=10, bits=4)
    assert np.isfinite(losses.numpy()).all() and losses.tolist() == again.tolist()


def test_gradients_of_a_product_against_differences():
    """f(X, W) = sum of G * (X W^T): with whole numbers that 4 bits hold, its differences in a direction are exactly the gradients' products with it."""
    import torch
    from paper_1912_08756_amd import binding as b
    g = torch.Generator(device="cuda").manual_seed(8)
    T, N, K = 70, 100, 90
    whole = lambda *s: torch.randint(-1, 3, s, device="cuda", generator=g).float()
    x, w, gr = whole(T, K), whole(N, K), whole(T, N)
    dirs = {"x": torch.randint(-1, 2, (T, K), device="cuda", generator=g).float(), "w": torch.randint(-1, 2, (N, K), device="cuda", generator=g).float()}

    def held(t, both=False):
        q = [b.icq_mx_codes(*t.shape), b.icq_mx_scales(*t.shape), b.icq_mx_codes(*t.t().shape), b.icq_mx_scales(*t.t().shape)]
        b.icq_mx_quantize(t, *q)
        v = torch.empty_like(t)
        assert torch.equal(b.icq_mx_dequantize(q[0], q[1], v), t)
        return q

    def product(a, c, M, n, k):
        out = torch.empty((M, n), device="cuda")
        need = b.icq_mx_matmul_workspace_bytes(M, n, k)
        return b.icq_mx_matmul(*a, *c, out, torch.empty(need, dtype=torch.uint8, device="cuda") if need else None, K=k)

    f = lambda x, w: float((gr * product(held(x)[:2], held(w)[:2], T, N, K)).double().sum())
    qx, qw, qg = held(x), held(w), held(gr)
    dx, dw = product(qg[:2], qw[2:], T, K, N), product(qg[2:], qx[2:], N, K, T)
    assert f(x + dirs["x"], w) - f(x, w) == float((dx * dirs["x"]).double().sum())
    assert f(x, w + dirs["w"]) - f(x, w) == float((dw * dirs["w"]).double().sum())
