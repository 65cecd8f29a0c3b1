"""Every form of the distillation's kernels: which one a size takes (the rules compiled for the host, 256 compute units), and loss and gradient
against the plain form, listed items on both sides of where a row's marking starts anew."""
import numpy as np
import pytest

import block_reference as ref
from test_distill import EPS, ROUND, _torch
from test_host_rules import _run as _compiled

gpu = pytest.mark.gpu
DISTINCT = 8
# rows, items, type: the fused kernel, the threads of the sums alone, slices of the two apart
FORMS = [(264, 4000, "f32", "256x4", 256, 1), (264, 6001, "f32", "256x8", 256, 1), (264, 12_003, "f32", "256x16", 256, 1),
         (264, 40_001, "f32", "long", 256, 1), (264, 70_001, "f32", "long", 512, 1), (264, 200_003, "f32", "long", 512, 1),
         (264, 6001, "bf16", "256x4", 256, 1), (264, 12_003, "bf16", "256x8", 256, 1), (264, 30_001, "bf16", "256x16", 256, 1),
         (264, 70_001, "bf16", "long", 256, 1), (264, 200_003, "bf16", "long", 512, 1),
         (264, 6001, "f16", "256x4", 256, 1), (264, 12_003, "f16", "256x8", 256, 1), (264, 30_001, "f16", "256x16", 256, 1),
         (264, 70_001, "f16", "long", 256, 1), (264, 140_003, "f16", "long", 512, 1),
         (200, 12_003, "f32", "1024x4", 256, 1), (200, 30_001, "bf16", "1024x4", 256, 3), (24, 16_001, "f16", "1024x4", 256, 1),
         (200, 500_003, "f32", "long", 256, 6), (200, 500_003, "bf16", "long", 256, 6), (120, 70_001, "f32", "slices", 256, 8)]


def test_the_sizes_take_the_forms_they_are_here_for(tmp_path):
    size = {"f32": 4, "f16": 2, "bf16": 2}
    out = _compiled(tmp_path, """
#include "icq_distill_plan.h"
#include <stdio.h>
int main() {
    const long s[][3] = {%s};
    const char *rows[] = {"1024x4", "256x4", "256x8", "256x16", "long"};
    for (const auto &c : s) {
        const int fused = icq_distill_splits(c[0], c[1], 256, c[1] * c[2]), apart = icq_distill_splits(c[0], c[1], 256, 0);
        printf("%%s:%%d:%%d\\n", fused > 1 ? "slices" : rows[icq_distill_row_form(c[0], c[1] * c[2], 256)], icq_distill_forward_threads(apart, c[1] * c[2]), apart);
    }
    return 0;
}
""" % ",".join("{%d,%d,%d}" % (R, V, size[t]) for R, V, t, *_ in FORMS))
    assert out == ["%s:%d:%d" % f[3:] for f in FORMS]


def _rows(V, topk, rest):
    """Eight distinct rows whose lists hold the items around every multiple of 65536 and the row's ends."""
    rng = np.random.default_rng(V + topk)
    edge = [v for m in range(0, V + 1, 65536) for v in range(max(0, m - 9), min(V, m + 9))] + list(range(V - 9, V))
    edge = np.unique(edge)[:topk]
    x = (rng.standard_normal((DISTINCT, V)) * 2.0).astype(np.float32)
    ids = np.full((DISTINCT, topk), ref.PAD_ID, dtype=np.uint32)
    values = np.full((DISTINCT, topk), np.inf, dtype=np.float32)
    for r in range(DISTINCT - 1):                              # (the last row's list is empty)
        n = topk if r % 3 else max(len(edge), topk // 2)
        chosen = np.concatenate([edge, rng.choice(np.setdiff1d(np.arange(V), edge), n - len(edge), replace=False)])
        ids[r, :n] = rng.permutation(chosen)
        values[r, :n] = np.sort(rng.random(n) * 4.0)
        x[r, ids[r, :n].astype(np.int64)] += 5.0 + 0.5 * values[r, :n]
    lse = None
    if rest:
        with np.errstate(divide="ignore"):
            lse = np.log(np.exp(-1.5 * values.astype(np.float64)).sum(1))
        lse = (np.where(np.isfinite(lse), lse, 0.0) + 0.3).astype(np.float32)
    return x, ids, values, lse, (rng.random(DISTINCT) + 0.5).astype(np.float32)


@gpu
@pytest.mark.parametrize("R,V,kind,form,threads,slices", FORMS)
@pytest.mark.parametrize("topk", [100, 300])
@pytest.mark.parametrize("rest", [False, True])
def test_loss_and_gradient_in_every_form(R, V, kind, form, threads, slices, topk, rest):
    torch, b = _torch()
    x, ids, values, lse, g = _rows(V, topk, rest)
    if kind == "f16":
        g = g * 64
    dtype = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[kind]
    few = torch.from_numpy(x).cuda().to(dtype)
    want, dwant, size, reach = ref.distill(few.float().cpu().numpy(), ids, values, 0.75, -1.5, lse, g)
    rel = EPS * (4 * reach + V / 1024 + 64)                    # as for the other sizes
    loss_tol = rel * (1 + np.abs(want))
    tol = rel[:, None] * size + ROUND[kind] * np.abs(dwant) + (2.0 ** -24 if kind == "f16" else 1e-37)
    n = R // DISTINCT
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    many = lambda t: t.repeat(*([n] + [1] * (t.dim() - 1)))
    xs = many(few)
    lists = (many(dev(ids.view(np.int32))), many(dev(values)), 0.75, -1.5, many(dev(lse)) if rest else None)
    loss, stats, grad = torch.empty((R,), device="cuda"), torch.empty((R, 4), device="cuda"), torch.empty_like(xs)
    ws = torch.empty(b.icq_distill_workspace_bytes(R, V), dtype=torch.uint8, device="cuda")
    want, dwant, loss_tol, tol = dev(want), dev(dwant), dev(loss_tol), dev(tol)

    def check(how):
        assert bool(((loss.double().view(n, DISTINCT) - want).abs() <= loss_tol).all()), how
        for k in range(n):                                     # (odd row lengths: every copy starts elsewhere within 16 bytes)
            off = (grad[k * DISTINCT:(k + 1) * DISTINCT].double() - dwant).abs()
            assert bool((off <= tol).all()), (how, k)

    b.icq_distill(xs, *lists, loss, stats, workspace=ws)
    b.icq_distill_backward(xs, *lists, stats, many(dev(g)), grad)
    check("apart")
    loss.fill_(-7.0)
    grad.fill_(-7.0)
    b.icq_distill(xs, *lists, loss, grad_loss=many(dev(g)), grad=grad, workspace=ws)
    check("fused")
    b.icq_distill(xs, *lists, loss, grad_loss=many(dev(g)), grad=xs, workspace=ws)
    assert torch.equal(xs, grad)                               # in the logits' place
