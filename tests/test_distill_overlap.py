"""A gradient that shares memory with the logits in another place than their own is refused; rows side by side are not."""
import ctypes

import numpy as np
import pytest

from test_distill import _case, _check, _torch
from test_host_rules import _run as _compiled

gpu = pytest.mark.gpu


def test_the_rule_against_every_byte(tmp_path):
    """All small matrices in 96 bytes of memory, equal and unequal distances."""
    out = _compiled(tmp_path, """
#include "icq_overlap.h"
#include <stdio.h>
int main() {
    long cases = 0, wrong = 0, shared = 0;
    for (int rows = 0; rows <= 4; ++rows)
        for (int len = 1; len <= 5; ++len)
            for (int lda = len; lda <= 8; ++lda)
                for (int ldb = len; ldb <= 8; ++ldb)
                    for (int b = 0; b < 72; ++b) {
                        bool used[128] = {}, hit = false;
                        for (int r = 0; r < rows; ++r) for (int i = 0; i < len; ++i) used[36 + r * lda + i] = true;
                        for (int r = 0; r < rows; ++r) for (int i = 0; i < len; ++i) hit |= used[b + r * ldb + i];
                        ++cases;
                        shared += hit;
                        wrong += hit != icq_rows_overlap(36, lda, b, ldb, rows, len);
                    }
    printf("%d %ld %d\\n", cases > 10000, wrong, shared > 1000);
    return 0;
}
""")
    assert out == ["1", "0", "1"]


def test_overlapping_gradients_are_refused():
    from paper_1912_08756_amd import binding as b
    lib, E = b.load(), b.ICQ_ERR_ARG
    at = lambda n: ctypes.c_void_p(1 << 20 | n)
    fwd = dict(x=at(0), type=2, R=3, V=10, ld=32, scale=1.0, ids=at(0), values=at(0), topk=3, ts=-1.0, lse=None, loss=at(0), stats=None, g=None, grad=None, ldg=32, ws=None, bytes=0)
    back = dict(x=at(0), type=2, R=3, V=10, ld=32, scale=1.0, ids=at(0), values=at(0), topk=3, ts=-1.0, lse=None, stats=at(0), g=None, grad=None, ldg=32)
    for kw in (dict(grad=at(2)), dict(grad=at(18)), dict(grad=at(64 + 18)), dict(grad=at(128)), dict(grad=at(4), ldg=10), dict(x=at(50), grad=at(40)),
               dict(x=at(64), grad=at(0))):
        assert lib.icq_distill(*{**fwd, **kw}.values(), None) == E, kw
        assert lib.icq_distill_backward(*{**back, **kw}.values(), None) == E, kw
    for kw in (dict(grad=at(0)), dict(grad=at(20)), dict(grad=at(44)), dict(grad=at(148)), dict(grad=at(192)), dict(x=at(20), grad=at(0)), dict(x=at(1024), grad=at(0), ldg=10)):
        # (no workspace: goes no further)
        assert lib.icq_distill(*{**fwd, **kw}.values(), None) in (b.ICQ_ERR_WORKSPACE, b.ICQ_ERR_HIP), kw


@gpu
@pytest.mark.parametrize("R,V", [(5, 1000), (3, 70_000), (300, 1000)])
def test_logits_and_gradient_side_by_side_in_one_buffer(R, V):
    torch, b = _torch()
    xs, ids, values, lse, g = _case(R, V, 10, V, rest=True)
    buf = torch.full((R, 2 * V + 8), -7.0, device="cuda")
    x, grad = buf[:, :V], buf[:, V + 4:2 * V + 4]
    x.copy_(torch.from_numpy(xs))
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    loss, ws = torch.empty((R,), device="cuda"), torch.empty(b.icq_distill_workspace_bytes(R, V), dtype=torch.uint8, device="cuda")
    lists = (dev(ids.view(np.int32)), dev(values), 0.75, -1.5, dev(lse))
    b.icq_distill(x, *lists, loss, grad_loss=dev(g), grad=grad, workspace=ws)
    _check(loss.double().cpu().numpy(), grad.double().cpu().numpy(), xs, ids, values, lse, g, 0.75, -1.5, "f32")
    assert (buf[:, V:V + 4] == -7.0).all() and (buf[:, 2 * V + 4:] == -7.0).all()
    with pytest.raises(b.IcqError) as e:
        b.icq_distill(x, *lists, loss, grad_loss=dev(g), grad=buf[:, 4:V + 4], workspace=ws)
    assert e.value.code == b.ICQ_ERR_ARG
