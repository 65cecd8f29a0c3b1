"""Every form of the block products: which one a size takes (the plan's rule compiled for the host, 256 compute units), and its results on
whole numbers, where every sum is exact."""
import pytest

from test_block_ops import _torch
from test_host_rules import _run as _compiled

gpu = pytest.mark.gpu

STEPS, TAILS = range(1, 15), (0, 1, 100)
# rows of a and b: the form of every contraction of one to fifteen scale blocks, by the result's type
PIPELINES = [(3900, 4000, "16", "wide"), (1300, 1900, "16", "deep"), (1300, 1900, "f32", "deep"), (1300, 3900, "f32", "small"),
             (2304, 2500, "16", "small"), (40, 130, "16", "little"), (40, 130, "f32", "little")]
# sizes: form and parts of the contraction
SPLIT = [(2048, 960, 16384, "16", "deep", 2), (2048, 960, 16300, "16", "deep", 2), (256, 5003, 16001, "16", "deep", 2),
         (2048, 960, 16300, "f32", "small", 4), (200, 131, 4100, "16", "little", 8), (200, 131, 9000, "16", "little", 16),
         (600, 700, 5000, "16", "little", 2), (600, 703, 5000, "f32", "little", 4)]
FEW = [(1, 16384, 384, "16", "few of 64", 1), (3, 16500, 300, "16", "few of 64", 1), (16, 16390, 1030, "f32", "few of 64", 1),
       (1, 70001, 5, "f32", "few of 64", 1), (8, 512, 8192, "16", "few", 2), (8, 512, 8200, "f32", "few", 2), (1, 40, 20001, "16", "few", 4),
       (16, 16, 65536, "16", "few", 16), (5, 300, 700, "16", "few", 1), (20, 500, 9000, "16", "few of 32", 2), (32, 4096, 1000, "f32", "few of 32", 1)]


def _plans(tmp_path, sizes):
    """(form, parts) of every (M, N, K, "16" or "f32")."""
    out = _compiled(tmp_path, """
#include "icq_matmul_plan.h"
#include <stdio.h>
int main() {
    const long s[][4] = {%s};
    const char *tiles[] = {"wide", "small", "deep", "little"};
    for (const auto &c : s) {
        const icq_product_plan p = icq_plan_product(c[0], c[1], c[2], c[3] != 0, 256);
        printf("%%s:%%d\\n", !p.few ? tiles[p.tiles] : c[0] > 16 ? "few_of_32" : icq_product_few_wide(c[0], c[1], 256) ? "few_of_64" : "few", p.splits);
    }
    return 0;
}
""" % ",".join("{%d,%d,%d,%d}" % (M, N, K, t == "f32") for M, N, K, t in sizes))
    return [(o.split(":")[0].replace("_", " "), int(o.split(":")[1])) for o in out]


def test_the_sizes_take_the_forms_they_are_here_for(tmp_path):
    want, sizes = [], []
    for M, N, kind, form in PIPELINES:
        for steps in STEPS:
            for tail in TAILS:
                sizes.append((M, N, 128 * steps + tail, kind))
                want.append(form)
    assert [(s, f) for s, (f, _) in zip(sizes, _plans(tmp_path, sizes))] == list(zip(sizes, want))
    fixed = SPLIT + FEW
    assert [(s, *p) for s, p in zip([c[:4] for c in fixed], _plans(tmp_path, [c[:4] for c in fixed]))] == [(c[:4], *c[4:]) for c in fixed]


def _exact(M, N, K, kind, block, pow2, fa="e4m3", fb="e4m3"):
    torch, b = _torch()
    formats = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
    g = torch.Generator(device="cuda").manual_seed(M + N + K)
    far = 2 if K <= 2048 else 1 if K <= 20001 else 0           # K * 9 * 4^(2 far) < 2^24: every partial sum is a whole number of units, exact in 32 bits
    assert K * 9 * 4 ** (2 * far) < 2 ** 24
    blocks = -(-K // 128)
    draw = lambda rows: torch.randint(-3, 4, (rows, K), device="cuda", generator=g).float()
    scales = lambda rows: torch.exp2(torch.randint(-far, far + 1, (rows, blocks), device="cuda", generator=g).float())
    x, w = draw(M), draw(N)
    ac, wc = b.icq_block_codes(M, K, formats[fa]), b.icq_block_codes(N, K, formats[fb])
    for c, v in ((ac, x), (wc, w)):
        c.untyped_storage().fill_(0x7F)                        # padding that would be NaN
        c.copy_(v.to(c.dtype))
    sa, sw = scales(M), scales(N if block == 1 else -(-N // 128))
    wide = sw if block == 1 else sw.repeat_interleave(128, 0)[:N]
    want = (sa.repeat_interleave(128, 1)[:, :K] * x).double() @ (wide.repeat_interleave(128, 1)[:, :K] * w).double().t().contiguous()
    ws = torch.empty(max(1, b.icq_block_matmul_workspace_bytes(M, N, K)), dtype=torch.uint8, device="cuda")
    for dtype in ((torch.float32,) if kind == "f32" else (torch.bfloat16, torch.float16)):
        y = torch.full((M, N), float("nan"), dtype=dtype, device="cuda")
        b.icq_block_matmul(ac, sa, wc, sw, y, ws, pow2=pow2)
        assert torch.equal(y, want.float().to(dtype))


@gpu
@pytest.mark.parametrize("steps", STEPS)
@pytest.mark.parametrize("M,N,kind,form", PIPELINES)
@pytest.mark.parametrize("block", [1, 128])
def test_every_number_of_scale_blocks_in_every_tile_form(M, N, kind, form, steps, block):
    for tail in TAILS:
        for pow2 in (False, True):
            _exact(M, N, 128 * steps + tail, kind, block, pow2, "e5m2" if steps % 2 else "e4m3", "e4m3" if steps % 3 else "e5m2")


@gpu
@pytest.mark.parametrize("M,N,K,kind,form,parts", SPLIT + FEW)
@pytest.mark.parametrize("block", [1, 128])
def test_parts_of_the_contraction_and_few_rows(M, N, K, kind, form, parts, block):
    for pow2 in (False, True):
        _exact(M, N, K, kind, block, pow2)
