"""Every form of the 4-bit products: which one a size takes (the plan's rule compiled for the host, 256 compute units), and its results on whole
numbers, where every sum is exact."""
import pytest

from test_host_rules import _run as _compiled

gpu = pytest.mark.gpu

# rows of a and b, numbers of stages of 256 values: the form of each with every tail
TAILS = (0, 1, 44, 129, 255)
PIPELINES = [(500, 65000, (2, 3, 4, 5, 6, 8, 9), "wide"), (4101, 16387, (4, 7), "wide"), (2500, 3300, (1, 2, 3, 4, 5, 8, 9), "small"),
             (1300, 1900, (5, 6, 7, 8, 9, 12), "deep"), (40, 130, (1, 2, 3, 4, 5, 6, 7, 8, 9, 12), "little"), (700, 900, (1, 4, 9), "little")]
# sizes: form and parts of the contraction
SPLIT = [(2048, 960, 16384, "deep", 2), (256, 5003, 16001, "deep", 2), (1000, 1000, 16300, "deep", 4), (200, 131, 4100, "little", 4), (256, 256, 65000, "little", 16),
         (130, 260, 30000, "little", 8), (17, 16384, 4096, "little", 1)]
# few rows: wavefronts of 32 rows of b or of 16, how many share them, parts, whether the kernel quantises values itself
FEW = [(1, 16384, 384, "few of 32", 2, 1, True), (3, 16500, 300, "few of 32", 2, 1, True), (16, 16390, 1030, "few of 32", 4, 1, False),
       (1, 70001, 5, "few of 32", 1, 1, True), (1, 200000, 2100, "few of 32", 4, 1, True), (8, 100003, 960, "few of 32", 4, 1, True), (8, 512, 8192, "few of 16", 8, 1, False),
       (1, 40, 20001, "few of 16", 8, 2, False), (16, 16, 65536, "few of 16", 8, 8, False), (5, 300, 700, "few of 16", 2, 1, True), (2, 4099, 4097, "few of 16", 8, 1, True),
       (16, 300, 900, "few of 16", 4, 1, True), (1, 1, 1, "few of 16", 1, 1, True), (1, 16, 8191, "few of 16", 8, 1, True), (2, 5000, 256, "few of 16", 1, 1, True),
       (12, 16384, 4096, "few of 32", 4, 1, False), (3, 65600, 4099, "few of 32", 4, 1, True), (16, 16384, 20000, "few of 32", 4, 3, False), (16, 9000, 9473, "few of 16", 4, 2, False),
       (16, 9000, 9472, "few of 16", 4, 1, False), (1, 300, 200000, "few of 16", 8, 13, False), (11, 40000, 129, "few of 32", 1, 1, True), (6, 3000, 1500, "few of 16", 4, 1, True)]


def _plans(tmp_path, sizes):
    """[form, parts, wavefronts that share rows, whether values are quantised in the kernel] of every (M, N, K)."""
    out = _compiled(tmp_path, """
#include "icq_mx_plan.h"
#include <stdio.h>
int main() {
    const long s[][3] = {%s};
    const char *tiles[] = {"wide", "small", "deep", "little"};
    for (const auto &c : s) {
        const icq_mx_plan p = icq_plan_mx(c[0], c[1], c[2], 256);
        printf("%%s:%%d:%%d:%%d\\n", !p.few ? tiles[p.tiles] : p.wide ? "few_of_32" : "few_of_16", p.splits, p.along, icq_mx_few_quantises(c[0], p.per));
    }
    return 0;
}
""" % ",".join("{%d,%d,%d}" % s for s in sizes))
    return [[f.replace("_", " ")] + [int(v) for v in o] for f, *o in (line.split(":") for line in out)]


def _lengths(stages):
    return sorted({k for s in stages for k in [256 * (s - 1) + t for t in TAILS if t] + [256 * s]})


def test_the_sizes_take_the_forms_they_are_here_for(tmp_path):
    sizes = [(M, N, K) for M, N, stages, _ in PIPELINES for K in _lengths(stages)]
    want = [form for _, _, stages, form in PIPELINES for _ in _lengths(stages)]
    assert [(s, p[0]) for s, p in zip(sizes, _plans(tmp_path, sizes))] == list(zip(sizes, want))
    assert [(s[:3], *p[:2]) for s, p in zip(SPLIT, _plans(tmp_path, [s[:3] for s in SPLIT]))] == [(s[:3], *s[3:]) for s in SPLIT]
    got = _plans(tmp_path, [s[:3] for s in FEW])
    assert [(s[:3], p[0], p[2], p[1], bool(p[3])) for s, p in zip(FEW, got)] == [(s[:3], *s[3:]) for s in FEW]


def test_no_part_of_the_contraction_is_empty_and_all_are_covered(tmp_path):
    sizes = [(M, N, K) for M in (1, 16, 17, 40, 200, 1000) for N in (1, 100, 4096, 70000) for K in list(range(1, 3000, 211)) + [8191, 16385, 40000, 1 << 20]]
    out = _compiled(tmp_path, """
#include "icq_mx_plan.h"
#include <stdio.h>
int main() {
    const long s[][3] = {%s};
    for (const auto &c : s) {
        const icq_mx_plan p = icq_plan_mx(c[0], c[1], c[2], 256);
        const long stages = (c[2] + 255) / 256;
        printf("%%d\\n", p.splits >= 1 && p.per >= 1 && (long)p.per * p.splits >= stages && (long)p.per * (p.splits - 1) < stages);
    }
    return 0;
}
""" % ",".join("{%d,%d,%d}" % s for s in sizes))
    assert out == ["1"] * len(sizes)


def _exact(M, N, K, values):
    import torch
    from paper_1912_08756_amd import binding as b
    b.load()
    g = torch.Generator(device="cuda").manual_seed(M + N + K)
    far = 2 if K <= 2048 else 1 if K <= 20001 else 0           # K * 9 * 4^(2 far) < 2^24: every partial sum is a whole number of units, exact in 32 bits
    assert K * 9 * 4 ** (2 * far) < 2 ** 24
    blocks = -(-K // 32)

    def held(rows):
        v = torch.randint(-3, 4, (rows, K), device="cuda", generator=g)
        table = torch.tensor([13, 12, 10, 0, 2, 4, 5], dtype=torch.uint8, device="cuda")       # -3 .. 3
        c = torch.nn.functional.pad(table[v + 3], (0, K % 2), value=0xF)                         # (an odd row's last half byte is not its own)
        codes, scales = b.icq_mx_codes(rows, K), b.icq_mx_scales(rows, K)
        codes.untyped_storage().fill_(0xFF)
        scales.untyped_storage().fill_(0xFF)                   # padding that would be NaN
        codes.copy_(c[:, ::2] | c[:, 1::2] << 4)
        e = torch.randint(-far, far + 1, (rows, blocks), device="cuda", generator=g)
        scales.copy_((e + 127).to(torch.uint8))
        return codes, scales, v.float() * torch.exp2(e.float()).repeat_interleave(32, 1)[:, :K]

    wc, ws, wv = held(N)
    if values:                                                 # a block's largest is 3 times a power of two: held as it is
        x = torch.randint(-3, 4, (M, K), device="cuda", generator=g).float()
        x[:, ::32] = 3.0
        x *= torch.exp2(torch.randint(-far, far + 1, (M, blocks), device="cuda", generator=g).float()).repeat_interleave(32, 1)[:, :K]
        a, xv = (x.bfloat16(), None), x
    else:
        *a, xv = held(M)
    want = xv @ wv.t()                                         # (exact in 32 bits, in whatever order)
    need = b.icq_mx_matmul_workspace_bytes(M, N, K, torch.bfloat16 if values else None)
    space = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        y = torch.full((M, N), float("nan"), dtype=dtype, device="cuda")
        b.icq_mx_matmul(*a, wc, ws, y, space, K=K)
        assert torch.equal(y, want.to(dtype)), dtype


@gpu
@pytest.mark.parametrize("M,N,stages,form", [(M, N, s, f) for M, N, stages, f in PIPELINES for s in stages])
def test_every_number_of_stages_in_every_tile_form(M, N, stages, form):
    for K in _lengths((stages,)):
        _exact(M, N, K, False)


@gpu
@pytest.mark.parametrize("M,N,K", [s[:3] for s in SPLIT + FEW])
@pytest.mark.parametrize("values", [False, True])
def test_parts_of_the_contraction_and_few_rows(M, N, K, values):
    _exact(M, N, K, values)


@gpu
@pytest.mark.parametrize("M,N,K,form", [(500, 65000, 960, "wide"), (2500, 3300, 700, "small"), (1300, 1900, 1100, "deep"), (40, 130, 300, "little"), (5, 300, 700, "few")])
def test_rows_of_wider_buffers_and_results_at_odd_addresses(M, N, K, form):
    import torch
    from paper_1912_08756_amd import binding as b
    b.load()
    g = torch.Generator(device="cuda").manual_seed(K)

    def held(rows):
        x = torch.randn((rows, K), device="cuda", generator=g)
        codes, scales = b.icq_mx_codes(rows, K + 2000)[:, 32:32 + -(-K // 2)], b.icq_mx_scales(rows, K + 999)[:, 8:8 + -(-K // 32)]
        b.icq_mx_quantize(x, codes, scales)
        v = torch.empty((rows, K), device="cuda")
        b.icq_mx_dequantize(codes, scales, v)
        return codes, scales, v

    ac, sa, av = held(M)
    wc, sw, wv = held(N)
    want = av @ wv.t()
    need = b.icq_mx_matmul_workspace_bytes(M, N, K)
    space = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
    for dtype, tol in ((torch.float32, 1e-5), (torch.bfloat16, 2.0 ** -8)):
        wide = torch.full((M, N + 11), -5.0, dtype=dtype, device="cuda")
        y = wide[:, 3:N + 3]
        b.icq_mx_matmul(ac, sa, wc, sw, y, space, K=K)
        assert bool(((y.float() - want).abs() <= tol * want.abs() + 1e-5 * want.abs().max()).all())
        assert (wide[:, :3] == -5).all() and (wide[:, N + 3:] == -5).all()


@gpu
def test_more_rows_than_a_launch_of_tiles_has_blocks_for():
    """2^23 tiles of 64 x 64 and more, and as many groups of few rows: results are those of calls on parts."""
    import torch
    from paper_1912_08756_amd import binding as b
    b.load()
    for M, N, dtype in ((33, (1 << 28) + 300, torch.bfloat16), (2, (1 << 29) + 70, torch.float32)):
        K = 16
        g = torch.Generator(device="cuda").manual_seed(M)
        w, sw = torch.empty((N, 16), dtype=torch.uint8, device="cuda"), torch.empty((N, 4), dtype=torch.uint8, device="cuda")
        w.view(torch.int64).random_(generator=g)
        sw.random_(120, 130, generator=g)
        a, sa = torch.randint(0, 256, (M, 16), dtype=torch.uint8, device="cuda", generator=g), torch.full((M, 4), 127, dtype=torch.uint8, device="cuda")
        out = torch.full((M, N), float("nan"), dtype=dtype, device="cuda")
        b.icq_mx_matmul(a[:, :8], sa[:, :1], w[:, :8], sw[:, :1], out, K=K)
        some = 1 << 16
        for at in (0, N // 2 - some // 2, N - some):
            part = torch.empty((M, some), dtype=dtype, device="cuda")
            b.icq_mx_matmul(a[:, :8], sa[:, :1], w[at:at + some, :8], sw[at:at + some, :1], part, K=K)
            assert torch.equal(out[:, at:at + some], part)     # (16 products of whole quarters: exact)
        for at in range(0, N, 1 << 24):
            assert not bool(torch.isnan(out[:, at:at + (1 << 24)]).any()), at
