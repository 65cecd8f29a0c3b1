"""4-bit products under every scale there is, in every form of the kernels: scales far apart within a row, the least and the largest, rows without a number."""
import pytest

pytestmark = pytest.mark.gpu

# a size of each form: few rows by wavefronts of 16 and 32 rows of b, tiles of 64, 128 (two depths) and 256, parts of the contraction
FORMS = [(5, 300, 700), (8, 17000, 960), (40, 130, 300), (2500, 3300, 700), (1300, 1900, 1100), (500, 65000, 960), (200, 131, 4100), (1, 40, 20001)]
VALUES = (0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6)


def _torch():
    import torch
    from paper_1912_08756_amd import binding
    binding.load()
    return torch, binding


def _held(torch, b, rows, K, least, most, seed):
    """Random codes, scale bytes of a range, and their values in 64 bits; what lies behind the rows' ends would be NaN."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    codes, scales = b.icq_mx_codes(rows, K), b.icq_mx_scales(rows, K)
    codes.untyped_storage().fill_(0xFF)
    scales.untyped_storage().fill_(0xFF)
    codes.copy_(torch.randint(0, 256, codes.shape, dtype=torch.uint8, device="cuda", generator=g))
    scales.copy_(torch.randint(least, most + 1, scales.shape, device="cuda", generator=g).to(torch.uint8))
    return codes, scales, _values(torch, codes, scales, K)


def _values(torch, codes, scales, K):
    table = torch.tensor(VALUES, dtype=torch.float64, device="cuda")
    each = torch.stack([codes & 15, codes >> 4], 2).flatten(1)[:, :K].long()
    return table[each] * torch.exp2(scales.double() - 127).repeat_interleave(32, 1)[:, :K]


def _product(torch, b, a, w, M, N, K, dtype):
    y = torch.full((M, N), float("nan"), dtype=dtype, device="cuda")
    need = b.icq_mx_matmul_workspace_bytes(M, N, K)
    return b.icq_mx_matmul(*a[:2], *w[:2], y, torch.empty(need, dtype=torch.uint8, device="cuda") if need else None, K=K)


@pytest.mark.parametrize("M,N,K", FORMS)
@pytest.mark.parametrize("bytes_", [(117, 137), (87, 167), (100, 107), (63, 69)], ids=["2^10", "2^40", "small", "below the normal numbers"])
def test_scales_far_apart(M, N, K, bytes_):
    """Each addition's rounding, half a unit in the last place of the sum or of the smallest numbers of 32 bits, and the result's."""
    torch, b = _torch()
    a, w = _held(torch, b, M, K, *bytes_, 1), _held(torch, b, N, K, *bytes_, 2)
    want, size = a[2] @ w[2].t(), a[2].abs() @ w[2].abs().t()
    assert float(size.max()) < 2.0 ** 127
    for dtype, half, least in ((torch.float32, 2.0 ** -24, 2.0 ** -149), (torch.bfloat16, 2.0 ** -8, 2.0 ** -133)):
        got = _product(torch, b, a, w, M, N, K, dtype).double()
        assert bool(((got - want).abs() <= (K + 8) * (2.0 ** -24 * size + 2.0 ** -149) + half * want.abs() + least).all())


@pytest.mark.parametrize("M,N,K", FORMS)
def test_the_largest_scales_times_the_least(M, N, K):
    """2^127 and 2^-127: sums of quarters below 2^24 units, exact in any order."""
    torch, b = _torch()
    for x, y in ((254, 0), (0, 254)):
        a, w = _held(torch, b, M, K, x, x, 3), _held(torch, b, N, K, y, y, 4)
        assert torch.equal(_product(torch, b, a, w, M, N, K, torch.float32).double(), a[2] @ w[2].t())


@pytest.mark.parametrize("M,N,K", FORMS)
def test_beyond_the_range_of_32_bits(M, N, K):
    torch, b = _torch()
    a, w = _held(torch, b, M, K, 254, 254, 5), _held(torch, b, N, K, 254, 254, 6)
    zeros = b.icq_mx_codes(M, K)
    zeros.untyped_storage().fill_(0)
    assert not _product(torch, b, (zeros, a[1]), w, M, N, K, torch.float32).any()                 # of whatever scale
    sums = a[2] @ w[2].t()
    assert not bool(torch.isfinite(_product(torch, b, a, w, M, N, K, torch.float32))[sums != 0].any())
    a, w = _held(torch, b, M, K, 0, 5, 7), _held(torch, b, N, K, 0, 5, 8)
    assert not _product(torch, b, a, w, M, N, K, torch.float32).any()                             # below the smallest number: zero


@pytest.mark.parametrize("M,N,K", FORMS)
def test_rows_without_a_number(M, N, K):
    """One scale of a row, in its first, a middle or its last block, and codes that are all zero there."""
    torch, b = _torch()
    a, w = _held(torch, b, M, K, 120, 130, 9), _held(torch, b, N, K, 120, 130, 10)
    last = -(-K // 32) - 1
    want = torch.zeros((M, N), dtype=torch.bool, device="cuda")
    for k, r in enumerate((0, M // 2, M - 1)[:M]):
        if M > 1:
            a[1][r, (0, last // 2, last)[k]] = 255
            want[r] = True
    for k, r in enumerate((1, N // 3, N - 1)):
        w[1][r, (last, 0, last // 2)[k]] = 255
        w[0][r] = 0
        want[:, r] = True
    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        assert torch.equal(torch.isnan(_product(torch, b, a, w, M, N, K, dtype)), want)
