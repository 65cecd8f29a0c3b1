"""Calls whose blocks are more than one launch's: results are those of calls on parts."""
import pytest

gpu = pytest.mark.gpu


def _torch():
    import torch
    from paper_1912_08756_amd import binding
    binding.load()
    return torch, binding


@gpu
def test_more_row_blocks_than_a_launch_has_threads_for():
    """2^28 rows of one block each: sixteen threads to a block."""
    torch, b = _torch()
    rows, cols = (1 << 28) + 5, 3
    x = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda")
    x.view(torch.int16).random_(0, 0x7000, generator=torch.Generator(device="cuda").manual_seed(1))
    codes, scales = b.icq_block_codes(rows, cols), torch.full((rows, 1), -1.0, device="cuda")
    b.icq_block_quantize(x, codes, scales)
    some = 1 << 16
    for at in (0, (1 << 27) - some // 2, rows - some):
        want, s = b.icq_block_codes(some, cols), torch.empty((some, 1), device="cuda")
        b.icq_block_quantize(x[at:at + some], want, s)
        assert torch.equal(codes[at:at + some].view(torch.uint8), want.view(torch.uint8)) and torch.equal(scales[at:at + some], s)
    assert bool((scales > 0).all())                            # every block was done


@gpu
@pytest.mark.parametrize("block", [1, 128])
def test_more_tiles_than_a_launch_has_threads_for(block):
    """2^23 tiles of 128 rows and one column: 512 threads to a tile."""
    torch, b = _torch()
    rows = (1 << 30) + 300
    x = torch.empty((rows, 1), dtype=torch.bfloat16, device="cuda")
    x.view(torch.int16).random_(0, 0x7000, generator=torch.Generator(device="cuda").manual_seed(2))
    blocks = -(-rows // 128)
    codes_t, scales_t = b.icq_block_codes(1, rows), torch.full((1, blocks), -1.0, device="cuda")
    b.icq_block_quantize(x, None, None, codes_t, scales_t, block_rows=block)
    some = 1 << 16
    for at in (0, (1 << 29) - some // 2, rows // 128 * 128 - some):
        want, s = b.icq_block_codes(1, some), torch.empty((1, some // 128), device="cuda")
        b.icq_block_quantize(x[at:at + some], None, None, want, s, block_rows=block)
        assert torch.equal(codes_t[:, at:at + some].view(torch.uint8), want.view(torch.uint8))
        assert torch.equal(scales_t[:, at // 128:at // 128 + some // 128], s)
    assert bool((scales_t > 0).all())


@gpu
@pytest.mark.parametrize("M,N,kind", [(1, (1 << 29) + 70, "bf16"), (2, (1 << 29) + 70, "f32"), (33, (1 << 30) + 200, "bf16")])
def test_products_of_more_blocks_than_a_launch_has_threads_for(M, N, kind):
    """Few rows: 64 rows of b to 512 threads.  More: tiles of 64 x 64 to 256 threads."""
    torch, b = _torch()
    K, dtype = 16, torch.float32 if kind == "f32" else torch.bfloat16
    g = torch.Generator(device="cuda").manual_seed(M)
    w = torch.empty((N, K), dtype=torch.uint8, device="cuda")
    w.view(torch.int64).random_(generator=g)                   # any bytes but NaN's
    w.bitwise_and_(0xBF)
    w = w.view(torch.float8_e4m3fn)
    a = torch.randint(0, 0x40, (M, K), dtype=torch.uint8, device="cuda", generator=g).view(torch.float8_e4m3fn)
    sa, sw = torch.rand((M, 1), device="cuda", generator=g) + 0.5, torch.rand((-(-N // 128), 1), device="cuda", generator=g) + 0.5
    out = torch.full((M, N), float("nan"), dtype=dtype, device="cuda")
    b.icq_block_matmul(a, sa, w, sw, out, None)
    some = 1 << 16
    for at in (0, (1 << 28) - some // 2, N // 128 * 128 - some):
        part = torch.empty((M, some), dtype=dtype, device="cuda")
        b.icq_block_matmul(a, sa, w[at:at + some], sw[at // 128:(at + some) // 128], part, None)
        if M > 2:                                              # (the same kernel, or one that sums in another order)
            assert torch.allclose(out[:, at:at + some].float(), part.float(), rtol=2.0 ** -6, atol=1e-3)
        else:
            assert torch.equal(out[:, at:at + some], part)
    step = 1 << 24
    for at in range(0, N, step):
        assert not bool(torch.isnan(out[:, at:at + step]).any()), at
