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
