"""4-bit calls whose blocks are more than one launch's, and offsets beyond 32 bits: results are those of calls on parts."""
import pytest

gpu = pytest.mark.gpu


def _torch():
    import torch
    from paper_1912_08756_amd import binding
    binding.load()
    return torch, binding


@gpu
def test_more_rows_than_a_launch_has_threads_for():
    """2^28 rows of one group of 128 each: sixteen threads to a group."""
    torch, b = _torch()
    rows, cols = (1 << 28) + 5, 3
    x = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda")
    x.view(torch.int16).random_(0x3000, 0x4F00, generator=torch.Generator(device="cuda").manual_seed(1))
    codes, scales = b.icq_mx_codes(rows, cols), b.icq_mx_scales(rows, cols)
    scales.untyped_storage().fill_(0)
    b.icq_mx_quantize(x, codes, scales)
    some = 1 << 16
    for at in (0, (1 << 27) - some // 2, rows - some):
        c, s = b.icq_mx_codes(some, cols), b.icq_mx_scales(some, cols)
        b.icq_mx_quantize(x[at:at + some], c, s)
        assert torch.equal(codes[at:at + some], c) and torch.equal(scales[at:at + some], s)
    assert bool((scales > 0).all())                            # every row was done
    values = torch.full((rows, cols), float("nan"), dtype=torch.bfloat16, device="cuda")
    b.icq_mx_dequantize(codes, scales, values)
    for at in (0, (1 << 27) - some // 2, rows - some):
        v = torch.empty((some, cols), dtype=torch.bfloat16, device="cuda")
        b.icq_mx_dequantize(codes[at:at + some], scales[at:at + some], v)
        assert torch.equal(values[at:at + some], v)
    assert not bool(torch.isnan(values).any())


@gpu
@pytest.mark.parametrize("block", [1, 32])
def test_more_tiles_than_a_launch_has_threads_for(block):
    """2^23 tiles of 128 rows and one column: 256 threads to a tile; one row of 2^29 bytes of codes."""
    torch, b = _torch()
    rows = (1 << 30) + 300
    x = torch.empty((rows, 1), dtype=torch.bfloat16, device="cuda")
    x.view(torch.int16).random_(0x3000, 0x4F00, generator=torch.Generator(device="cuda").manual_seed(2))
    codes, scales = b.icq_mx_codes(1, rows), b.icq_mx_scales(1, rows)
    scales.untyped_storage().fill_(0)
    b.icq_mx_quantize(x, None, None, codes, scales, block_rows=block)
    some = 1 << 16
    for at in (0, (1 << 29) - some // 2, rows // 128 * 128 - some):
        c, s = b.icq_mx_codes(1, some), b.icq_mx_scales(1, some)
        b.icq_mx_quantize(x[at:at + some], None, None, c, s, block_rows=block)
        assert torch.equal(codes[:, at // 2:(at + some) // 2], c) and torch.equal(scales[:, at // 32:(at + some) // 32], s)
    assert bool((scales > 0).all())


@gpu
@pytest.mark.parametrize("M", [5, 40])
def test_held_rows_beyond_32_bits_of_offset(M):
    """Matrices of more than 2^32 bytes of codes."""
    torch, b = _torch()
    N, K = (1 << 22) + 77, 2048 + 64                           # 4.3 GiB of codes
    g = torch.Generator(device="cuda").manual_seed(M)
    w, sw = b.icq_mx_codes(N, K), b.icq_mx_scales(N, K)
    w.untyped_storage().copy_(torch.randint(0, 256, (w.untyped_storage().nbytes(),), dtype=torch.uint8, device="cuda", generator=g).untyped_storage())
    sw.untyped_storage().fill_(127)
    a, sa = torch.randint(0, 256, (M, K // 2), dtype=torch.uint8, device="cuda", generator=g), torch.full((M, K // 32 + 2), 127, dtype=torch.uint8, device="cuda")[:, :K // 32]
    out = torch.empty((M, N), device="cuda")
    b.icq_mx_matmul(a, sa, w, sw, out, K=K)
    some = 1 << 12
    for at in (0, N // 2, N - some):
        part = torch.empty((M, some), device="cuda")
        need = b.icq_mx_matmul_workspace_bytes(M, some, K)
        b.icq_mx_matmul(a, sa, w[at:at + some], sw[at:at + some], part, torch.empty(need, dtype=torch.uint8, device="cuda") if need else None, K=K)
        assert torch.equal(out[:, at:at + some], part)         # (quarters below 2^24: exact in any order)


@gpu
def test_gradients_beyond_32_bits_of_offset():
    torch, b = _torch()
    n = (1 << 32) + 12345
    x = torch.empty((n,), dtype=torch.bfloat16, device="cuda")
    x.fill_(2.0 ** -14)
    x[0], x[1 << 31], x[n - 1] = 3.0, 4.0, 12.0
    lst, norm = b.icq_grad_list_create([x]), torch.empty((1,), device="cuda")
    b.icq_grad_norm_clip(lst, norm, 1.0, torch.empty(b.icq_grad_workspace_bytes(lst), dtype=torch.uint8, device="cuda"))
    want = (9.0 + 16.0 + 144.0 + (n - 3) * 2.0 ** -28) ** 0.5
    assert abs(float(norm) - want) <= 2.0 ** -23 * want
    f = 1.0 / want
    for at, v in ((0, 3.0), (1 << 31, 4.0), (n - 1, 12.0), (7, 2.0 ** -14), ((1 << 32) + 5, 2.0 ** -14)):
        assert abs(float(x[at]) - v * f) <= 2.0 ** -8 * v * f
    step = 1 << 28
    rest = torch.tensor(2.0 ** -14 * f, dtype=torch.bfloat16)
    for at in range(0, n, step):
        assert int((x[at:at + step] != rest.to(x.device)).sum()) == sum(at <= k < at + step for k in (0, 1 << 31, n - 1))
