"""Scales whose multiple by log2(e) is beyond 32 bits would make every exponential NaN: refused."""
import ctypes


def test_scales_beyond_what_an_exponential_takes_are_refused():
    from paper_1912_08756_amd import binding as b
    lib, p = b.load(), ctypes.c_void_p(256)
    for scale, refused in ((2.3e38, False), (2.4e38, True), (3.4e38, True), (1e-38, False)):
        rc = lib.icq_distill(p, 0, 2, 10, 10, scale, p, p, 3, -1.0, None, p, None, None, None, 0, None, 0, None)       # (no workspace: goes no further)
        assert (rc == b.ICQ_ERR_ARG) == refused, scale
        if refused:
            assert lib.icq_distill_backward(p, 0, 2, 10, 10, scale, p, p, 3, -1.0, None, p, None, ctypes.c_void_p(1 << 20), 10, None) == b.ICQ_ERR_ARG
