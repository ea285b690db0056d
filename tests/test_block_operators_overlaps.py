"""What the C ABI refuses of the group quantizer, its inverse, the matrix-vector product and the block norm to codes: outputs in the
memory of scales and zero-points, which every block reads while others write (no GPU: none of these calls reaches a kernel)."""
import ctypes as C

import pytest

from test_block_operators_abi import FAKE, L, block, matvec, quantize  # noqa: F401  (L: the library)

FAR = 0x40000000     # scales and zero-points away from everything else


def test_quantizer_outputs_are_apart(L):
    """W 64 x 256 fp32 (64 KB), codes 64 x 128, scales 4 x 64 fp32, zero-points 4 x 64."""
    q = lambda **kw: quantize(L, **{**dict(s=FAR, z=2 * FAR), **kw})
    w_end, c_end, s_end = FAKE + 64 * 256 * 4, 2 * FAKE + 64 * 128, FAR + 4 * 64 * 4
    for at in (FAKE, FAKE + 1024, w_end - 16):               # in the weights
        assert q(s=at) == 5 and q(z=at) == 5
    for at in (2 * FAKE, c_end - 16):                        # in the codes
        assert q(s=at) == 5 and q(z=at) == 5
    for at in (FAR, s_end - 16):                             # zero-points in the scales
        assert q(z=at) == 5
    assert q(s=FAKE - 4 * 64 * 4 + 16) == 5 and q(z=FAKE - 4 * 64 + 16) == 5        # their ends in the weights


def test_dequantizer_writes_apart_from_scales(L):
    d = lambda **kw: quantize(L, back=True, **{**dict(s=FAR, z=2 * FAR), **kw})
    w_end = FAKE + 64 * 256 * 4
    for at in (FAKE, FAKE + 1024, w_end - 16):
        assert d(s=at) == 5 and d(z=at) == 5


def test_product_writes_apart_from_scales(L):
    """Y 4 x 64 bf16, scales 4 x 64 fp32, zero-points 4 x 64."""
    m = lambda **kw: matvec(L, **{**dict(s=FAR, z=2 * FAR), **kw})
    for at in (FAR, FAR + 512, FAR + 1024 - 2, FAR - 510):
        assert m(Y=at) == 5, hex(at)
    for at in (2 * FAR, 2 * FAR + 128, 2 * FAR + 256 - 2, 2 * FAR - 510):
        assert m(Y=at) == 5, hex(at)


def test_norm_to_codes_writes_apart_from_its_scales(L):
    """H 4 x 64 fp32, codes 4 x 64, one scale a K-segment."""
    b = lambda **kw: block(L, codes=True, **{**dict(s_pos=FAR, s_neg=2 * FAR), **kw})
    for which, at in (("s_pos", FAR), ("s_neg", 2 * FAR)):
        assert b(c_pos=at) == 5 and b(c_neg=at) == 5 and b(H=at) == 5, which
        assert b(**{which: 5 * FAKE + 252}) == 5 and b(**{which: 6 * FAKE + 252}) == 5       # its last bytes
        assert b(H=3 * FAKE, **{which: 3 * FAKE + 1020}) == 5
