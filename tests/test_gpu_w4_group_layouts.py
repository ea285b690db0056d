"""The group quantizer and its inverse where rows lie on 16-byte boundaries only, and for groups that are no power of two: codes, scales and
zero-points equal to the definition in numpy."""
import numpy as np
import pytest
import torch

from paper_2507_14811_b200 import binding as B
from test_gpu_w4_group import BF, DEV, F32, pack_np, quantize_np, weights

pytestmark = pytest.mark.gpu


def odd16(t, pitch=1):
    """A copy on the GPU whose base address is an odd multiple of 16 bytes, and its pitch as well (pitch=1) or not (0)."""
    unit = 16 // t.element_size()
    units = -(-t.shape[1] // unit)
    units += (units + pitch) % 2
    buf = torch.zeros(((t.shape[0] + 1) * units + 1) * unit, dtype=t.dtype, device=DEV)
    assert buf.data_ptr() % 32 == 0
    out = buf[unit:unit + t.shape[0] * units * unit].view(t.shape[0], units * unit)[:, :t.shape[1]]
    return out.copy_(t)


def check(W, laid_out, G, s_dtype, zp):
    N, K = W.shape
    codes, s, z = quantize_np(W.float().numpy(), G, s_dtype == BF, zp)
    W4, s_w, z_w = B.segquant_quantize_w4_group(laid_out, G, s_dtype, zp)
    np.testing.assert_array_equal(s_w.float().cpu().numpy(), s)
    if zp:
        np.testing.assert_array_equal(z_w.cpu().numpy(), z)
    np.testing.assert_array_equal(W4.cpu().numpy(), pack_np(codes))
    spread = lambda t: np.repeat(t, G, 0)[:K].T
    value = ((codes - (spread(z) if zp else 0)).astype(np.float32) * spread(s)).astype(np.float32)
    for out in (F32, BF):
        assert torch.equal(B.segquant_dequantize_w4_group(W4, s_w, G, K, z_w, dtype=out).cpu(), torch.from_numpy(value).to(out))


@pytest.mark.parametrize("zp", [False, True])
@pytest.mark.parametrize("s_dtype", [F32, BF])
@pytest.mark.parametrize("pitch", [0, 1])
@pytest.mark.parametrize("N,K,G,dtype", [(32, 512, 32, BF), (70, 1544, 64, BF), (33, 1028, 128, F32), (16, 2056, 256, BF), (40, 1024, 512, F32)])
def test_rows_on_odd_multiples_of_16_bytes(N, K, G, dtype, pitch, s_dtype, zp):
    W = weights(N, K, N + K + G, dtype)
    laid_out = odd16(W, pitch)
    assert laid_out.data_ptr() % 32 == 16 and (laid_out.stride(0) * laid_out.element_size()) % 32 == 16 * pitch
    check(W, laid_out, G, s_dtype, zp)


@pytest.mark.parametrize("zp", [False, True])
@pytest.mark.parametrize("s_dtype", [F32, BF])
@pytest.mark.parametrize("N,K,G,dtype", [(9, 2000, 768, F32), (20, 700, 768, BF), (33, 3000, 768, BF), (5, 2700, 1280, F32), (18, 1300, 1280, BF)])
def test_groups_that_are_no_power_of_two(N, K, G, dtype, s_dtype, zp):
    W = weights(N, K, N + K + G, dtype)
    check(W, odd16(W), G, s_dtype, zp)
