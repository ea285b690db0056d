"""Block norms that write over what they read, in the shapes where a row's successor is fetched before the row is stored: rows of 8 and 16
lanes whose samples end inside a warp, two rows a block, rows whose vectors are made in two steps; and the largest values."""
import pytest
import torch

from paper_2507_14811_b200 import binding as B
from test_gpu_block_norm import BF, CASES, DEV, F32, build, check_values, reference

pytestmark = pytest.mark.gpu


def case_of(M, C, T):
    return next(c for c in CASES if c[:3] == (M, C, T))


@pytest.mark.parametrize("case", [case_of(5003, 64, 100), case_of(3001, 128, 1), case_of(3000, 100, 17), case_of(1250, 6000, 1250),
                                  case_of(760, 8001, 100), case_of(801, 5000, 401), case_of(2, 16384, 2), case_of(300, 12000, 300),
                                  (700, 16384, 350, BF, BF, "rms", "layer", ("post_w", "post_b", "gate", "w", "b", "scale", "shift"), True, True, False)])
def test_outputs_in_the_place_of_inputs(case):
    R, Y, a = build(case)
    want = B.segquant_block_norm(R, Y, **a)
    for swap in (False, True):                               # H over R and out over Y, or the other way round
        R, Y, a = build(case)
        H, O = (Y, R) if swap else (R, Y)
        got = B.segquant_block_norm(R, Y, H=H, out=O, **a)
        assert got[0].data_ptr() == H.data_ptr() and torch.equal(H, want[0]) and torch.equal(O, want[1])
    R, Y, a = build(case)
    C = R.shape[1]
    s = torch.ones(1, device=DEV) * 0.02
    seg = B.SegTable([0, C], [0, 8])
    _, codes, _ = B.segquant_block_norm_quantize(R, seg, s, None, "int8", Y, **a)
    H, again, _ = B.segquant_block_norm_quantize(R, seg, s, None, "int8", Y, H=R, **a)
    assert torch.equal(R, want[0]) and torch.equal(again, codes)


@pytest.mark.parametrize("norm", ["rms", "layer"])
@pytest.mark.parametrize("M,C", [(3, 64), (3, 16384), (1300, 1024)])
def test_values_up_to_the_range_of_the_sum_of_squares(M, C, norm):
    """|x| below 2^64 / sqrt(C): the sum of a row's squares is below 2^128."""
    g = torch.Generator(device=DEV).manual_seed(C)
    x = (torch.rand((M, C), generator=g, device=DEV) * 0.5 + 0.5) * (0.99 * 2.0 ** 64 / C ** 0.5)
    x[:, ::2] *= -1
    if norm == "layer":                                      # (the centred values have to be in the range)
        x -= x.double().mean(1, keepdim=True).float()
        x *= 0.9
    _, got = B.segquant_block_norm(x, norm=norm, eps=1e-6)
    assert bool(torch.isfinite(got).all())
    check_values(got, reference(x, None, dict(norm=norm, eps=1e-6))[1], "out")
