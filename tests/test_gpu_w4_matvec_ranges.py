"""The matrix-vector product with 4-bit weights at the ends of its ranges: activations that are no numbers behind an activation function."""
import pytest
import torch

from paper_2507_14811_b200 import binding as B
from test_gpu_w4_group import random_codes

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("x", [BF, F32])
@pytest.mark.parametrize("y", [BF, F32])
def test_what_is_no_number_stays_none_behind_an_activation(x, y, act):
    """NaN and infinities of either sign make their row NaN whatever the activation makes of them (GELU's limit at -inf is 0); other
    rows keep their bits."""
    M, K, N, G = 8, 600, 90, 64
    W4, s_w, z_w = random_codes(N, K, G, True, F32, 5)
    X = torch.randn((M, K), device=DEV).to(x)
    clean = B.segquant_w4_matvec(X, W4, s_w, G, z_w, act=act, y_dtype=y)
    X[1, 3], X[4, 599], X[5, 0], X[7, 300] = float("inf"), float("nan"), float("-inf"), -float("nan")
    got = B.segquant_w4_matvec(X, W4, s_w, G, z_w, act=act, y_dtype=y)
    for m in (0, 2, 3, 6):
        assert torch.equal(got[m], clean[m])
    for m in (1, 4, 5, 7):
        assert bool(torch.isnan(got[m]).all()), m
