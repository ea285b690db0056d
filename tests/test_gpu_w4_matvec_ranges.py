"""The matrix-vector product with 4-bit weights at the ends of its ranges: activations that are no numbers behind an activation function,
zero-points anywhere in int8, activations of very different magnitude in front of fp32 outputs.

Tolerances.  u = 2^-24 is a rounding's share.  A term of a sum is on its way through at most 50 + ceil(K / 256) roundings: the zero-point's and the
scale's multiply-add, up to eight blocks of a unit, the units, then sixteen runs, the bytes, lanes, eight CTAs and the bias.  The bytes that an
activation is split into are at most 3.03 times as large together as the activation: those below the leading one, 256^p of which the
activation has at least half of, add up to at most 0.502 of 256^p, and the leading one is off the activation by that much again.
An activation is off by at most 2^-22 of the largest magnitude of its row in its 256 inputs, or 2^-123; 2^-37 instead of 2^-22 where the output is
fp32 and the activations are fp32 or come out of an activation function.  bf16 outputs are rounded once more, by at
most half a step."""
import pytest
import torch

from paper_2507_14811_b200 import binding as B
from test_gpu_w4_group import act64, act_error, random_codes, weights64

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32
U = 2.0 ** -24


def check(Y, X, W, K, act=None, fixed=2.0 ** -22, error=act_error):
    """fixed: an activation's error relative to the largest; error(x, act): the activation function's."""
    x = X.double()
    a = act64(x, act)
    of_act = a.abs() * error(x, act)
    pad = torch.zeros((a.shape[0], -(-K // 256) * 256), dtype=torch.float64, device=DEV)
    pad[:, :K] = a.abs() + of_act
    largest = pad.view(a.shape[0], -1, 256).amax(2).repeat_interleave(256, 1)[:, :K]
    off = (of_act + fixed * largest + 2.0 ** -123) * (a != 0)
    want = a @ W.t()
    tol = off @ W.abs().t() + (50 + -(-K // 256)) * U * 3.03 * ((a.abs() + off) @ W.abs().t()) + 2.0 ** -140
    if Y.dtype == BF:
        tol = tol + 2.0 ** -8 * (want.abs() + tol)
    err = (Y.double() - want).abs()
    assert bool(torch.all(err <= tol)), f"worst {float((err / tol).max()):.3g} of the tolerance"


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


@pytest.mark.parametrize("M,K,N,G,x,y", [
    (1, 1111, 77, 32, BF, F32), (3, 1000, 130, 64, F32, F32), (8, 2048, 300, 128, BF, BF), (9, 900, 64, 256, BF, F32), (6, 700, 48, 512, F32, F32)])
def test_any_zero_point(M, K, N, G, x, y):
    """Matrices packed elsewhere may have zero-points anywhere in int8."""
    W4, s_w, _ = random_codes(N, K, G, False, F32, 11)
    z_w = torch.randint(-128, 128, (s_w.shape[0], -(-N // 16) * 16), device=DEV, dtype=torch.int8)[:, :N]
    z_w[0, 0], z_w[0, 1] = -128, 127
    g = torch.Generator(device=DEV).manual_seed(12)
    X = (torch.rand((M, K), generator=g, device=DEV) + 0.5).to(x)            # (one sign: large sums)
    Y = B.segquant_w4_matvec(X, W4, s_w, G, z_w, y_dtype=y)
    check(Y, X, weights64(W4, s_w, z_w, G, K), K)


def test_zero_points_of_weights_next_to_nothing():
    """Ranges of a few subnormal steps: the quantizer's own zero-points go beyond [-8, 7] there, because its scale is a whole number of steps."""
    W = torch.full((16, 128), -22 * 2.0 ** -149)
    W4, s_w, z_w = B.segquant_quantize_w4_group(W.to(DEV), 128, F32, True)
    assert int(z_w.max()) > 7
    X = torch.full((2, 128), float(0x3F7F7F) * 2.0 ** 78, device=DEV)          # (bytes as large as they get)
    for y in (BF, F32):
        check(B.segquant_w4_matvec(X, W4, s_w, 128, z_w, y_dtype=y), X, weights64(W4, s_w, z_w, 128, 128), 128)


@pytest.mark.parametrize("ratio", [10.0 ** 3, 10.0 ** 4])
@pytest.mark.parametrize("act", [None, "silu", "gelu"])
@pytest.mark.parametrize("M", [1, 2, 5, 13])
def test_small_activations_beside_a_large_one(M, act, ratio):
    """fp32 outputs have the digits of fp32 products: one activation in 256 is `ratio` times as large as the other one that there is, and its
    weights are zero."""
    K, N, G = 1024, 64, 64
    W4, s_w, _ = random_codes(N, K, G, False, F32, 13)
    g = torch.Generator(device=DEV).manual_seed(14)
    X = torch.zeros((M, K), device=DEV)
    for u in range(K // 256):
        X[:, u * 256] = ratio
        at = torch.randint(1, 256, (M,), generator=g, device=DEV) + u * 256
        X[torch.arange(M, device=DEV), at] = torch.rand(M, generator=g, device=DEV) + 0.5
        W4[:, u * 128] &= 0xF0                               # code 0
    check(B.segquant_w4_matvec(X, W4, s_w, G, act=act, y_dtype=F32), X, weights64(W4, s_w, None, G, K), K, act, fixed=2.0 ** -37)


@pytest.mark.parametrize("x", [BF, F32])
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_activation_functions_in_front_of_fp32_outputs(x, act):
    """One activation a row, over the range in which its function's value is an ordinary number: 16 roundings and the bytes' own (a number's
    bytes below the leading one, which is at least 32 here, are together at most 0.502 / 32 of it, so that all but the last of their
    additions round 2^-24 of less than a sixtieth)."""
    K, N, G, M = 32, 8, 32, 8192
    W4 = torch.zeros((N, 16), dtype=torch.uint8, device=DEV)
    W4[:, 3] = 0x01                                          # input 6 alone counts, once
    s_w = torch.ones((1, N), device=DEV)
    X = torch.zeros((M, K), device=DEV, dtype=x)
    X[:, 6] = torch.linspace(-80.0 if act == "silu" else -9.0, 9.0, M, device=DEV).to(x)
    Y = B.segquant_w4_matvec(X, W4, s_w, G, act=act, y_dtype=F32)
    v = X[:, 6].double()
    want = act64(v, act)
    tol = want.abs() * (16 * U + 2.0 ** -37 + 1.1 * U) + 2.0 ** -123
    err = (Y[:, 0].double() - want).abs()
    assert bool(torch.all(err <= tol)), f"worst {float((err / tol).max()):.3g} of the tolerance"
    assert torch.equal(Y, Y[:, :1].expand(M, N))


@pytest.mark.parametrize("x,y", [(BF, F32), (F32, F32), (F32, BF)])
def test_scales_up_to_2_96(x, y):
    K, N, G = 512, 40, 32
    W4, s_w, _ = random_codes(N, K, G, False, F32, 15)
    z_w = torch.randint(-128, 128, (K // G, 48), device=DEV, dtype=torch.int8)[:, :N]
    s_w.copy_(s_w.clone().clamp(0.008, 0.01) * (2.0 ** 96 / 0.01))
    X = (torch.randn((3, K), device=DEV) * 2.0 ** -60).to(x)
    check(B.segquant_w4_matvec(X, W4, s_w, G, z_w, y_dtype=y), X, weights64(W4, s_w, z_w, G, K), K)


@pytest.mark.parametrize("x,y", [(BF, BF), (F32, F32)])
@pytest.mark.parametrize("M,K,N,G", [(1, 2000, 33, 768), (4, 3000, 50, 768), (2, 2700, 24, 1280), (3, 700, 17, 768)])
def test_groups_that_are_no_power_of_two(M, K, N, G, x, y):
    W4, s_w, z_w = random_codes(N, K, G, True, F32, 16)
    X = torch.randn((M, K), device=DEV).to(x)
    check(B.segquant_w4_matvec(X, W4, s_w, G, z_w, y_dtype=y), X, weights64(W4, s_w, z_w, G, K), K)
