"""4-bit weights with one scale (and zero-point) per channel and group of inputs: codes, scales and zero-points against the
definition in numpy (fp32 divisions are IEEE on both sides, so they have to be equal), and the matrix-vector product against
64-bit sums.

Tolerance of the product.  An activation enters as a fixed-point number that is off by at most 2^-22 of the largest magnitude of
its row in its 256 inputs, or 2^-123; products with codes and their sums over a block (a group, 128 inputs of a longer one) are exact integers.
Behind that roundings of 2^-24 of partial sums that are no larger than the sum of magnitudes (of the three bytes of an activation: at most
1.02 times that of the activation, and the fixed-point error again): one sum per block and one per 256 inputs, then sums over at
most eight CTAs, sixteen runs and three bytes, and the bias.  The activation functions come with the errors that the C header gives.  bf16
outputs are rounded once more, by at most half a step (2^-8)."""
import numpy as np
import pytest
import torch

from paper_2507_14811_b200 import binding as B
from paper_2507_14811_b200.layer import W4GroupLinear

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


def pitched(t, unit=16, extra=0):
    """A copy on the GPU with rows on 16-byte boundaries (`extra` further units of pitch)."""
    buf = torch.zeros((t.shape[0], (-(-t.shape[1] // unit) + extra) * unit), dtype=t.dtype, device=DEV)
    buf[:, : t.shape[1]] = t.to(DEV)
    return buf[:, : t.shape[1]]


def stored(s, bf16):
    """fp32 numpy -> fp32 numpy rounded to the storage type; 0 -> 1."""
    if bf16:
        s = torch.from_numpy(s).to(BF).float().numpy()
    return np.where(s == 0, np.float32(1), s).astype(np.float32)


def quantize_np(W, G, bf16, zp):
    """codes [N, K] int, scales [groups, N] fp32, zero-points [groups, N] int | None by the definition."""
    N, K = W.shape
    codes, scales, zeros = np.zeros((N, K), np.int64), [], []
    for k in range(0, K, G):
        w = W[:, k:k + G].astype(np.float32)
        if zp:
            lo, hi = np.minimum(w.min(1), 0).astype(np.float32), np.maximum(w.max(1), 0).astype(np.float32)
            s = stored((hi - lo) / np.float32(15), bf16)
            z = -8 - np.rint(lo / s)
            codes[:, k:k + G] = np.clip(np.rint(w / s[:, None]) + z[:, None], -8, 7)
            zeros.append(z.astype(np.int64))
        else:
            s = stored(np.abs(w).max(1) / np.float32(7), bf16)
            codes[:, k:k + G] = np.clip(np.rint(w / s[:, None]), -7, 7)
        scales.append(s)
    return codes, np.stack(scales), np.stack(zeros) if zp else None


def pack_np(codes):
    N, K = codes.shape
    even = np.zeros((N, (K + 1) // 2 * 2), np.int64)
    even[:, :K] = codes & 15
    return (even[:, 0::2] | even[:, 1::2] << 4).astype(np.uint8)


def weights(N, K, seed, dtype=F32):
    g = torch.Generator().manual_seed(seed)
    W = torch.randn((N, K), generator=g) * 0.02
    W[0] = 0.0                                               # no range at all
    if N > 1:
        W[1] = W[1].abs()                                    # one polarity each
        W[2 % N] = -W[2 % N].abs()
    if N > 4:
        W[3] *= 1e-40                                        # scales that underflow, and some that are subnormal
        W[4] *= 1e37
    return W.to(dtype)


@pytest.mark.parametrize("zp", [False, True])
@pytest.mark.parametrize("s_dtype", [F32, BF])
@pytest.mark.parametrize("N,K,G,dtype", [
    (1, 1, 32, F32), (3, 31, 32, BF), (33, 33, 32, F32), (40, 64, 64, BF), (31, 130, 64, F32), (64, 255, 128, BF), (37, 1111, 128, F32),
    (100, 512, 256, BF), (20, 777, 256, F32), (9, 1300, 512, BF), (5, 900, 1024, F32), (257, 1024, 32, BF), (1003, 1152, 128, F32)])
def test_codes_scales_and_zero_points(N, K, G, dtype, s_dtype, zp):
    W = weights(N, K, N + K + G, dtype)
    codes, s, z = quantize_np(W.float().numpy(), G, s_dtype == BF, zp)
    W4, s_w, z_w = B.segquant_quantize_w4_group(pitched(W, extra=N % 2), G, s_dtype, zp)
    assert W4.shape == (N, (K + 1) // 2) and s_w.dtype == s_dtype and s_w.shape == s.shape
    np.testing.assert_array_equal(s_w.float().cpu().numpy(), s)
    if zp:
        np.testing.assert_array_equal(z_w.cpu().numpy(), z)
    else:
        assert z_w is None
    np.testing.assert_array_equal(W4.cpu().numpy(), pack_np(codes))
    # and back: one fp32 product, one rounding
    spread = lambda t: np.repeat(t, G, 0)[:K].T
    value = ((codes - (spread(z) if zp else 0)).astype(np.float32) * spread(s)).astype(np.float32)
    for out in (F32, BF):
        got = B.segquant_dequantize_w4_group(W4, s_w, G, K, z_w, dtype=out)
        assert torch.equal(got.cpu(), torch.from_numpy(value).to(out))


def test_dequantize_leaves_what_lies_outside():
    W4, s_w, z_w = B.segquant_quantize_w4_group(pitched(weights(7, 45, 1)), 32)
    buf = torch.full((8, 64), 9.0, device=DEV)
    B.segquant_dequantize_w4_group(W4, s_w, 32, 45, W=buf[:7, :45])
    assert bool(torch.all(buf[7] == 9)) and bool(torch.all(buf[:7, 45:] == 9))


# ------------------------------------------------------------------------------------------------ the product

def act64(x, act):
    if act == "silu":
        return x / (1 + torch.exp(-x))
    if act == "gelu":
        return 0.5 * x * torch.special.erfc(-x / 2 ** 0.5)
    return x


def act_error(x, act):
    """relative error of the activation (C header)"""
    if act == "silu":
        return (x.abs() + 8) * 2.0 ** -23
    if act == "gelu":
        return (3 * x * x + 48) * 2.0 ** -24
    return torch.zeros_like(x)


def random_codes(N, K, G, zp, s_dtype, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    groups = -(-K // G)
    pad = lambda n: -(-n // 16) * 16
    W4 = torch.randint(0, 256, (N, pad((K + 1) // 2)), generator=g, device=DEV, dtype=torch.uint8)[:, :(K + 1) // 2]
    s_w = ((torch.rand((groups, pad(N)), generator=g, device=DEV) + 0.5) * 0.01).to(s_dtype)[:, :N]
    z_w = torch.randint(-8, 8, (groups, pad(N)), generator=g, device=DEV, dtype=torch.int8)[:, :N] if zp else None
    return W4, s_w, z_w


def weights64(W4, s_w, z_w, G, K):
    """(c - z) s in 64 bits [N, K]"""
    n = torch.stack((W4 & 15, W4 >> 4), 2).reshape(W4.shape[0], -1)[:, :K].to(torch.int64)
    c = torch.where(n >= 8, n - 16, n).double()
    if z_w is not None:
        c = c - z_w.double().t().repeat_interleave(G, 1)[:, :K]
    return c * s_w.double().t().repeat_interleave(G, 1)[:, :K]


def check_product(Y, X, W, bias, act, G, K):
    x = X.double()
    a = act64(x, act)
    blk = min(G, 128)
    pad = torch.zeros((a.shape[0], -(-K // 256) * 256), dtype=torch.float64, device=DEV)
    pad[:, :K] = a.abs() * (1 + act_error(x, act))
    largest = pad.view(a.shape[0], -1, 256).amax(2).repeat_interleave(256, 1)[:, :K]
    fixed = (2.0 ** -22 * largest + 2.0 ** -123) @ W.abs().t()
    want = a @ W.t()
    mags = a.abs() @ W.abs().t()
    of_act = (a.abs() * act_error(x, act)) @ W.abs().t()
    if bias is not None:
        want, mags = want + bias.double(), mags + bias.double().abs()
    roundings = 3 * -(-K // blk) + 8 * 16 * 3 + 2
    tol = fixed + of_act + roundings * 2.0 ** -24 * (1.02 * mags + fixed) + 2.0 ** -140
    if Y.dtype == BF:
        tol = tol + 2.0 ** -8 * (want.abs() + tol)
    err = (Y.double() - want).abs()
    assert bool(torch.all(err <= tol)), f"worst {float((err / tol).max()):.3g} of the tolerance"


@pytest.mark.parametrize("M,K,N,G,x,y,s,zp,act,bias", [
    # one row; K of one input, one unit, a unit and one; single channels
    (1, 1, 1, 32, BF, F32, F32, False, None, False), (1, 2, 5, 32, F32, F32, BF, True, None, True),
    (1, 31, 16, 32, BF, BF, F32, True, "silu", True), (1, 32, 17, 32, F32, F32, F32, False, "gelu", False),
    (1, 256, 15, 64, BF, F32, BF, False, None, True), (1, 257, 33, 64, BF, F32, F32, True, None, True),
    (1, 1152, 6912, 128, BF, BF, F32, False, "silu", True), (1, 8192, 1000, 128, BF, F32, BF, True, None, True),
    (1, 4096, 320, 1024, F32, F32, F32, True, None, False), (1, 131072, 24, 256, F32, F32, F32, False, None, True),
    (1, 131072, 40, 32, BF, F32, BF, True, "silu", True),
    # a few rows: every number of eight-column blocks, passes of rows
    (2, 1111, 1003, 32, F32, F32, F32, True, None, True), (3, 300, 130, 128, F32, BF, F32, False, "silu", True),
    (5, 1111, 1003, 32, F32, F32, F32, True, None, True), (8, 1536, 9216, 64, BF, BF, F32, False, "silu", True),
    (8, 4608, 500, 256, BF, F32, F32, True, None, False), (9, 777, 257, 128, BF, F32, BF, True, None, True),
    (10, 640, 96, 64, F32, F32, F32, False, None, True), (11, 640, 96, 64, F32, F32, F32, False, "gelu", True),
    (16, 2048, 300, 32, BF, F32, F32, True, None, True), (17, 515, 100, 128, BF, BF, F32, False, None, False),
    (24, 1024, 64, 512, BF, F32, BF, False, None, True), (32, 300, 48, 64, BF, F32, F32, True, None, True),
    (33, 300, 48, 64, BF, F32, F32, True, None, True), (70, 200, 40, 32, BF, F32, F32, True, "silu", True),
    # activations that do not fit beside the ring in one go: fewer rows a pass
    (10, 65536, 20, 128, F32, F32, F32, False, None, True), (32, 32768, 33, 64, BF, F32, F32, True, None, True),
    # many tiles per CTA
    (1, 96, 40000, 32, BF, F32, F32, False, None, True), (4, 512, 30011, 128, BF, F32, F32, True, None, True)])
def test_product(M, K, N, G, x, y, s, zp, act, bias):
    W4, s_w, z_w = random_codes(N, K, G, zp, s, M + K + N)
    g = torch.Generator(device=DEV).manual_seed(7)
    X = (torch.randn((M, K), generator=g, device=DEV) * 2).to(x)
    b = torch.randn(N, generator=g, device=DEV) if bias else None
    Y = B.segquant_w4_matvec(X, W4, s_w, G, z_w, b, act=act, y_dtype=y)
    assert Y.shape == (M, N) and Y.dtype == y
    W = weights64(W4, s_w, z_w, G, K)
    check_product(Y, X, W, b, act, G, K)
    # the same bits again: nothing depends on the order of arrival
    assert torch.equal(Y, B.segquant_w4_matvec(X, W4, s_w, G, z_w, b, act=act, y_dtype=y))


def test_large_mean_of_activations():
    """All activations alike: sums of codes times a large number, where an offset taken out behind the sum would cost digits."""
    W4, s_w, z_w = random_codes(300, 1024, 128, True, F32, 3)
    X = 1000.0 + torch.rand((3, 1024), device=DEV)
    check_product(B.segquant_w4_matvec(X, W4, s_w, 128, z_w, None, y_dtype=F32), X, weights64(W4, s_w, z_w, 128, 1024), None, None, 128, 1024)


@pytest.mark.parametrize("x", [BF, F32])
def test_rows_do_not_see_one_another(x):
    """Infinities and NaN stay in their rows; columns that are not used by any row hold nothing that counts."""
    M, K, N, G = 7, 600, 90, 64
    W4, s_w, _ = random_codes(N, K, G, False, F32, 5)
    X = torch.randn((M, K), device=DEV).to(x)
    clean = B.segquant_w4_matvec(X, W4, s_w, G, y_dtype=F32)
    X[1, 3], X[4, 599], X[5, 0] = float("inf"), float("nan"), float("-inf")
    got = B.segquant_w4_matvec(X, W4, s_w, G, y_dtype=F32)
    for m in (0, 2, 3, 6):
        assert torch.equal(got[m], clean[m])
    for m in (1, 4, 5):
        assert bool(torch.isnan(got[m]).all())


def test_ranges_of_inputs():
    """A large value costs nothing beyond its 256 inputs; bf16 values down to 2^-14 of their largest are exact."""
    K, N, G = 512, 64, 64
    W4, s_w, z_w = random_codes(N, K, G, True, F32, 4)
    s_w.fill_(1.0)
    g = torch.Generator(device=DEV).manual_seed(6)
    X = torch.randint(-255, 256, (2, K), generator=g, device=DEV).float() * 2.0 ** -7
    X[:, ::7] *= 2.0 ** -6
    X = X.to(BF)
    W = weights64(W4, s_w, z_w, G, K)
    X[0, :256] = 0
    Y = B.segquant_w4_matvec(X, W4, s_w, G, z_w, y_dtype=F32)
    assert float((Y.double() - X.double() @ W.t()).abs().max()) <= 2.0 ** -24 * 40 * float((X.double().abs() @ W.abs().t()).max())
    big = X.clone()
    big[0, 10] = 2.0 ** 30
    Z = B.segquant_w4_matvec(big, W4, s_w, G, z_w, y_dtype=F32).double()
    only = W[:, 10] * 2.0 ** 30
    assert bool(torch.all((Z[0] - only - Y[0].double()).abs() <= 2.0 ** -23 * only.abs() + 2.0 ** -20 * (X.double().abs() @ W.abs().t())[0]))


def test_largest_values_and_subnormals_of_fp32():
    K, N, G = 64, 40, 32
    W4, s_w, _ = random_codes(N, K, G, False, F32, 6)
    W = weights64(W4, s_w, None, G, K)
    X = torch.randn((3, K), device=DEV)
    X[0] *= 2.0 ** 115
    X[1] *= 2.0 ** -120                                      # below the smallest range
    X[2, :] = 0
    X[2, 5] = torch.finfo(F32).max / 2 ** 8                   # (a whole significand of ones)
    Y = B.segquant_w4_matvec(X, W4, s_w, G, y_dtype=F32)
    check_product(Y, X, W, None, None, G, K)


def test_strides_alignment_and_what_lies_outside():
    """X and Y at odd addresses and pitches, a wider pitch of weights and scales; nothing but Y is written."""
    M, K, N, G = 5, 333, 77, 64
    W4, s_w, z_w = random_codes(N, K, G, True, BF, 8)
    wide4, wide_s, wide_z = pitched(W4, 16, 2), pitched(s_w, 16, 1), pitched(z_w, 16, 3)
    base = torch.randn((M, 2 * K + 3), device=DEV).to(BF)
    X = base[:, 1:K + 1]
    want = B.segquant_w4_matvec(X.contiguous(), W4, s_w, G, z_w, y_dtype=F32)
    buf = torch.full((M + 1, N + 9), 3.0, device=DEV)
    Y = buf[:M, 1:N + 1]
    out = B.segquant_w4_matvec(X, wide4, wide_s, G, wide_z, Y=Y)
    assert out.data_ptr() == Y.data_ptr() and torch.equal(Y, want)
    assert bool(torch.all(buf[M] == 3)) and bool(torch.all(buf[:M, 0] == 3)) and bool(torch.all(buf[:M, N + 1:] == 3))


def test_offsets_beyond_32_bits():
    N, K, G = 70016, 131072, 1024                            # 4.6 GB of codes
    W4 = torch.randint(0, 256, (N, K // 2), device=DEV, dtype=torch.uint8)
    s_w = (torch.rand((K // G, N), device=DEV) + 0.5) * 1e-3
    X = torch.randn((1, K), device=DEV).to(BF)
    Y = B.segquant_w4_matvec(X, W4, s_w, G, y_dtype=F32)
    for n in (0, 32767, 32768, 65535, N - 1):
        check_product(Y[:, n:n + 1], X, weights64(W4[n:n + 1], s_w[:, n:n + 1], None, G, K), None, None, G, K)


def test_streams_and_capture():
    """Two streams at once and a captured call, replayed on new inputs: every call's own bits."""
    cases = []
    for i in range(2):
        W4, s_w, z_w = random_codes(2000, 2304, 128, True, F32, 20 + i)
        cases.append(((torch.randn((4, 2304), device=DEV)).to(BF), W4, s_w, 128, z_w))
    want = [B.segquant_w4_matvec(*c, y_dtype=F32) for c in cases]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                got[i].append(B.segquant_w4_matvec(*cases[i], y_dtype=F32))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(y, want[i]) for y in got[i])
    X = cases[0][0].clone()
    Y = torch.empty((4, 2000), device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.segquant_w4_matvec(X, *cases[0][1:], Y=Y)
    X.copy_(cases[1][0])
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(Y, B.segquant_w4_matvec(cases[1][0], *cases[0][1:], y_dtype=F32))


def test_layer_object():
    g = torch.Generator().manual_seed(2)
    W, b = torch.randn((300, 200), generator=g) * 0.02, torch.randn(300, generator=g)
    for zp in (False, True):
        layer = W4GroupLinear(W, b, group=64, zero_points=zp, s_dtype=BF)
        X = torch.randn((3, 200), generator=g).to(DEV)
        W4, s_w, z_w = B.segquant_quantize_w4_group(W.to(DEV), 64, BF, zp)
        assert torch.equal(layer.forward(X, act="silu"), B.segquant_w4_matvec(X, W4, s_w, 64, z_w, b.to(DEV), act="silu"))
        back = layer.weights(F32)
        assert float((back.cpu() - W).abs().max()) <= 0.02 * 5 / 7


def test_refusals_on_the_gpu():
    W4, s_w, z_w = random_codes(64, 128, 64, True, F32, 9)
    X = torch.zeros((2, 128), dtype=BF, device=DEV)
    with pytest.raises(ValueError, match="s_w"):
        B.segquant_w4_matvec(X, W4, s_w[:1], 64, z_w)                     # fewer groups than K has
    with pytest.raises(ValueError, match="Wq4"):
        B.segquant_w4_matvec(X[:, :100], W4, s_w, 64, z_w)                # another K
    with pytest.raises(TypeError, match="z_w"):
        B.segquant_w4_matvec(X, W4, s_w, 64, z_w.to(torch.int32))
    with pytest.raises(ValueError, match="bias"):
        B.segquant_w4_matvec(X, W4, s_w, 64, z_w, torch.zeros(63, device=DEV))
    with pytest.raises(ValueError, match="CUDA"):
        B.segquant_w4_matvec(X.cpu(), W4, s_w, 64, z_w)
    with pytest.raises(B.SegquantError, match="UNSUPPORTED"):             # Y in X's memory
        both = torch.zeros((2, 128), dtype=BF, device=DEV)
        B.segquant_w4_matvec(both, W4, s_w, 64, z_w, Y=both[:, :64])
    with pytest.raises(B.SegquantError, match="UNSUPPORTED"):
        B.segquant_w4_matvec(X, W4, s_w[:2], 96, z_w[:2])                 # a group that is none of the sizes
    with pytest.raises(B.SegquantError, match="SHAPE|NULL"):
        B.segquant_w4_matvec(X[:0], W4, s_w, 64, z_w)                     # no rows (an empty tensor has no address)
