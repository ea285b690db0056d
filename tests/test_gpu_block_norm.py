"""End of one block and start of the next (gate, residual, norms) against 64-bit arithmetic, as values and as codes.

Tolerance: the error of the fp32 evaluation is carried along with the 64-bit one (`Err`), to first order and with half as much
again for the second.  u = 2^-24 is a rounding's share.  A sum over a row is at most 53 additions deep (six chunks of eight in a lane,
five shuffles; or four chunks, five shuffles, sixteen warps), 64 counted.  Outputs in bf16 are rounded by at most half a step, 2^-8 of
the value.  A code has to lie between those of the two ends of the quotient's interval."""
import pytest
import torch

from paper_2507_14811_b200 import binding as B
from paper_2507_14811_b200.layer import SegQuantLinear, W4GroupLinear

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32
U, DEPTH = 2.0 ** -24, 64


class Err:
    """A 64-bit value and a bound on how far the fp32 one is from it."""

    def __init__(self, v, e=None):
        self.v, self.e = v, torch.zeros_like(v) if e is None else e

    def linear(self, factors, terms):
        """self times the factors plus the terms (each a list of factors), in any order that takes at most six roundings on the
        way of each product or term to the result: 6 u of the sum of their magnitudes.  (Here: at most two products of the factors
        among themselves, or one sum and one product, one with self, and two additions.)"""
        scale = torch.ones_like(self.v)
        for f in factors:
            scale = scale * f
        v, mags = self.v * scale, (self.v * scale).abs()
        for t in terms:
            x = torch.ones_like(self.v)
            for f in t:
                x = x * f
            v, mags = v + x, mags + x.abs()
        return Err(v, self.e * scale.abs() + 6 * U * mags)

    def normed(self, kind, eps):
        if kind == "none":
            return self
        x, e = self.v, self.e
        if kind == "layer":
            mean = x.mean(1, keepdim=True)
            e_mean = e.mean(1, keepdim=True) + DEPTH * U * x.abs().mean(1, keepdim=True) + U * mean.abs()
            x = x - mean
            e = e + e_mean + U * x.abs()
        ss = (x * x).mean(1, keepdim=True)
        rstd = (ss + eps) ** -0.5
        e_ss = 2 * (e * x.abs()).mean(1, keepdim=True) + (e * e).mean(1, keepdim=True) + (DEPTH + 3) * U * ss
        rel = 0.5 * (e_ss / (ss + eps).clamp(min=1e-300)).clamp(max=1e6) + 4 * U
        return Err(x * rstd, (e + x.abs() * (rel + U)) * rstd)


def spread(v, rows, T):
    v = v.double()
    return v[None, :] if v.dim() == 1 else v.repeat_interleave(T, 0)[:rows] if v.shape[0] > 1 else v


def reference(R, Y, a):
    M, C = (Y if R is None else R).shape
    T = a.get("rows_per_sample") or M
    get = lambda *names: [spread(a[k], M, T) for k in names if a.get(k) is not None]
    if Y is None:
        h = Err(R.double())
    else:
        u = Err(Y.double()).normed(a.get("post") or "none", a["eps"])
        alpha = [torch.tensor(a.get("alpha", 1.0), dtype=F32, device=DEV).double()]
        terms = ([] if a.get("post_b") is None else [get("post_b", "gate") + alpha]) + ([] if R is None else [[R.double()]])
        h = u.linear(get("post_w", "gate") + alpha, terms)
    modulate = [1.0 + v for v in get("scale")]
    terms = ([] if a.get("b") is None else [get("b") + modulate]) + ([] if a.get("shift") is None else [get("shift")])
    return h, h.normed(a.get("norm") or "none", a["eps"]).linear(get("w") + modulate, terms)


def check_values(got, want, what):
    tol = 1.5 * want.e + 2.0 ** -140
    if got.dtype == BF:
        tol = tol + 2.0 ** -8 * (want.v.abs() + tol)
    else:
        tol = tol + U * want.v.abs()
    err = (got.double() - want.v).abs()
    assert bool(torch.all(err <= tol)), f"{what}: worst {float((err / tol).max()):.3g} of the tolerance"


def code_value(q, code, lo, hi):
    """codes of real quotients, as numbers"""
    q = q.clamp(lo, hi)
    return torch.round(q) if code == "int8" else q.float().to(torch.float8_e4m3fn).double()


def stored_value(c, code):
    return c.view(torch.int8).double() if code == "int8" else c.view(torch.float8_e4m3fn).double()


def check_codes(c_pos, c_neg, o, kb, s_pos, s_neg, code, lo=None):
    widths = torch.tensor([b - a for a, b in zip(kb, kb[1:])], device=DEV)
    top = 127.0 if code == "int8" else 448.0
    low = -top if s_neg is None else lo if lo is not None else -128.0 if code == "int8" else -448.0
    same = total = 0
    for c, s, a, b in ((c_pos, s_pos, low if s_neg is None else 0.0, top), (c_neg, s_neg, low, 0.0)):
        if c is None:
            continue
        step = s.double().repeat_interleave(widths)
        q, e = o.v / step, (1.5 * o.e + U * o.v.abs() + 2.0 ** -140) / step + U * (o.v / step).abs()
        got = stored_value(c, code)
        # the clamp in fp32 of e4m3's conversion has a rounding of its own below its subnormals' half step
        assert bool(torch.all(got >= code_value(q - e, code, a, b))) and bool(torch.all(got <= code_value(q + e, code, a, b)))
        same += int((got == code_value(q, code, a, b)).sum())
        total += got.numel()
    assert same >= 0.99 * total or total - same <= 3


def rows(g, M, C, dtype, extra=0, spread_rows=True):
    buf = torch.zeros((M, (C + 7) // 8 * 8 + 8 * extra), dtype=dtype, device=DEV)
    x = torch.randn((M, C), generator=g, device=DEV) + 0.25
    if spread_rows:
        x = x * torch.exp(torch.randn((M, 1), generator=g, device=DEV))
    buf[:, :C] = x
    return buf[:, :C]


def vectors(g, C, samples, pdt, names, odd):
    """Vectors over the channels; odd: chunks of a wider matrix at addresses that no 16 bytes divide."""
    a = {}
    for i, k in enumerate(names):
        if k in ("gate", "scale", "shift"):
            buf = torch.randn((samples, 3 * C + 5), generator=g, device=DEV).to(pdt)
            at = {"gate": 2 * C + 1, "scale": C, "shift": 0}[k] if odd else 0
            a[k] = buf[:, at:at + C] if odd else (torch.randn((samples, C), generator=g, device=DEV) * 0.5).to(pdt)
        else:
            v = (torch.randn(C + 3, generator=g, device=DEV) * 0.5 + (1.0 if k.endswith("w") else 0.0)).to(pdt)
            a[k] = v[1:C + 1] if odd else v[:C].clone()
    return a


ALL = ("post_w", "post_b", "gate", "w", "b", "scale", "shift")
CASES = [
    # M, C, T, types of rows and vectors, post, norm, vectors, R, Y, odd addresses
    (1, 1, 1, F32, F32, "none", "layer", ("w", "b"), True, False, False),
    (1, 7, 1, BF, F32, "layer", "rms", ALL, True, True, True),
    (3, 8, 3, BF, BF, "rms", "layer", ALL, True, True, False),
    (5, 64, 2, F32, BF, "layer", "layer", ALL, True, True, False),
    (2, 1111, 1, F32, F32, "none", "rms", ("w",), True, False, True),
    (7, 1024, 4, BF, BF, "none", "layer", ("gate", "scale", "shift"), True, True, False),
    (9, 1025, 4, F32, F32, "rms", "rms", ("post_w", "w"), True, True, True),
    (4, 2049, 4, BF, F32, "none", "none", ("gate",), True, True, False),
    (3, 4096, 1, BF, BF, "layer", "none", ("post_w", "post_b", "scale", "shift"), False, True, False),
    (6, 4100, 5, F32, F32, "layer", "layer", ALL, True, True, True),
    (2, 8200, 1, BF, BF, "rms", "layer", ALL, True, True, False),
    (2, 16384, 2, F32, F32, "layer", "rms", ALL, True, True, False),
    (1, 16383, 1, BF, BF, "rms", "layer", ("post_w", "b"), True, True, False),
    # many rows: one warp each, every number of chunks a lane; a last sample that is short
    (1300, 200, 256, BF, BF, "none", "layer", ("gate", "scale", "shift"), True, True, False),
    (1300, 256, 1, F32, F32, "rms", "rms", ALL, True, True, False),
    (1301, 257, 77, BF, F32, "layer", "layer", ALL, True, True, True),
    (1200, 512, 1200, F32, BF, "none", "rms", ("w",), True, False, False),
    (1500, 1000, 499, BF, BF, "rms", "layer", ALL, True, True, False),
    (1201, 1152, 256, BF, BF, "none", "layer", ("gate", "scale", "shift"), True, True, False),
    (1201, 1152, 256, F32, F32, "layer", "layer", ALL, True, True, False),
    (2500, 1536, 1250, BF, F32, "rms", "rms", ("post_w", "w"), True, True, False),
    (1190, 1543, 100, BF, BF, "none", "layer", ("scale", "shift"), False, True, False),
    (5000, 40, 7, F32, F32, "layer", "layer", ALL, True, True, True),
    # rows of a few lanes, samples that end inside a warp or a block; vectors of every row
    (5003, 64, 100, BF, BF, "rms", "layer", ALL, True, True, False),
    (3001, 128, 1, F32, F32, "none", "layer", ("gate", "scale", "shift"), True, True, False),
    (3000, 100, 17, BF, F32, "layer", "rms", ALL, True, True, True),
    (40000, 8, 40000, BF, BF, "none", "rms", ("w",), True, False, False),
    (1190, 640, 1, BF, BF, "rms", "layer", ALL, True, True, False),
    (1300, 1300, 3, F32, BF, "layer", "layer", ALL, True, True, False),
    # wider rows, many of them
    (1200, 4096, 64, BF, BF, "none", "layer", ("gate", "scale", "shift"), True, True, False),
    (1190, 2000, 16, F32, F32, "layer", "layer", ALL, True, True, False),
    (1184, 3080, 1184, BF, BF, "rms", "rms", ("post_w", "w"), True, True, False),
    (1184, 1500, 592, BF, BF, "layer", "layer", ALL, True, True, False),
    (1250, 6000, 1250, BF, BF, "rms", "rms", ("post_w", "w"), True, True, False),
    (760, 8001, 100, BF, F32, "layer", "layer", ALL, True, True, True),
    (801, 5000, 401, F32, F32, "none", "layer", ("gate", "scale", "shift"), True, True, False),
    (750, 5000, 2, BF, BF, "rms", "layer", ALL, True, True, False),
    (400, 6000, 200, BF, BF, "none", "layer", ("gate", "scale", "shift"), True, True, False),
    (300, 12000, 300, F32, BF, "rms", "layer", ALL, True, True, False),
]


def build(case, seed=0):
    M, C, T, dt, pdt, post, norm, names, has_r, has_y, odd = case
    g = torch.Generator(device=DEV).manual_seed(M + C + seed)
    a = dict(post=post, norm=norm, rows_per_sample=T, eps=1e-5, alpha=0.7 if odd else 1.0)
    a.update(vectors(g, C, -(-M // T), pdt, names, odd))
    return rows(g, M, C, dt) if has_r else None, rows(g, M, C, dt, 1) if has_y else None, a


@pytest.mark.parametrize("case", CASES)
def test_values(case):
    R, Y, a = build(case)
    H, O = B.segquant_block_norm(R, Y, **a)
    h, o = reference(R, Y, a)
    if Y is None:
        assert H is R
    else:
        check_values(H, h, "H")
    check_values(O, o, "out")


@pytest.mark.parametrize("code,dual", [("int8", False), ("int8", True), ("e4m3", False), ("e4m3", True)])
@pytest.mark.parametrize("case", CASES)
def test_codes(case, code, dual):
    R, Y, a = build(case)
    M, C = (Y if R is None else R).shape
    P = min(3, C)
    kb = [0, C] if P == 1 else [0, C // 3 + 1 if C > 3 else 1, C] if P == 2 else [0, C // 3, C // 3 * 2 + 1, C]
    P = len(kb) - 1
    h, o = reference(R, Y, a)
    top = 127.0 if code == "int8" else 448.0
    s_pos = torch.tensor([2.0 + p for p in range(P)], device=DEV) / top
    s_neg = s_pos * 0.6 if dual else None
    H, c_pos, c_neg = B.segquant_block_norm_quantize(R, B.SegTable(kb, [0, 8]), s_pos, s_neg, code, Y, **a)
    if Y is not None:
        assert torch.equal(H, B.segquant_block_norm(R, Y, store_out=False, **a)[0])
        check_values(H, h, "H")
    check_codes(c_pos, c_neg, o, kb, s_pos, s_neg, code)
    if code == "int8" and dual:
        H, c_pos, c_neg = B.segquant_block_norm_quantize(R, B.SegTable(kb, [0, 8]), s_pos, s_neg, code, Y, flags=B.SQ_FLAG_QMIN_SYM, **a)
        check_codes(c_pos, c_neg, o, kb, s_pos, s_neg, code, lo=-127.0)


@pytest.mark.parametrize("s", [2.0 ** -90, 2.0 ** 105, 2.0 ** -40])
def test_codes_behind_extreme_scales(s):
    R, Y, a = build(CASES[13])
    _, o = reference(R, Y, a)
    kb = [0, 100, 200]
    s_pos = torch.tensor([s, 0.02], device=DEV)
    for code in ("int8", "e4m3"):
        for s_neg in (None, s_pos):
            _, c_pos, c_neg = B.segquant_block_norm_quantize(R, B.SegTable(kb, [0, 8]), s_pos, s_neg, code, Y, **a)
            check_codes(c_pos, c_neg, o, kb, s_pos, s_neg, code)


@pytest.mark.parametrize("case", [CASES[4], CASES[9], CASES[15], CASES[18], CASES[20]])
def test_in_place_and_what_lies_outside(case):
    R, Y, a = build(case)
    M, C = R.shape
    want = B.segquant_block_norm(R, Y, **a)
    guard = torch.full((M + 1, (C + 15) // 8 * 8), 5.0, dtype=R.dtype, device=DEV)
    out = guard[:M, :C]
    got = B.segquant_block_norm(R, Y, out=out, **a)
    assert torch.equal(got[1], want[1])
    assert bool(torch.all(guard[M] == 5)) and bool(torch.all(guard[:M, C:] == 5))
    if Y is not None:
        pad = [t._base[:, C:].clone() for t in (R, Y)]
        got = B.segquant_block_norm(R, Y, H=R, out=Y, **a)
        assert got[0].data_ptr() == R.data_ptr() and torch.equal(R, want[0]) and torch.equal(Y, want[1])
        assert all(torch.equal(t._base[:, C:], p) for t, p in zip((R, Y), pad))
    codes = torch.full((M + 1, (C + 31) // 16 * 16), 77, dtype=torch.uint8, device=DEV)
    R, Y, a = build(case)
    B.segquant_block_norm_quantize(R, B.SegTable([0, C], [0, 8]), torch.ones(1, device=DEV) * 0.02, None, "int8", Y, c_pos=codes[:M, :C], **a)
    assert bool(torch.all(codes[M] == 77)) and bool(torch.all(codes[:M, C:] == 77))


@pytest.mark.parametrize("M,C", [(6, 300), (1400, 300), (3, 5000)])
@pytest.mark.parametrize("norm", ["rms", "layer"])
def test_rows_do_not_see_one_another(M, C, norm):
    """NaN, infinities, rows of one value and of zeros: each row's own affair."""
    g = torch.Generator(device=DEV).manual_seed(1)
    R = rows(g, M, C, F32)
    _, clean = B.segquant_block_norm(R, norm=norm, eps=1e-5)
    R[0, 5], R[1, C - 1], R[2] = float("nan"), float("inf"), 3.0
    if M > 3:
        R[3] = 0.0
    _, got = B.segquant_block_norm(R, norm=norm, eps=1e-5)
    assert torch.equal(got[4:], clean[4:])
    assert bool(torch.isnan(got[0]).all()) and bool(torch.isnan(got[1, C - 1]))
    if norm == "layer":
        assert bool(torch.all(got[2].abs() <= 1e-2))         # the mean of equal values, rounded, over sqrt(eps)
    else:
        check_values(got[2:3], reference(R[2:3], None, dict(norm=norm, eps=1e-5))[1], "constant row")
    if M > 3:
        assert bool(torch.all(got[3] == 0))
    _, got0 = B.segquant_block_norm(torch.zeros((2, 64), device=DEV), norm=norm, eps=0.0)
    assert bool(torch.isnan(got0).all())                     # 0 / 0, as the formula has it


def test_large_mean():
    """A layer norm's variance is that of the centred values: a mean of 1000 spreads costs no digits of it."""
    g = torch.Generator(device=DEV).manual_seed(2)
    for M, C in ((2, 1000), (1300, 1000)):
        R = torch.randn((M, C), generator=g, device=DEV) + 1000.0
        _, got = B.segquant_block_norm(R, norm="layer", eps=1e-6)
        check_values(got, reference(R, None, dict(norm="layer", eps=1e-6))[1], "out")


def test_broadcast_vectors():
    """[C], [1, C] and [samples, C] of equal rows are the same modulation."""
    g = torch.Generator(device=DEV).manual_seed(3)
    R, Y = rows(g, 50, 320, BF), rows(g, 50, 320, BF)
    v = torch.randn((3, 320), generator=g, device=DEV).to(BF)
    forms = [lambda t: t, lambda t: t[None], lambda t: t[None].repeat(5, 1), lambda t: t[None].expand(5, 320)]
    outs = [B.segquant_block_norm(R, Y, gate=f(v[0]), scale=f(v[1]), shift=f(v[2]), rows_per_sample=10) for f in forms]
    for H, O in outs[1:]:
        assert torch.equal(H, outs[0][0]) and torch.equal(O, outs[0][1])


def test_a_copy_of_the_stream():
    """H given without Y: the residual stream is stored there as it is, with and without an output."""
    g = torch.Generator(device=DEV).manual_seed(8)
    for M, C in ((5, 301), (1300, 301)):
        R = rows(g, M, C, BF)
        H = torch.zeros((M, 304), dtype=BF, device=DEV)[:, :C]
        got, O = B.segquant_block_norm(R, H=H)
        assert got is H and torch.equal(H, R) and torch.equal(O, B.segquant_block_norm(R)[1])
        H.zero_()
        assert B.segquant_block_norm(R, H=H, store_out=False)[1] is None and torch.equal(H, R)


def test_offsets_beyond_32_bits():
    M, C = 140000, 16384                                     # 4.6 GB of bf16
    R = torch.zeros((M, C), dtype=BF, device=DEV)
    tail = torch.randn((3, C), device=DEV).to(BF)
    R[-3:] = tail
    _, O = B.segquant_block_norm(R, norm="rms", out=R)       # in place
    check_values(O[-3:], reference(tail, None, dict(norm="rms", eps=1e-6))[1], "last rows")
    assert bool(torch.all(O[:-3].view(torch.int16).view(-1)[::4097] == 0))


def test_streams_and_capture():
    R, Y, a = build(CASES[18])
    R2, Y2, _ = build(CASES[18], seed=9)
    want = [B.segquant_block_norm(r, y, **a) for r, y in ((R, Y), (R2, Y2))]
    streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], [[], []]
    torch.cuda.synchronize()
    for _ in range(5):
        for i, (r, y) in enumerate(((R, Y), (R2, Y2))):
            with torch.cuda.stream(streams[i]):
                got[i].append(B.segquant_block_norm(r, y, **a))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(h, want[i][0]) and torch.equal(o, want[i][1]) for h, o in got[i])
    H, O = torch.empty_like(R), torch.empty_like(R)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.segquant_block_norm(R, Y, H=H, out=O, **a)
    R.copy_(R2)
    Y.copy_(Y2)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(H, want[1][0]) and torch.equal(O, want[1][1])


def test_a_block_with_its_modulation():
    """The operators together, as a block uses them: conditioning vectors -> modulation by 4-bit weights -> modulated norm -> codes
    -> layer -> gated residual and the next modulated norm -> codes -> layer; against the separate calls, bit for bit, and the
    whole against 64-bit arithmetic on the quantized weights."""
    g = torch.Generator().manual_seed(4)
    samples, T, C, F = 3, 50, 256, 512
    mod = W4GroupLinear(torch.randn((6 * C, C), generator=g) * 0.03, torch.randn(6 * C, generator=g) * 0.1, group=64)
    fc1 = SegQuantLinear(torch.randn((F, C), generator=g) * 0.05, torch.randn(F, generator=g) * 0.1, [0, 128, C], [0, F], False)
    fc2 = SegQuantLinear(torch.randn((C, F), generator=g) * 0.05, None, [0, F], [0, C], True)
    out = SegQuantLinear(torch.randn((C, C), generator=g) * 0.05, None, [0, C], [0, C], True, "e4m3")
    c = torch.randn((samples, C), generator=g).to(DEV)
    R = torch.randn((samples * T, C), generator=g).to(DEV).to(BF)

    six = mod.forward(c, act="silu")                         # [samples, 6 C] bf16
    shift1, scale1, gate1, shift2, scale2, _ = six.chunk(6, 1)
    m1 = dict(norm="layer", scale=scale1, shift=shift1, rows_per_sample=T)
    _, o1 = B.segquant_block_norm(R, **m1)
    fc1.calibrate(o1)
    _, y1 = fc1.forward_block(R, **m1)
    codes = B.segquant_block_norm_quantize(R, fc1.seg, fc1.s_pos, None, "int8", **m1)[1]
    assert torch.equal(y1, B.segquant_seglinear_gemm(codes, fc1.Wq, fc1.seg, "int8", fc1.s_pos, fc1.s_w, fc1.bias, fc1.workspace))
    a1 = torch.nn.functional.gelu(y1.float()).to(BF)
    fc2.calibrate(a1)
    y2 = fc2.forward(a1)
    m2 = dict(gate=gate1, norm="layer", scale=scale2, shift=shift2, rows_per_sample=T)
    H, o2 = B.segquant_block_norm(R, y2, **m2)
    out.calibrate(o2)
    H2, y3 = out.forward_block(R, y2, **m2)
    assert torch.equal(H, H2)

    # 64 bits: weights as their codes stand for, activations unquantized; 8-bit steps of two ranges put a few parts in a thousand
    # of a row's norm between the two (a step is at most 1/127 of the largest value)
    six64 = (c.double() / (1 + torch.exp(-c.double()))) @ mod.weights(F32).double().t() + mod.bias.double()
    assert float((six.double() - six64).abs().max()) <= 2.0 ** -8 * float(six64.abs().max()) + 1e-5
    h, o = reference(R, y2, {**m2, "eps": 1e-6})
    check_values(H, h, "H")
    W = out.Wq.view(torch.float8_e4m3fn).double() * out.s_w.double()
    want = o.v @ W.t()
    # e4m3 codes are off by at most 2^-4 of the value, or half the smallest subnormal's step
    bound = (2.0 ** -4 * o.v.abs() + 2.0 ** -10 * out.s_pos.double().clamp(min=out.s_neg.double())) @ W.abs().t()
    assert bool(torch.all((y3.double() - want).abs() <= bound * 1.01 + 2.0 ** -8 * want.abs() + 1e-5))


def test_refusals_on_the_gpu():
    R = torch.zeros((4, 64), device=DEV)
    v = torch.zeros(64, device=DEV)
    with pytest.raises(ValueError, match="channels"):
        B.segquant_block_norm(R, w=v[:32])
    with pytest.raises(TypeError, match="dtype"):
        B.segquant_block_norm(R, w=v, b=v.to(BF))
    with pytest.raises(ValueError, match="samples"):
        B.segquant_block_norm(R, scale=v[None].repeat(3, 1), rows_per_sample=1)
    with pytest.raises(ValueError, match="shape"):
        B.segquant_block_norm(R, R[:3])
    with pytest.raises(TypeError, match="Y"):
        B.segquant_block_norm(R, R.to(BF))
    with pytest.raises(ValueError, match="CUDA"):
        B.segquant_block_norm(R.cpu())
    with pytest.raises(ValueError, match="norm"):
        B.segquant_block_norm(R, norm="batch")
    with pytest.raises(B.SegquantError, match="NULL"):
        B.segquant_block_norm(R, gate=v)                      # a gate without a block output
    with pytest.raises(B.SegquantError, match="UNSUPPORTED"):
        B.segquant_block_norm(torch.zeros((2, 16400), device=DEV))
    both = torch.zeros((9, 64), device=DEV)
    with pytest.raises(B.SegquantError, match="UNSUPPORTED"):
        B.segquant_block_norm(both[:8], out=both[1:])         # a row further on: overwritten before it is read
    B.segquant_block_norm(torch.zeros((4, 128), device=DEV)[:, :64], out=torch.zeros((4, 128), device=DEV)[:, 64:])


def test_a_captured_block():
    """Modulation, norm and layer in one graph, replayed on new inputs: the bits of the eager calls.  The kernels start before the
    ones in front of them are done; each must wait for what it reads."""
    g = torch.Generator().manual_seed(6)
    samples, T, C = 2, 700, 384
    mod = W4GroupLinear(torch.randn((3 * C, C), generator=g) * 0.03, torch.randn(3 * C, generator=g) * 0.1, group=128, zero_points=True)
    fc = SegQuantLinear(torch.randn((512, C), generator=g) * 0.05, torch.randn(512, generator=g) * 0.1, [0, C], [0, 512], True)
    new = lambda: (torch.randn((samples, C), generator=g).to(DEV), torch.randn((samples * T, C), generator=g).to(DEV).to(BF),
                   torch.randn((samples * T, C), generator=g).to(DEV).to(BF))
    fc.calibrate(torch.randn((64, C), generator=g).to(BF))

    def block(c, R, X):
        shift, scale, gate = mod.forward(c, act="silu").chunk(3, 1)
        return fc.forward_block(R, X, gate=gate, scale=scale, shift=shift, rows_per_sample=T)

    static = [t.clone() for t in new()]
    block(*static)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        H, Y = block(*static)
    for _ in range(3):
        fresh = new()
        for s, f in zip(static, fresh):
            s.copy_(f)
        graph.replay()
        want = block(*fresh)
        torch.cuda.synchronize()
        assert torch.equal(H, want[0]) and torch.equal(Y, want[1])


def test_the_first_call_of_a_process_may_be_captured():
    """What is looked up once per device and kernel is looked up outside of the stream."""
    import os
    import subprocess
    import sys
    code = """
import torch
from paper_2507_14811_b200 import binding as B
X, W4 = torch.ones((1, 4096), device="cuda", dtype=torch.bfloat16), torch.full((64, 2048), 0x11, dtype=torch.uint8, device="cuda")
s, R = torch.ones((32, 64), device="cuda"), torch.ones((1200, 4096), device="cuda")
v = torch.ones(4096, device="cuda")
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    Y = B.segquant_w4_matvec(X, W4, s, 128, y_dtype=torch.float32)
    H, O = B.segquant_block_norm(R, R, gate=v, norm="rms", eps=0.0, w=v, b=v)
graph.replay()
torch.cuda.synchronize()
assert torch.all(Y == 4096) and torch.all(H == 2) and torch.all(O == 2)
"""
    subprocess.run([sys.executable, "-c", code], check=True, cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))), timeout=300)
