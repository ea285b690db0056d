"""4-bit weights with group scales and block norms: what the C ABI refuses on the host, and what the native module refuses of
tensors (no GPU: none of these calls reaches a kernel)."""
import ctypes as C

import pytest
import torch

from paper_2507_14811_b200 import binding as B
from paper_2507_14811_b200 import build as build_mod

FAKE = 0x100000   # a non-null address on a 256-byte boundary that is never dereferenced on these paths


@pytest.fixture(scope="module")
def L():
    build_mod.build()
    return B.lib()


def ptr(v):
    return C.c_void_p(v)


def quantize(L, W=FAKE, dt=0, N=64, K=256, ld=256, group=64, W4=2 * FAKE, ldw=128, s=3 * FAKE, sdt=0, lds=64, z=0, ldz=64, back=False):
    i = C.c_int64
    if back:
        return L.segquant_dequantize_w4_group(ptr(W4), i(ldw), i(N), i(K), i(group), ptr(s), C.c_int(sdt), i(lds), ptr(z), i(ldz), ptr(W),
                                              C.c_int(dt), i(ld), None)
    return L.segquant_quantize_w4_group(ptr(W), C.c_int(dt), i(N), i(K), i(ld), i(group), ptr(W4), i(ldw), ptr(s), C.c_int(sdt), i(lds),
                                        ptr(z), i(ldz), None)


@pytest.mark.parametrize("back", [False, True])
def test_group_quantizer_refusals(L, back):
    q = lambda **kw: quantize(L, back=back, **kw)
    assert q(W=0) == 1 and q(W4=0) == 1 and q(s=0) == 1
    assert q(N=0) == 2 and q(K=-1) == 2 and q(ld=255) == 2 and q(ldw=127) == 2 and q(lds=63) == 2 and q(z=FAKE, ldz=63) == 2
    assert q(W=FAKE + 4) == 4 and q(ld=258) == 4 and q(W4=FAKE + 8) == 4 and q(ldw=136) == 4 and q(s=FAKE + 4) == 4 and q(lds=66) == 4
    assert q(sdt=1, lds=68) == 4 and q(z=FAKE + 8) == 4 and q(z=FAKE, ldz=72) == 4
    assert q(dt=5) == 5 and q(sdt=5) == 5
    assert q(W4=FAKE + 1024) == 5                               # codes in the weights' memory
    for group in (0, -32, 16, 48, 96, 192, 255, 300):
        assert q(group=group) == 5, group
    if back:
        assert q(N=1 << 23, lds=1 << 23, W=1 << 44) == 2                   # more channel blocks than a grid has


def matvec(L, X=FAKE, dt=1, M=4, K=256, ldx=256, act=0, W4=2 * FAKE, ldw=128, N=64, group=64, s=3 * FAKE, sdt=0, lds=64, z=0, ldz=64,
           bias=0, Y=4 * FAKE, ydt=1, ldy=64):
    i = C.c_int64
    return L.segquant_w4_matvec(ptr(X), C.c_int(dt), i(M), i(K), i(ldx), C.c_int(act), ptr(W4), i(ldw), i(N), i(group), ptr(s), C.c_int(sdt),
                                i(lds), ptr(z), i(ldz), ptr(bias), ptr(Y), C.c_int(ydt), i(ldy), None)


def test_matvec_refusals(L):
    m = lambda **kw: matvec(L, **kw)
    assert m(X=0) == 1 and m(Y=0) == 1 and m(W4=0) == 1 and m(s=0) == 1
    assert m(M=0) == 2 and m(M=65536) == 2 and m(K=0) == 2 and m(K=131073, ldx=131073, ldw=65552) == 2 and m(ldx=255) == 2 and m(ldy=63) == 2
    assert m(N=0) == 2 and m(lds=32) == 2 and m(ldw=64) == 2
    assert m(X=FAKE + 1) == 4 and m(Y=FAKE + 1) == 4 and m(ydt=0, Y=4 * FAKE + 2) == 4 and m(bias=FAKE + 2) == 4 and m(W4=2 * FAKE + 8) == 4
    assert m(dt=2) == 5 and m(ydt=2) == 5 and m(act=3) == 5 and m(act=9) == 5 and m(group=100) == 5
    assert m(Y=FAKE) == 5 and m(Y=FAKE + 4 * 512 - 2) == 5      # Y in X's memory
    assert m(bias=4 * FAKE + 256) == 5 and m(Y=2 * FAKE + 64 * 128 - 2) == 5           # .. the bias's, the weights'


class Norm(C.Structure):
    _fields_ = [("post", C.c_int), ("post_w", C.c_void_p), ("post_b", C.c_void_p), ("alpha", C.c_float), ("gate", C.c_void_p),
                ("ld_gate", C.c_int64), ("pre", C.c_int), ("w", C.c_void_p), ("b", C.c_void_p), ("scale", C.c_void_p), ("ld_scale", C.c_int64),
                ("shift", C.c_void_p), ("ld_shift", C.c_int64), ("p_dtype", C.c_int), ("rows_per_sample", C.c_int64), ("eps", C.c_float)]


def block(L, Y=0, ldy=64, R=FAKE, ldr=64, dt=0, M=4, Cn=64, H=0, ldh=64, O=4 * FAKE, ldo=64, norm=True, codes=False, seg=None, s_pos=FAKE,
          s_neg=0, code=0, c_pos=5 * FAKE, c_neg=6 * FAKE, ldc=64, **kw):
    n = Norm(alpha=1.0, pre=2, p_dtype=0, rows_per_sample=4, eps=1e-6)
    for k, v in kw.items():
        setattr(n, k, v)
    i = C.c_int64
    ref = C.byref(n) if norm else None
    if codes:
        seg = B.SegTable([0, 64], [0, 8]) if seg is None else seg
        return L.segquant_block_norm_quantize(ptr(Y), i(ldy), ptr(R), i(ldr), C.c_int(dt), i(M), i(Cn), ref, ptr(H), i(ldh), seg.ref(),
                                              ptr(s_pos), ptr(s_neg), C.c_int(code), C.c_uint32(0), ptr(c_pos), ptr(c_neg), i(ldc), None)
    return L.segquant_block_norm(ptr(Y), i(ldy), ptr(R), i(ldr), C.c_int(dt), i(M), i(Cn), ref, ptr(H), i(ldh), ptr(O), i(ldo), None)


@pytest.mark.parametrize("codes", [False, True])
def test_block_norm_refusals(L, codes):
    b = lambda **kw: block(L, codes=codes, **kw)
    assert b(R=0) == 1 and b(norm=False) == 1
    assert b(gate=FAKE) == 1 and b(post=1) == 1 and b(post_w=FAKE) == 1       # nothing of them without Y
    assert b(M=0) == 2 and b(ldr=60) == 2 and b(Y=2 * FAKE, ldy=60) == 2 and b(rows_per_sample=0) == 2
    assert b(Y=2 * FAKE, gate=FAKE, ld_gate=32) == 2 and b(scale=FAKE, ld_scale=63) == 2 and b(shift=FAKE, ld_shift=-64) == 2
    assert b(R=FAKE + 4) == 4 and b(ldr=66) == 4 and b(w=FAKE + 2) == 4 and b(H=2 * FAKE + 8) == 4
    assert b(dt=3) == 5 and b(p_dtype=3) == 5 and b(pre=3) == 5 and b(Y=2 * FAKE, post=7) == 5 and b(eps=-1.0) == 5 and b(eps=float("nan")) == 5
    assert b(H=FAKE + 256) == 5                                               # the new stream one row off the old one
    assert b(Y=2 * FAKE, H=2 * FAKE + 256) == 5
    assert b(H=3 * FAKE, w=3 * FAKE + 256) == 5 and b(H=3 * FAKE, scale=3 * FAKE - 400, ld_scale=64, rows_per_sample=2) == 5    # a vector's place
    if codes:
        assert b(s_pos=0) == 1 and b(c_pos=0) == 1 and b(s_neg=FAKE, c_neg=0) == 1
        assert b(ldc=48) == 2 and b(seg=B.SegTable([0, 32], [0, 8])) == 3 and b(ldc=72) == 4 and b(code=4) == 5
        assert b(c_pos=FAKE) == 5 and b(s_neg=FAKE, c_neg=5 * FAKE) == 5      # codes in the input's or one another's memory
    else:
        assert b(O=0) == 1 and b(H=4 * FAKE, O=4 * FAKE) == 5 and b(O=FAKE + 16) == 5
        assert b(Cn=16400, ldr=16400, ldo=16400) == 5


@pytest.mark.parametrize("call,args,error", [
    ("w4_matvec", (), TypeError),
    ("w4_matvec", ("real", "bytes", "real", 64, None, None, 0, None, 1), ValueError),           # tensors of the host
    ("w4_matvec", ("real", "real", "real", 64, None, None, 0, None, 1), TypeError),             # weights that are no bytes
    ("w4_matvec", ("half", "bytes", "real", 64, None, None, 0, None, 1), TypeError),
    ("w4_matvec", ("vector", "bytes", "real", 64, None, None, 0, None, 1), ValueError),
    ("quantize_w4_group", ("real", 0, 0, False), ValueError),
    ("quantize_w4_group", ("real", "x", 0, False), (TypeError, ValueError)),
    ("dequantize_w4_group", ("bytes", "real", 64, 8, None, None, 0), ValueError),
    ("block_norm", ("real",), TypeError),
    ("block_norm", (None, None, 0, None, None, 1.0, None, 2, None, None, None, None, None, 1e-6, None, None, True), ValueError),
    ("block_norm", ("real", None, 0, None, None, "x", None, 2, None, None, None, None, None, 1e-6, None, None, True), (TypeError, ValueError)),
    ("block_norm", ("half", None, 0, None, None, 1.0, None, 2, None, None, None, None, None, 1e-6, None, None, True), TypeError),
])
def test_native_calls_turn_bad_arguments_into_exceptions(L, call, args, error):
    named = {"real": torch.zeros(4, 8), "bytes": torch.zeros((4, 4), dtype=torch.uint8), "half": torch.zeros(4, 8, dtype=torch.float16),
             "vector": torch.zeros(8)}
    with pytest.raises(error):
        getattr(B._calls(), call)(*[named.get(a, a) if isinstance(a, str) else a for a in args])


@pytest.mark.parametrize("call,kw", [
    (B.segquant_w4_matvec, dict(act="geglu")), (B.segquant_w4_matvec, dict(act="relu")), (B.segquant_block_norm, dict(norm="batch")),
    (B.segquant_block_norm, dict(post=3))])
def test_names_that_are_unknown(L, call, kw):
    t = torch.zeros(4, 8)
    with pytest.raises(ValueError, match="unknown"):
        call(t, t, t, 64, **kw) if call is B.segquant_w4_matvec else call(t, **kw)
