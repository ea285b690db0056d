// SiLU, GELU and gated GELU in fp32, two elements at a time.  Used by the quantize kernels (the act-to-linear prologue) and by
// the matrix-vector products with 4-bit weights (with fp32 outputs: the precise forms).
#pragma once
#include "quant_codes.cuh"

namespace sq {
namespace {

// The act-to-linear segment in front of the quantizer (Sec. 4.3.2; App. B: SiLU and GELU feed DualScale layers),
// evaluated in fp32 and rounded once to the dtype the unfused graph would have stored the activation in.
// SiLU(h) = h sigma(h) with z = exp(-|h|): sigma = 1 / (1 + z) for h >= 0, z / (1 + z) below (no overflow).  The
// exponential is the hardware base-2 approximation of h log2(e) (the rounding of that product costs |h| 2^-24
// relative, the approximation itself about one unit in the last place) and the division the hardware's fast one
// (2 units in the last place for a divisor in [1, 2]): relative error <= (|h| + 8) 2^-23, a fraction of a bf16
// half-step (2^-9) for every |h| below the underflow of the result.
// GELU(h) = h Phi(h) with E = erfc(t), t = |h| / sqrt 2: h (1 - E / 2) for h >= 0, (h / 2) E below.
// erfc(t) = exp(-t^2) g(t); the smooth factor g (the scaled complementary error function) is a degree-9
// polynomial in z = (t - 2.5) / (t + 2.5), which maps [0, 9.6] into [-1, 0.59) (coefficients from a least-squares
// fit of the relative error on Chebyshev nodes, 2^-29, by gelu_coefficients.py; beyond t = 9.6 the exponential
// has underflowed).  t^2 is
// split into its rounded value s and the rounding error e = fma(t, t, -s), and exp(-t^2) = exp(-s) (1 - e) to
// first order, so that the rounding of the square, which the exponential would amplify by t^2, does not count.
// What remains is the hardware exponential's own error (|s| 2^-24 from the product with log2 e, one unit in the
// last place from the approximation), the fast division's 2 units and a dozen roundings: relative error
// <= (3 h^2 + 48) 2^-24; in |h| <= 4 it stays below 2^-19.  The exponential keeps subnormal results (a GELU of h < -13.2
// under a small scale, or times a large gated value, is an ordinary number; 2 us of the 8192 x 2560 gated pass).
// Both are written for TWO elements: the multiplies, FMAs and adds go two per instruction (packed fp32 pairs), each of
// them rounding exactly as the scalar instruction does, which is what bounds the fused pass (the ALUs, not memory).
// (8192 x 2560 gated GELU, dual int8, 126 MB: 49.4 us one element at a time with the gate half one row ahead in registers,
// 37.9 us with pairs and the gate half in the ring; without the table, 54 M elements of GELU 93 -> 80 us.)
// GELU without branches: with a = min(|h|, 20), v = max(h, 0) - (a / 2) E in one FMA is h - (h / 2) E for h >= 0 and
// (h / 2) E below; at a = 20 the exponential has long underflowed to zero, so v is h or +0 beyond it and t^2 stays
// finite for every h.
__device__ __forceinline__ float rcp_approx(float x)
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float ex2_approx(float x)         // keeps subnormal results
{
    float r;
    asm("ex2.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ uint64_t dup2(float v) { return pack2(v, v); }
__device__ __forceinline__ uint64_t silu2(float h0, float h1)
{
    const float z0 = __expf(-fabsf(h0)), z1 = __expf(-fabsf(h1));
    float d0, d1, n0, n1;
    unpack2(add2(pack2(z0, z1), dup2(1.0f)), d0, d1);
    unpack2(mul2(pack2(h0, h1), pack2(z0, z1)), n0, n1);
    return mul2(pack2(h0 >= 0.0f ? h0 : n0, h1 >= 0.0f ? h1 : n1), pack2(rcp_approx(d0), rcp_approx(d1)));
}
// erfc(a / sqrt 2) for 0 <= a <= 20
__device__ __forceinline__ uint64_t gelu_tail2(uint64_t a)
{
    const uint64_t t = mul2(a, dup2(0.70710678118654752440f));
    float d0, d1;
    unpack2(add2(t, dup2(2.5f)), d0, d1);
    const uint64_t z = mul2(add2(t, dup2(-2.5f)), pack2(rcp_approx(d0), rcp_approx(d1)));
    uint64_t g = fma2(dup2(-5.388610225e-05f), z, dup2(2.161547454e-04f));
    g = fma2(g, z, dup2(8.157527773e-04f));
    g = fma2(g, z, dup2(-2.643950749e-03f));
    g = fma2(g, z, dup2(-3.974915482e-03f));
    g = fma2(g, z, dup2(3.992317244e-02f));
    g = fma2(g, z, dup2(-1.250353903e-01f));
    g = fma2(g, z, dup2(2.517131865e-01f));
    g = fma2(g, z, dup2(-3.717366457e-01f));
    g = fma2(g, z, dup2(2.108063698e-01f));
    const uint64_t s = mul2(t, t);
    const uint64_t neg_e = fma2(mul2(t, dup2(-1.0f)), t, s);      // t^2 = s - neg_e exactly
    float x0, x1;
    unpack2(mul2(s, dup2(-1.4426950408889634f)), x0, x1);
    const uint64_t E = mul2(pack2(ex2_approx(x0), ex2_approx(x1)), g);
    return fma2(E, neg_e, E);                                     // exp(-(s + e)) = exp(-s) (1 - e) to first order
}
__device__ __forceinline__ uint64_t gelu_from_tail2(float h0, float h1, uint64_t a, uint64_t E)
{
    return fma2(mul2(a, dup2(-0.5f)), E, pack2(fmaxf(h0, 0.0f), fmaxf(h1, 0.0f)));
}
__device__ __forceinline__ uint64_t gelu2(float h0, float h1)
{
    const uint64_t a = pack2(fminf(fabsf(h0), 20.0f), fminf(fabsf(h1), 20.0f));
    return gelu_from_tail2(h0, h1, a, gelu_tail2(a));
}
// The same two functions where fp32 outputs are made of them: the CUDA library's exponential, complementary error function (2 and 4
// units in the last place) and IEEE divisions, relative error <= 2^-20 (16 roundings of 2^-24; counted: 7 for SiLU, 11 for GELU) as long as the result is
// no subnormal.  GELU(h) = (h / 2) erfc(-h / sqrt 2): the argument is rounded to z, and what the rounding and the constant's took
// away, d, comes back by the derivative, erfc(z + d) = erfc(z) - d (2 / sqrt pi) exp(-z^2) to first order (else h^2 2^-24 of the value).
// (1 x 1152 -> 6912 with SiLU, GELU 4.6, 4.7 -> 5.0, 5.2 us; 8 x 1536 -> 9216 14.7, 15.4 -> 16.1, 17.2.)
__device__ __forceinline__ float silu_precise(float h)
{
    const float z = expf(-fabsf(h));
    return h * ((h >= 0.0f ? 1.0f : z) / (1.0f + z));
}
__device__ __forceinline__ float gelu_precise(float h)
{
    constexpr float c = 0.70710678118654752440f, c_rest = float(0.70710678118654752440 - double(c));
    const float z = -h * c, d = fmaf(-h, c, -z) - h * c_rest;
    return 0.5f * h * fmaf(-1.12837916709551257390f * __expf(-z * z), d, erfcf(z));
}
// two activations as the unfused graph would have stored them
template <typename Tin>
__device__ __forceinline__ uint64_t rounded2(uint64_t a)
{
    if (sizeof(Tin) == 2) {
        float a0, a1;
        unpack2(a, a0, a1);
        const __nv_bfloat162 r = __floats2bfloat162_rn(a0, a1);
        const uint32_t w = *reinterpret_cast<const uint32_t *>(&r);
        a = pack2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
    }
    return a;
}
// times the per-channel multipliers (one fp32 multiply)
template <typename Tin>
__device__ __forceinline__ uint64_t stored2(uint64_t a, uint64_t mult) { return mul2(rounded2<Tin>(a), mult); }
template <typename Tin>
__device__ __forceinline__ uint64_t pre2(float h0, float h1, int act, uint64_t mult)
{
    if (!act) return mul2(pack2(h0, h1), mult);
    return stored2<Tin>(act == 1 ? silu2(h0, h1) : gelu2(h0, h1), mult);
}
// Gated GELU (App. B lists GEGLU with SiLU and GELU): value * GELU(gate), the product in fp32 (one more rounding
// on top of the GELU's error: relative error <= (3 g^2 + 49) 2^-24), rounded once to the stored dtype.
template <typename Tin>
__device__ __forceinline__ uint64_t pre_gated2(float v0, float v1, float g0, float g1, uint64_t mult)
{
    return stored2<Tin>(mul2(pack2(v0, v1), gelu2(g0, g1)), mult);
}
// single elements (row tails, segment bounds inside a chunk, extreme scales)
template <typename Tin>
__device__ __forceinline__ float pre1(float h, int act, float mult)
{
    float lo, hi;
    unpack2(pre2<Tin>(h, h, act, dup2(mult)), lo, hi);
    return lo;
}
template <typename Tin>
__device__ __forceinline__ float pre_gated(float value, float gate, float mult)
{
    float lo, hi;
    unpack2(pre_gated2<Tin>(value, value, gate, gate, dup2(mult)), lo, hi);
    return lo;
}

}  // namespace
}  // namespace sq
