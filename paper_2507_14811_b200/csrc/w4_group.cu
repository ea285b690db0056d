// 4-bit weights with one scale (and zero-point) per output channel and group of inputs: quantization, dequantization and
// the matrix-vector product (few rows of activations).
//
//   w'[n][k] = (c[n][k] - z[g][n]) s[g][n],  g = k / group          y[m][n] = sum_g s[g][n] sum_{k in g} (c - z) a(x[m][k]) + b[n]
//
// The product is bound by reading the codes once: N K / 2 bytes, 12.8 T codes a second at copy bandwidth.  That leaves 148 SMs 2.8 lane
// instructions per code, and half of that on either arithmetic pipe, so codes are not turned into real numbers one by one.  A byte of
// two codes is two signed bytes 16 c after one mask each (0.4 instructions per code), which integer matrix instructions take as they are:
// mma.m16n8k32, 16 channels on its rows.  The activations become 23-bit fixed-point numbers, as three signed bytes in three of
// its 8 columns (38 bits in five, where fp32 activations make fp32 outputs); products and a group's sums are exact integers, and
// scales and zero-points come in behind a group.
// (Expanded to bf16 instead, 1.4 instructions per code, the same design took 38.3 us for 1 x 8192 -> 28672 with zero-points.)  tcgen05
// would want the expanded codes in shared memory, twice the bytes that came in, and has nothing to offer: the tensor pipe is no bound here.
#include <cuda_bf16.h>
#include <algorithm>
#include <atomic>
#include <mutex>
#include <type_traits>
#include <vector>
#include "activation.cuh"

namespace sq {
namespace {

// ---------------------------------------------------------------------------------------------- quantize / dequantize

constexpr int kTileRows = 64;        // dequantize: channels per block
constexpr int kTileK = 256;          // .. inputs per block: 8 per lane of a warp
constexpr int kRowsPerWarp = 8;      // .. 8 warps
template <typename Tin> constexpr int kWarpRows = sizeof(Tin) == 2 ? 4 : 2;      // quantize: channels per warp, 64 bytes a lane
constexpr int kQuantK = 512;         // .. inputs per block (or one longer group): 16 per lane

// elements k .. k + 7 of a row of K, zero behind its end; wide: 16 bytes at a time
template <typename Tin>
__device__ __forceinline__ void load8(const Tin *row, int64_t k, int64_t K, float (&x)[8], bool wide = true)
{
    constexpr int W = sizeof(Tin) / 2;               // 16-byte words
    if (wide && k + 8 <= K) {
        uint4 v[W];
#pragma unroll
        for (int i = 0; i < W; i++) v[i] = __ldg(reinterpret_cast<const uint4 *>(row + k) + i);
        const uint32_t *w = reinterpret_cast<const uint32_t *>(v);
#pragma unroll
        for (int i = 0; i < 8; i++)
            x[i] = sizeof(Tin) == 4 ? __uint_as_float(w[i])
                                    : __uint_as_float((i & 1) ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++) x[i] = k + i < K ? load1(row + k + i) : 0.0f;
    }
}

// a scale as stored; where that is 0 (no range, or one that underflows) it is 1
__device__ __forceinline__ float stored_scale(float s, bool bf16)
{
    const float r = bf16 ? __bfloat162float(__float2bfloat16_rn(s)) : s;
    return r == 0.0f ? 1.0f : r;
}

// 32 bytes at once; the address is a multiple of 32
__device__ __forceinline__ void load32(const void *p, uint4 &a, uint4 &b)
{
    asm("ld.global.nc.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
        : "=r"(a.x), "=r"(a.y), "=r"(a.z), "=r"(a.w), "=r"(b.x), "=r"(b.y), "=r"(b.z), "=r"(b.w) : "l"(p));
}

__device__ __forceinline__ uint32_t max_bf16x2(uint32_t a, uint32_t b)
{
    uint32_t d;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
__device__ __forceinline__ uint32_t min_bf16x2(uint32_t a, uint32_t b)
{
    uint32_t d;
    asm("min.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
// x / d, correctly rounded, for d = 7 or 15 and r = RN(1 / d): a quotient corrected by its remainder (checked on the CPU for all
// significands against the IEEE division), for x that its remainder does not underflow for
__device__ __forceinline__ float over(float x, float d, float r)
{
    const float q = x * r;
    return fmaf(fmaf(-q, d, x), r, q);
}

struct W4QuantParams {
    const void *W;
    int64_t ld;
    int N, K;
    int group, span, tiles_k;        // span: inputs per block
    int wide;                        // rows on 32-byte boundaries
    uint8_t *W4;
    int64_t ldw;
    void *s;
    int s_bf16;
    int64_t lds;
    int8_t *z;
    int64_t ldz;
    int groups;
};

// Sixteen codes of a lane -> two words.  Clip, then round (the bounds are whole numbers): the nibble is the sum's last bits,
// plus the zero-point's.  Only the upper bound of codes with zero-points needs the clip: a scale of the fast form is its extremum
// over 7 (or 15) to within 2^-9, so that no symmetric quotient rounds beyond 7, and -8 - round(lo / s) + round(lo / s) is the lower bound
// itself; the upper one is passed by 1 where both ends round up.
template <bool ZP>
__device__ __forceinline__ uint2 codes16(const float (&x)[16], const SegConst &c, float hi, uint32_t z4)
{
    const uint64_t r2 = pack2(c.r, c.r), ns2 = pack2(-c.s, -c.s), magic2 = pack2(kRoundMagic, kRoundMagic);
    uint32_t v[16], w[2];
#pragma unroll
    for (int i = 0; i < 16; i += 2) {
        float q0, q1;
        unpack2(div2_rn_fast(pack2(x[i], x[i + 1]), ns2, r2), q0, q1);     // (see SegConst: the codes of the IEEE quotients)
        if (ZP) q0 = fminf(q0, hi), q1 = fminf(q1, hi);
        unpack2u(add2(pack2(q0, q1), magic2), v[i], v[i + 1]);
    }
#pragma unroll
    for (int i = 0; i < 2; i++) {                                          // last bytes of the even and of the odd codes
        const uint32_t *u = v + 8 * i;
        uint32_t even = __byte_perm(__byte_perm(u[0], u[2], 0x0040), __byte_perm(u[4], u[6], 0x0040), 0x5410);
        uint32_t odd = __byte_perm(__byte_perm(u[1], u[3], 0x0040), __byte_perm(u[5], u[7], 0x0040), 0x5410);
        if (ZP) even = (even & 0x0F0F0F0Fu) + z4, odd = (odd & 0x0F0F0F0Fu) + z4;
        w[i] = (even & 0x0F0F0F0Fu) | (odd << 4 & 0xF0F0F0F0u);
    }
    return make_uint2(w[0], w[1]);
}
// .. where the scale is outside the fast form
template <bool ZP>
__device__ __noinline__ uint2 codes16_slow(const float *x, float s, float lo, float hi, uint32_t z4)
{
    uint32_t w[2] = {0, 0};
    for (int i = 0; i < 16; i++) {
        const uint32_t v = __float_as_uint(fminf(fmaxf(__fdiv_rn(x[i], s), lo), hi) + kRoundMagic) + (ZP ? z4 : 0u);
        w[i >> 3] |= (v & 15u) << (4 * (i & 7));
    }
    return make_uint2(w[0], w[1]);
}

// Bound by reading W.  A warp takes 512 consecutive inputs of a channel, 16 per lane, and four channels (fp32: two), whose loads all go
// out first; LANES lanes of a group agree on its extrema by shuffles, and the codes leave as 256 consecutive bytes.  Groups longer
// than 512 (LONG) read the channel's group twice, the second time from cache.  Scales and zero-points are [groups][N]; a block
// gathers those of its channels in shared memory, so that they leave as runs.  (Eight inputs per lane and loops for any group: 43
// instructions per weight, 128 us for 18432 x 4608 bf16; 16 inputs and fixed lanes, 16 instructions, 64 us, with two channels per warp
// as with four and at 24 as at 32 warps, as long as a row's branches kept the rows one behind the other; without them 41 us.)
template <typename Tin, bool ZP, int LANES, bool LONG>
__global__ void __launch_bounds__(256) quantize_w4_group_kernel(const __grid_constant__ W4QuantParams prm)
{
    constexpr int G = 32 / LANES;                        // groups of a warp's inputs
    constexpr int ROWS = kWarpRows<Tin>, BLOCK_ROWS = 8 * ROWS, V = int(sizeof(Tin));        // V: 16-byte words of 16 inputs
    __shared__ float sm_s[G][BLOCK_ROWS + 1];            // (a pitch that keeps the groups of a channel on different banks)
    __shared__ int8_t sm_z[G][BLOCK_ROWS + 4];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int tile_n = int(blockIdx.x) / prm.tiles_k, kb = (int(blockIdx.x) - tile_n * prm.tiles_k) * prm.span;
    const int n0 = tile_n * BLOCK_ROWS + warp * ROWS, k0 = kb + lane * 16;
    const int k_end = LONG ? min(prm.K, kb + prm.span) : prm.K;
    const Tin *W = static_cast<const Tin *>(prm.W) + int64_t(n0) * prm.ld;
    const bool inside = n0 + ROWS <= prm.N && kb + kQuantK <= k_end;     // nothing to look at
    uint4 raw[ROWS][V];
    if (inside) {
#pragma unroll
        for (int r = 0; r < ROWS; r++)
#pragma unroll
            for (int i = 0; i < V; i += 2) {
                const uint4 *p = reinterpret_cast<const uint4 *>(W + r * prm.ld + k0) + i;
                if (prm.wide) load32(p, raw[r][i], raw[r][i + 1]);
                else raw[r][i] = __ldg(p), raw[r][i + 1] = __ldg(p + 1);
            }
    }
    // The usual case in one go, without a branch for the rows to wait at: ranges and scales inside the fast form.
    bool done = false;
    if (!LONG && inside) {
        auto expand = [&](int r, float (&x)[16]) {
            const uint32_t *w = reinterpret_cast<const uint32_t *>(raw[r]);
#pragma unroll
            for (int i = 0; i < 16; i++)
                x[i] = sizeof(Tin) == 4 ? __uint_as_float(w[i]) : __uint_as_float((i & 1) ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
        };
        float hi[ROWS], neg[ROWS], s[ROWS], z[ROWS];
        SegConst c[ROWS];
#pragma unroll
        for (int r = 0; r < ROWS; r++) {
            if (sizeof(Tin) == 2) {                      // two at a time
                const uint32_t *w = reinterpret_cast<const uint32_t *>(raw[r]);
                uint32_t top = w[0], low = w[0];
#pragma unroll
                for (int i = 1; i < 8; i++) top = max_bf16x2(top, w[i]), low = min_bf16x2(low, w[i]);
                hi[r] = fmaxf(__uint_as_float(top << 16), __uint_as_float(top & 0xFFFF0000u));
                neg[r] = -fminf(__uint_as_float(low << 16), __uint_as_float(low & 0xFFFF0000u));
            } else {
                float x[16];
                expand(r, x);
                hi[r] = x[0], neg[r] = -x[0];
#pragma unroll
                for (int i = 1; i < 16; i++) hi[r] = fmaxf(hi[r], x[i]), neg[r] = fmaxf(neg[r], -x[i]);
            }
            if (!ZP) hi[r] = fmaxf(hi[r], neg[r]);
        }
#pragma unroll
        for (int o = 1; o < LANES; o <<= 1) {
#pragma unroll
            for (int r = 0; r < ROWS; r++) {
                hi[r] = fmaxf(hi[r], __shfl_xor_sync(0xFFFFFFFFu, hi[r], o));
                if (ZP) neg[r] = fmaxf(neg[r], __shfl_xor_sync(0xFFFFFFFFu, neg[r], o));
            }
        }
        bool easy = true;
#pragma unroll
        for (int r = 0; r < ROWS; r++) {
            hi[r] = fmaxf(hi[r], 0.0f), neg[r] = fmaxf(neg[r], 0.0f);
            const float range = ZP ? __fadd_rn(hi[r], neg[r]) : hi[r];
            s[r] = stored_scale(ZP ? over(range, 15.0f, 1.0f / 15.0f) : over(range, 7.0f, 1.0f / 7.0f), prm.s_bf16);
            c[r] = seg_const(s[r]);
            easy = easy && range >= 1e-25f && c[r].fast;
            z[r] = 0.0f;                                 // (-8 - round(lo / s): rounding is symmetric; the quotient as the codes')
            if (ZP) {
                const float q = neg[r] * c[r].r;
                z[r] = (fmaf(fmaf(-q, s[r], neg[r]), c[r].r, q) + kRoundMagic - kRoundMagic) - 8.0f;
            }
        }
        done = __all_sync(0xFFFFFFFFu, easy);
        if (done) {
            uint8_t *out = prm.W4 + n0 * prm.ldw + k0 / 2;
#pragma unroll
            for (int r = 0; r < ROWS; r++) {
                float x[16];
                expand(r, x);
                const uint32_t z4 = (__float_as_uint(z[r] + kRoundMagic) & 15u) * 0x01010101u;
                *reinterpret_cast<uint2 *>(out + r * prm.ldw) = codes16<ZP>(x, c[r], 7.0f - z[r], z4);
            }
            if (lane % LANES == 0) {
#pragma unroll
                for (int r = 0; r < ROWS; r++) {
                    sm_s[lane / LANES][warp * ROWS + r] = s[r];
                    if (ZP) sm_z[lane / LANES][warp * ROWS + r] = int8_t(int(__float_as_uint(z[r] + kRoundMagic)) - kMagicBits);
                }
            }
        }
    }
    auto load16 = [&](int r, int k, float (&x)[16]) {
        float a[8], b[8];
        if (n0 + r < prm.N) {
            load8(W + r * prm.ld, k, k_end, a);
            load8(W + r * prm.ld, k + 8, k_end, b);
        } else {
#pragma unroll
            for (int i = 0; i < 8; i++) a[i] = b[i] = 0.0f;
        }
#pragma unroll
        for (int i = 0; i < 8; i++) x[i] = a[i], x[i + 8] = b[i];
    };
#pragma unroll 1
    for (int r = 0; r < ROWS && !done; r++) {
        float x[16];
        load16(r, k0, x);
        float hi = 0.0f, neg = 0.0f;                     // extrema: of both polarities (hi, -lo), or of the magnitude
        auto extrema = [&](const float (&v)[16]) {
#pragma unroll
            for (int i = 0; i < 16; i++) {
                hi = fmaxf(hi, ZP ? v[i] : fabsf(v[i]));
                if (ZP) neg = fmaxf(neg, -v[i]);
            }
        };
        extrema(x);
        if (LONG) {
            for (int k = k0 + kQuantK; k < k_end; k += kQuantK) {
                float more[16];
                load16(r, k, more);
                extrema(more);
            }
        }
#pragma unroll
        for (int o = 1; o < LANES; o <<= 1) {
            hi = fmaxf(hi, __shfl_xor_sync(0xFFFFFFFFu, hi, o));
            if (ZP) neg = fmaxf(neg, __shfl_xor_sync(0xFFFFFFFFu, neg, o));
        }
        const float s = stored_scale(ZP ? __fdiv_rn(__fadd_rn(hi, neg), 15.0f) : __fdiv_rn(hi, 7.0f), prm.s_bf16);
        const float z = ZP ? rintf(__fdiv_rn(neg, s)) - 8.0f : 0.0f;      // (-8 - round(lo / s): rounding is symmetric)
        const SegConst c = seg_const(s);
        const float lo = (ZP ? -8.0f : -7.0f) - z, top = 7.0f - z;
        const uint32_t z4 = (uint32_t(int(z)) & 15u) * 0x01010101u;
        for (int k = k0; k < k_end; k += kQuantK) {
            if (LONG && k != k0) load16(r, k, x);
            const uint2 w = c.fast ? codes16<ZP>(x, c, top, z4) : codes16_slow<ZP>(x, s, lo, top, z4);
            if (n0 + r < prm.N) {
                uint8_t *out = prm.W4 + (n0 + r) * prm.ldw + k / 2;
                if (k + 16 <= k_end) {
                    *reinterpret_cast<uint2 *>(out) = w;
                } else {                                 // the row's last codes, a zero nibble behind an odd one
                    const uint64_t both = uint64_t(w.y) << 32 | w.x, kept = both & (~uint64_t(0) >> (4 * (k + 16 - k_end)));
                    for (int j = 0; 2 * j < k_end - k; j++) out[j] = uint8_t(kept >> (8 * j));
                }
            }
            if (!LONG) break;
        }
        if (lane % LANES == 0) {
            sm_s[lane / LANES][warp * ROWS + r] = s;
            if (ZP) sm_z[lane / LANES][warp * ROWS + r] = int8_t(z);
        }
    }
    __syncthreads();
    for (int j = threadIdx.x; j < G * BLOCK_ROWS; j += 256) {
        const int gi = j / BLOCK_ROWS, i = j % BLOCK_ROWS, g = kb / prm.group + gi, n = tile_n * BLOCK_ROWS + i;
        if (g < prm.groups && n < prm.N) {
            if (prm.s_bf16) static_cast<__nv_bfloat16 *>(prm.s)[g * prm.lds + n] = __float2bfloat16_rn(sm_s[gi][i]);
            else static_cast<float *>(prm.s)[g * prm.lds + n] = sm_s[gi][i];
            if (ZP) prm.z[g * prm.ldz + n] = sm_z[gi][i];
        }
    }
}

struct W4DequantParams {
    const uint8_t *W4;
    int64_t ldw, N, K;
    int group;
    const void *s;
    int s_bf16;
    int64_t lds;
    const int8_t *z;
    int64_t ldz;
    void *W;
    int64_t ld;
    int64_t groups;
};

// Eight codes -> eight values in order.  A nibble with its top bit flipped is c + 8, and the bits 0x4300 | (c + 8) are the bf16 number
// 136 + c: codes i and i + 4 of a word in one shift and one mask.  neg_off: -(136 + z), twice; the product is the one fp32 product.
__device__ __forceinline__ void values8(uint32_t word, uint64_t neg_off, uint64_t s2, float (&v)[8])
{
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const uint32_t pair = (word >> (4 * i) & 0x000F000Fu) ^ 0x43084308u;
        unpack2(mul2(add2(pack2(__uint_as_float(pair << 16), __uint_as_float(pair & 0xFFFF0000u)), neg_off), s2), v[i], v[i + 4]);
    }
}
template <typename Tout>
__device__ __forceinline__ void store8(Tout *out, const float (&v)[8])
{
    if (sizeof(Tout) == 4) {
        reinterpret_cast<float4 *>(out)[0] = make_float4(v[0], v[1], v[2], v[3]);
        reinterpret_cast<float4 *>(out)[1] = make_float4(v[4], v[5], v[6], v[7]);
    } else {
        __nv_bfloat162 b[4];
#pragma unroll
        for (int i = 0; i < 4; i++) b[i] = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        *reinterpret_cast<uint4 *>(out) = *reinterpret_cast<const uint4 *>(b);
    }
}

// The reverse, bound by writing W: a lane turns four bytes into eight values, for eight channels whose words it has loaded first; the block's
// scales and zero-points come through shared memory.  (One code at a time and bounds for every word: 14.5 instructions per weight, 49 us for
// 18432 x 4608 in groups of 32 with zero-points, 76 % of the issue slots; now 47, and 36 instead of 42 in groups of 128.)
template <typename Tout>
__global__ void __launch_bounds__(256) dequantize_w4_group_kernel(const __grid_constant__ W4DequantParams prm)
{
    __shared__ float sm_s[8][kTileRows + 1];             // (a pitch that keeps the groups of a channel on different banks)
    __shared__ float sm_z[8][kTileRows + 1];             // -(136 + z)
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t n0 = int64_t(blockIdx.y) * kTileRows, k0 = int64_t(blockIdx.x) * kTileK, g0 = k0 / prm.group;
    const int in_block = prm.group >= kTileK ? 1 : kTileK / prm.group;
    const bool inside = n0 + kTileRows <= prm.N && k0 + kTileK <= prm.K;
    uint32_t word[kRowsPerWarp];
    const int64_t k = k0 + lane * 8, n = n0 + warp * kRowsPerWarp;
    const uint8_t *p = prm.W4 + n * prm.ldw + k / 2;
    if (inside) {
#pragma unroll
        for (int r = 0; r < kRowsPerWarp; r++) word[r] = __ldg(reinterpret_cast<const uint32_t *>(p + r * prm.ldw));
    } else {
#pragma unroll
        for (int r = 0; r < kRowsPerWarp; r++) {
            word[r] = 0;
            if (n + r < prm.N && k < prm.K) {
                if (k + 8 <= prm.K) word[r] = __ldg(reinterpret_cast<const uint32_t *>(p + r * prm.ldw));
                else for (int j = 0; k + 2 * j < prm.K; j++) word[r] |= uint32_t(__ldg(p + r * prm.ldw + j)) << (8 * j);
            }
        }
    }
    for (int i = threadIdx.x; i < in_block * kTileRows; i += blockDim.x) {
        const int64_t g = g0 + i / kTileRows, m = n0 + i % kTileRows;
        float s = 0.0f, z = 0.0f;
        if (g < prm.groups && m < prm.N) {
            s = prm.s_bf16 ? load1(static_cast<const __nv_bfloat16 *>(prm.s) + g * prm.lds + m)
                           : __ldg(static_cast<const float *>(prm.s) + g * prm.lds + m);
            if (prm.z) z = float(prm.z[g * prm.ldz + m]);
        }
        sm_s[i / kTileRows][i % kTileRows] = s;
        sm_z[i / kTileRows][i % kTileRows] = -136.0f - z;
    }
    __syncthreads();
    if (k >= prm.K) return;
    const int gi = prm.group >= kTileK ? 0 : lane * 8 / prm.group;
    Tout *out = static_cast<Tout *>(prm.W) + n * prm.ld + k;
#pragma unroll
    for (int r = 0; r < kRowsPerWarp; r++) {
        const float s = sm_s[gi][warp * kRowsPerWarp + r], z = sm_z[gi][warp * kRowsPerWarp + r];
        float v[8];
        values8(word[r], pack2(z, z), pack2(s, s), v);
        if (inside) {
            store8(out + r * prm.ld, v);
        } else if (n + r < prm.N) {
            if (k + 8 <= prm.K) {
                store8(out + r * prm.ld, v);
            } else {
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    if (k + i >= prm.K) break;
                    if (sizeof(Tout) == 4) reinterpret_cast<float *>(out + r * prm.ld)[i] = v[i];
                    else reinterpret_cast<__nv_bfloat16 *>(out + r * prm.ld)[i] = __float2bfloat16_rn(v[i]);
                }
            }
        }
    }
}

// ---------------------------------------------------------------------------------------------- matrix-vector product

constexpr int kWarps = 16;
constexpr int kTileN = 16;           // channels of a tile: the MMA's rows
constexpr int kUnitK = 256;          // codes per channel and ring stage: 128 bytes
constexpr int kUnitBytes = kTileN * kUnitK / 2;
constexpr int kMaxStages = 4;        // of a warp's ring; 2 or 3 where the activations leave no room for more
constexpr int kRedPitch = 20;        // floats per column of a tile's sums (16 used; 20 keeps the stores off one bank)
constexpr int kMaxCols = 32;         // columns of a pass: 10 rows of three bytes each, 6 of five
constexpr int kAhead = 3;            // loads of eight activations that a thread has in flight
constexpr int kMaxBlock = 128;       // inputs of an exact sum: a group, or this many of a longer one

struct MatvecParams {
    const void *X;
    int64_t ldx;
    int M, rows;                     // rows of X, rows of one pass (grid.y)
    uint32_t per_row;                // 2^32 / rows, rounded up
    int K;
    int x_f32, x_wide, act;
    const uint8_t *W4;
    int64_t ldw;
    int N, row_bytes;
    int groups, unit_groups;         // in all; of a unit (at least 1)
    int units_group;                 // units of a group (at least 1)
    const uint8_t *s;
    int s_bytes;                     // 4 or 2
    int64_t lds;                     // bytes
    const int8_t *z;
    int64_t ldz;
    const float *bias;
    void *Y;
    int y_f32;
    int64_t ldy;
    int cl;                          // CTAs of a cluster, which share K
    int units, units_cta;            // of K, of a CTA
    int tiles, clusters;
    int tiles_round;                 // tiles whose sums fit in shared memory
    int parts;                       // bytes of an activation, 3 or 5
    int cols, cols8;                 // columns in use, parts * rows; rounded up to whole MMAs
    int stages;
    uint32_t stage_bytes, z_off, x_off, f_off, xs_off, red_off, head_off, out_off;
};

__device__ __forceinline__ uint32_t smem_addr(const void *p) { return uint32_t(__cvta_generic_to_shared(p)); }
// 16 bytes from global to shared memory, of which `bytes` are read and the others zero
__device__ __forceinline__ void copy16(uint32_t dst, const void *src, int bytes)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ void load_matrices(uint32_t addr, uint32_t (&r)[4])
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
// d = a b + c with signed bytes
__device__ __forceinline__ void mma(int (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1, const int (&c)[4])
{
    asm("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %11, %12, %13};"
        : "=r"(d[0]), "=r"(d[1]), "=r"(d[2]), "=r"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "r"(c[0]), "r"(c[1]), "r"(c[2]), "r"(c[3]));
}
__device__ __forceinline__ uint32_t shared_u32(uint32_t at)
{
    uint32_t v;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(at));
    return v;
}
__device__ __forceinline__ int shared_s8(uint32_t at)
{
    int v;
    asm volatile("ld.shared.s8 %0, [%1];" : "=r"(v) : "r"(at));
    return v;
}
__device__ __forceinline__ uint4 shared_v4(uint32_t at)
{
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at));
    return v;
}
__device__ __forceinline__ uint2 shared_v2(uint32_t at)
{
    uint2 v;
    asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(at));
    return v;
}
// bytes 0, 1 and 2 of four words
__device__ __forceinline__ void bytes_of(uint32_t a, uint32_t b, uint32_t c, uint32_t d, uint32_t (&p)[3])
{
    const uint32_t ab = __byte_perm(a, b, 0x5140), cd = __byte_perm(c, d, 0x5140);
    p[0] = __byte_perm(ab, cd, 0x5410);
    p[1] = __byte_perm(ab, cd, 0x7632);
    p[2] = __byte_perm(__byte_perm(a, b, 0x0062), __byte_perm(c, d, 0x0062), 0x5410);
}
// max(|a|, |b|), a NaN where either is one
__device__ __forceinline__ float largest(float a, float b)
{
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(fabsf(a)), "f"(fabsf(b)));
    return d;
}
__device__ __forceinline__ float largest8(const float (&x)[8])
{
    return largest(largest(largest(x[0], x[1]), largest(x[2], x[3])), largest(largest(x[4], x[5]), largest(x[6], x[7])));
}
__device__ __forceinline__ void cluster_barrier()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// Output o of a CTA's tiles is channel o % 16 of row o / 16 % rows; its tile, by a product (x / rows is the upper half of x times
// per_row for x < 2^28 and rows > 1)
__device__ __forceinline__ int tile_of_output(const MatvecParams &prm, int o)
{
    return prm.rows == 1 ? o >> 4 : int(__umulhi(uint32_t(o >> 4), prm.per_row));
}
// log2 of the lanes that put an output together: a tile lies in about 16 / tiles runs, and all threads together go through the
// outputs once
__device__ __forceinline__ int lanes_of_output(int tiles, int outs)
{
    int share = tiles >= 16 ? 0 : tiles >= 8 ? 1 : tiles >= 4 ? 2 : tiles >= 2 ? 3 : 4;
    while (share > 0 && outs << share > kWarps * 32) share--;
    return share;
}

// A CTA of 16 warps holds its share of the activations in shared memory as MMA operands.  Its work is a list of units, 16 channels x 256 codes,
// tile after tile of 16 channels, and every warp takes an equal run of that list: whole tiles, and the end of one and the start of
// another.  So no warp waits for another until all of them are done, whatever the number of channels and inputs (one tile at a time, K shared by
// the warps and their sums joined behind each, took half as long again).  A tile's sum is then put together from the runs that it lies
// in, in their order.  K may also be shared by the `cl` CTAs of a cluster, which write their sums to one another.
// Every warp streams its units through a ring of its own (asynchronous copies; nothing but the warp itself waits for them).
//
// Codes of one channel that share 16 bytes are handed to the four lanes of a row by ldmatrix, eight each: (w << 4) & 0xF0F0F0F0 are the
// bytes 16 c of codes 0, 2, 4, 6 and w & 0xF0F0F0F0 those of 1, 3, 5, 7, and the activations are laid out in that order, too; any order
// of K will do as long as both operands have it.
//
// Fixed point: with 2^E <= max|x| < 2^(E+1) over the 256 inputs of a unit, q = round(x 2^(21 - E)), |q| <= 2^22, off by at most
// 2^-22 of that maximum (a bf16 x down to 2^-14 of it is exact, and behind a bf16 rounding of the outputs the others are good enough);
// the lower three bytes of (q + 0x8080) ^ 0x8080 are signed q0, q1, q2 with q = q0 + 256 q1 + 65536 q2.
// fp32 outputs of fp32 activations, or of an activation function's values, are to have the digits of fp32 products: there
// round(2^15 (x 2^(21 - E) - q)) makes two more bytes, off by at most 2^-37 of the maximum (an fp32 x down to 2^-13 of it is exact).
// The rule looks at types alone.  (Three bytes there: an input in 256 a thousand times the others, its weights a thousand times
// smaller: 4.9e-5 of the output instead of 2e-7.  Five cost a row nothing, 25.9 -> 26.0 us for 1 x 8192 -> 28672, two rows 26.7 -> 33.0;
// 8 x 4608 -> 18432 19.3 -> 41.3, because more than six take a second pass.)
// A block, a group or 128 inputs of a longer one, has a sum of 16 c q_i within 2^21, so that it becomes a float by starting at the
// bits of 1.5 * 2^23, the MMA's addend, and subtracting that number.  One FMA takes off the zero-point times the block's sum of 16 q_i
// (whole numbers of fp32, as are their product and the difference for zero-points in [-8, 7]; beyond, one rounding.  As the MMA's addend
// they would leave the range of the start there).  One FMA takes it with its scale to the unit's sum, and one the unit's sum with
// 2^(E - 25) 256^i to the tile's, two columns per instruction.  A unit with an infinity or a NaN has the factor NaN.  (A range per group
// instead of one per unit: 26.3 us against 25.8 for 1 x 8192 -> 28672, 9.7 against 8.8 for 8 x 1536 -> 9216 with SiLU.)
// GB: blocks of a unit (2, 4, 8).  PARTS: bytes of an activation (3, 5).
template <int NT, int GB, bool ZP, int PARTS>
__global__ void __launch_bounds__(kWarps * 32, 1) w4_matvec_kernel(const __grid_constant__ MatvecParams prm)
{
    extern __shared__ __align__(128) uint8_t smem[];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    const int cl = prm.cl, rank = cl > 1 ? int(blockIdx.x) % cl : 0, cluster = int(blockIdx.x) / cl;
    const int m0 = int(blockIdx.y) * prm.rows, rows = min(prm.rows, prm.M - m0);
    const uint32_t sm0 = smem_addr(smem), ring = sm0 + warp * prm.stages * prm.stage_bytes;
    const int u_first = rank * prm.units_cta, U = max(0, min(prm.units - u_first, prm.units_cta));   // this CTA's units of a tile
    const int t_first = int(int64_t(cluster) * prm.tiles / prm.clusters), t_last = int((int64_t(cluster) + 1) * prm.tiles / prm.clusters);

    const int wr = lane >> 3, wc = lane & 7;             // this lane's 16-byte pieces of a unit: rows wr, wr + 4, ..
    const uint32_t d0 = wr * 128 + ((wc ^ wr) << 4), d1 = (wr + 4) * 128 + ((wc ^ wr ^ 4) << 4);
    const int64_t row4 = 4 * prm.ldw;
    const int pieces = prm.s_bytes, s_group = lane / pieces, s_n = lane % pieces * (16 / prm.s_bytes);   // 16-byte pieces of 16 channels' scales
    const bool s_lane = lane < prm.unit_groups * pieces, z_lane = ZP && lane < prm.unit_groups;
    const uint32_t lm_row = (lane & 15) * 128, lm_seg = lane >> 4, lm_x = lane & 7;      // ldmatrix: rows 0-15 of two pieces
    uint32_t lm[4];
#pragma unroll
    for (int i = 0; i < 4; i++) lm[i] = lm_row + (((2 * i + lm_seg) ^ lm_x) << 4);
    uint32_t xb[NT];                                     // this lane's activations: column g (+ 8 per MMA), codes 8 t ..
#pragma unroll
    for (int nt = 0; nt < NT; nt++) xb[nt] = sm0 + prm.x_off + min(g + 8 * nt, prm.cols - 1) * 64 + t * 16;
    const uint32_t s_shift = prm.s_bytes == 2 && g % 2 == 0 ? 16 : 0, s_mask = prm.s_bytes == 2 ? 0xFFFF0000u : 0xFFFFFFFFu;
    const uint32_t x_pair = prm.cols * 64;               // 64 codes of all columns
    const uint32_t s_step = prm.unit_groups == GB ? 16 * prm.s_bytes : 0, z_step = prm.unit_groups == GB ? 16 : 0;

    asm volatile("griddepcontrol.launch_dependents;\n\tgriddepcontrol.wait;" ::: "memory");     // nothing is read before the kernel in front is done

    if (cl > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    // raw activations: what a thread converts, kAhead times eight inputs in flight.  Eight e of row m: inputs u_first kUnitK + 8 e ..
    const int eights = U * (kUnitK / 8), all_eights = eights * rows;
    struct Place {
        int i, m, e;
        __device__ void next(int eights)
        {
            i += kWarps * 32;
            for (e += kWarps * 32; e >= eights; e -= eights) m++;
        }
    };
    Place ahead{tid, 0, tid}, here;
    if (tid < all_eights) ahead.m = tid / eights, ahead.e = tid - ahead.m * eights;
    here = ahead;
    const int k_first = u_first * kUnitK;
    uint4 raw[kAhead][2];
    auto is_wide = [&](const Place &p) { return prm.x_wide && k_first + p.e * 8 + 8 <= prm.K; };
    auto fetch = [&]() {
#pragma unroll
        for (int b = 0; b < kAhead; b++) {
            if (ahead.i < all_eights) {
                if (is_wide(ahead)) {
                    const int64_t at = (m0 + ahead.m) * prm.ldx + k_first + ahead.e * 8;
                    const uint4 *p = prm.x_f32 ? reinterpret_cast<const uint4 *>(static_cast<const float *>(prm.X) + at)
                                               : reinterpret_cast<const uint4 *>(static_cast<const __nv_bfloat16 *>(prm.X) + at);
                    raw[b][0] = __ldg(p);
                    if (prm.x_f32) raw[b][1] = __ldg(p + 1);
                }
                ahead.next(eights);
            }
        }
    };
    fetch();
    // the bias of this thread's first output, as far as that can be told before the tiles are split
    float bias0 = 0.0f;
    if (prm.bias) {
        const int tiles = min(prm.tiles_round, t_last - t_first);
        const int o = cl > 1 ? tid * cl + rank : tid >> lanes_of_output(tiles, tiles * kTileN * prm.rows);
        const int n = (t_first + tile_of_output(prm, o)) * kTileN + (o & 15);
        if (n < prm.N) bias0 = __ldg(prm.bias + n);
    }

    for (int t0 = t_first; t0 < t_last; t0 += prm.tiles_round) {
        const int nt_round = min(prm.tiles_round, t_last - t0);
        // this warp's run of the list
        const int total = nt_round * U, begin = int(int64_t(warp) * total / kWarps), end = int((int64_t(warp) + 1) * total / kWarps);

        // ---- the ring: copies of unit (pt, pu), one stage after the other
        int left = end - begin, pt = 0, pu = 0;
        if (left > 0) pt = begin / U, pu = begin - pt * U;
        const uint8_t *src = nullptr, *s_src = nullptr, *z_src = nullptr;
        int n0 = 0;
        auto new_tile = [&]() {
            n0 = (t0 + pt) * kTileN;
            src = prm.W4 + int64_t(n0 + wr) * prm.ldw + wc * 16;
            s_src = prm.s + int64_t(n0 + s_n) * prm.s_bytes + s_group * prm.lds;
            z_src = reinterpret_cast<const uint8_t *>(prm.z) + n0 + lane * prm.ldz;
        };
        if (left > 0) new_tile();
        auto issue = [&](int slot) {
            if (left > 0) {
                const uint32_t dst = ring + slot * prm.stage_bytes;
                const int unit = u_first + pu, off = unit * (kUnitK / 2);
                const int g0 = prm.units_group > 1 ? unit / prm.units_group : unit * prm.unit_groups;
                const uint8_t *p = src + off;
                if (n0 + kTileN <= prm.N && off + kUnitK / 2 <= prm.row_bytes) {
                    copy16(dst + d0, p, 16);
                    copy16(dst + d1, p + row4, 16);
                    copy16(dst + d0 + 1024, p + 2 * row4, 16);
                    copy16(dst + d1 + 1024, p + 3 * row4, 16);
                    if (s_lane) copy16(dst + kUnitBytes + lane * 16, s_src + g0 * prm.lds, 16);
                    if (z_lane) copy16(dst + prm.z_off + lane * 16, z_src + g0 * prm.ldz, 16);
                } else {
                    const int bytes = max(0, min(16, prm.row_bytes - off - wc * 16));
#pragma unroll
                    for (int i = 0; i < 4; i++) {
                        const bool in = n0 + wr + 4 * i < prm.N && bytes > 0;
                        copy16(dst + (i & 1 ? d1 : d0) + (i >> 1) * 1024, in ? p + i * row4 : prm.W4, in ? bytes : 0);
                    }
                    if (s_lane) {
                        const int rest = min(prm.N - n0 - s_n, 16) * prm.s_bytes;
                        const bool in = g0 + s_group < prm.groups && rest > 0;
                        copy16(dst + kUnitBytes + lane * 16, in ? s_src + g0 * prm.lds : prm.s, in ? min(16, rest) : 0);
                    }
                    if (z_lane) {
                        const bool in = g0 + lane < prm.groups;
                        copy16(dst + prm.z_off + lane * 16, in ? z_src + g0 * prm.ldz : reinterpret_cast<const uint8_t *>(prm.z),
                               in ? min(16, prm.N - n0) : 0);
                    }
                }
                left--;
                if (++pu == U) {
                    pu = 0, pt++;
                    if (left > 0) new_tile();
                }
            }
            copies_commit();
        };
        for (int i = 0; i < prm.stages - 1; i++) issue(i);

        // ---- activations (once): fixed point, a lane takes eight inputs; per 64 inputs [column][four eights][16 bytes], two words for each
        // half of the 64; zero behind the last input, so that whatever lies there in a row of codes counts for nothing.  Whole warps go
        // through the loop: the lanes of a block settle on its range by shuffles.
        if (t0 == t_first) {
            constexpr int kBlockLanes = 32 / GB;
#pragma unroll 1
            for (int b = 0; here.i < all_eights; here.next(eights)) {                   // (a multiple of 32)
                const int m = here.m, e = here.e;
                float x[8];
                if (is_wide(here)) {
                    if (prm.x_f32) {
                        const uint32_t w[8] = {raw[0][0].x, raw[0][0].y, raw[0][0].z, raw[0][0].w, raw[0][1].x, raw[0][1].y, raw[0][1].z, raw[0][1].w};
#pragma unroll
                        for (int j = 0; j < 8; j++) x[j] = __uint_as_float(w[j]);
                    } else {
                        const uint32_t w[4] = {raw[0][0].x, raw[0][0].y, raw[0][0].z, raw[0][0].w};
#pragma unroll
                        for (int j = 0; j < 8; j++) x[j] = __uint_as_float((j & 1) ? w[j / 2] & 0xFFFF0000u : w[j / 2] << 16);
                    }
                } else if (prm.x_f32) {
                    load8(static_cast<const float *>(prm.X) + (m0 + m) * prm.ldx, k_first + e * 8, prm.K, x, false);
                } else {
                    load8(static_cast<const __nv_bfloat16 *>(prm.X) + (m0 + m) * prm.ldx, k_first + e * 8, prm.K, x, false);
                }
#pragma unroll
                for (int j = 0; j + 1 < kAhead; j++) raw[j][0] = raw[j + 1][0], raw[j][1] = raw[j + 1][1];
                if (++b == kAhead) b = 0, fetch();
                if (prm.act == SQ_ACT_SILU) {
#pragma unroll
                    for (int j = 0; j < 8; j += 2) {
                        if constexpr (PARTS == 5) x[j] = silu_precise(x[j]), x[j + 1] = silu_precise(x[j + 1]);
                        else unpack2(silu2(x[j], x[j + 1]), x[j], x[j + 1]);
                    }
                } else if (prm.act == SQ_ACT_GELU) {
                    const float in = largest8(x);
#pragma unroll
                    for (int j = 0; j < 8; j += 2) {
                        if constexpr (PARTS == 5) x[j] = gelu_precise(x[j]), x[j + 1] = gelu_precise(x[j + 1]);
                        else unpack2(gelu2(x[j], x[j + 1]), x[j], x[j + 1]);
                    }
                    if (!(in < __uint_as_float(0x7F800000u))) x[0] = in;                // (GELU may make 0 of a NaN and of -infinity)
                }
                float top = largest8(x);
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) top = largest(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
                const bool finite = top < __uint_as_float(0x7F800000u);
                // biased E; smaller ranges count as 2^-86 (five bytes) and 2^-101
                const uint32_t be = max(__float_as_uint(top) >> 23, PARTS == 5 ? 41u : 26u);
                const float up = finite ? __uint_as_float((275u - be) << 23) : 0.0f;    // 2^(21 - E); (other blocks: any bytes)
                uint8_t *dst = smem + prm.x_off + size_t(e >> 3) * x_pair + (e & 3) * 16 + (e >> 2 & 1) * 8;
                // the lower COUNT bytes of v to columns p0, p0 + 1, ..: the first two offset by 128, a third signed as it is
                auto put = [&](const uint32_t (&v)[8], int p0, auto count) {
                    constexpr int COUNT = decltype(count)::value;
                    uint32_t even[3], odd[3];
                    bytes_of(v[0], v[2], v[4], v[6], even);
                    bytes_of(v[1], v[3], v[5], v[7], odd);
                    int sum[COUNT];
#pragma unroll
                    for (int p = 0; p < COUNT; p++) {
                        const uint2 b2 = p < 2 ? make_uint2(even[p] ^ 0x80808080u, odd[p] ^ 0x80808080u) : make_uint2(even[p], odd[p]);
                        *reinterpret_cast<uint2 *>(dst + ((p0 + p) * prm.rows + m) * 64) = b2;
                        if (ZP) sum[p] = __dp4a(int(b2.x), 0x01010101, __dp4a(int(b2.y), 0x01010101, 0));
                    }
                    if (ZP) {
#pragma unroll
                        for (int d = 1; d < kBlockLanes; d <<= 1) {
#pragma unroll
                            for (int p = 0; p < COUNT; p++) sum[p] += __shfl_xor_sync(0xFFFFFFFFu, sum[p], d);
                        }
                        if (lane % kBlockLanes == 0) {
                            float *xs = reinterpret_cast<float *>(smem + prm.xs_off) + e / kBlockLanes * prm.cols8 + m;
#pragma unroll
                            for (int p = 0; p < COUNT; p++) xs[(p0 + p) * prm.rows] = float(16 * sum[p]);
                        }
                    }
                };
                constexpr uint32_t offset = 0x4B400000u - 0x8080u;
                uint32_t v[8];
                if constexpr (PARTS == 5) {
#pragma unroll
                    for (int j = 0; j < 8; j++) {
                        const float q = fmaf(x[j], up, kRoundMagic) - kRoundMagic, rest = fmaf(x[j], up, -q);      // (both exact)
                        v[j] = __float_as_uint(fmaf(rest, 32768.0f, kRoundMagic)) - offset;
                    }
                    put(v, 0, std::integral_constant<int, 2>());
                }
#pragma unroll
                for (int j = 0; j < 8; j++) v[j] = __float_as_uint(fmaf(x[j], up, kRoundMagic)) - offset;
                put(v, PARTS - 3, std::integral_constant<int, 3>());
                if (lane < PARTS) {
                    float *f = reinterpret_cast<float *>(smem + prm.f_off) + (e >> 5) * prm.cols8 + m;
                    const int exponent = int(be) - 25 + (lane < PARTS - 3 ? 8 * lane - 15 : 8 * (lane - (PARTS - 3)));
                    f[lane * prm.rows] = finite ? __uint_as_float(uint32_t(exponent) << 23) : __uint_as_float(0x7FC00000u);
                }
            }
            __syncthreads();
        }

        // ---- the run
        float *red = reinterpret_cast<float *>(smem + prm.red_off), *head = reinterpret_cast<float *>(smem + prm.head_off);
        int slot = 0, tile = 0, u = 0;
        if (end > begin) tile = begin / U, u = begin - tile * U;
        float *to = u == 0 ? red + tile * (prm.cols * kRedPitch) : head + warp * (prm.cols * kRedPitch);
        uint64_t acc[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; nt++) acc[nt][0] = acc[nt][1] = 0;
        for (int i = begin; i < end; i++) {
            if (prm.stages == 4) copies_wait<2>();
            else if (prm.stages == 3) copies_wait<1>();
            else copies_wait<0>();
            __syncwarp();
            issue(slot == 0 ? prm.stages - 1 : slot - 1);   // the stage that was used up last
            const uint32_t st = ring + slot * prm.stage_bytes, x_unit = uint32_t(u) * 4 * x_pair;
            const uint32_t f_at = sm0 + prm.f_off + (u * prm.cols8 + 2 * t) * 4, xs_at = sm0 + prm.xs_off + (u * GB * prm.cols8 + 2 * t) * 4;
            const uint32_t s_at = st + kUnitBytes + (g * prm.s_bytes & ~3), z_at = st + prm.z_off + g;
            int sum[NT][4];
            uint64_t part[NT][2];                        // two columns at a time
            // what the sums of a block start from
            auto start = [&]() {
#pragma unroll
                for (int nt = 0; nt < NT; nt++)
#pragma unroll
                    for (int j = 0; j < 4; j++) sum[nt][j] = kMagicBits;
            };
            // and what becomes of those of block b
            auto finish = [&](int b) {
                // an fp32 scale, or one half of the word that a bf16 one lies in; without a branch, which would keep the blocks apart
                const float s0 = __uint_as_float(shared_u32(s_at + b * s_step) << s_shift & s_mask);
                const float s1 = __uint_as_float(shared_u32(s_at + b * s_step + 8 * prm.s_bytes) << s_shift & s_mask);
                float z0 = 0.0f, z1 = 0.0f;              // -z
                if (ZP) {
                    z0 = kRoundMagic - __int_as_float(kMagicBits + shared_s8(z_at + b * z_step));
                    z1 = kRoundMagic - __int_as_float(kMagicBits + shared_s8(z_at + b * z_step + 8));
                }
                const uint64_t sc[2] = {pack2(s0, s0), pack2(s1, s1)}, z[2] = {pack2(z0, z0), pack2(z1, z1)};
#pragma unroll
                for (int nt = 0; nt < NT; nt++) {
                    uint2 xs = make_uint2(0u, 0u);
                    if (ZP) xs = shared_v2(xs_at + (b * prm.cols8 + nt * 8) * 4);
#pragma unroll
                    for (int j = 0; j < 2; j++) {
                        uint64_t v = add2(pack2(__int_as_float(sum[nt][2 * j]), __int_as_float(sum[nt][2 * j + 1])), pack2(-kRoundMagic, -kRoundMagic));
                        if (ZP) v = fma2(z[j], pack2(__uint_as_float(xs.x), __uint_as_float(xs.y)), v);
                        part[nt][j] = b == 0 ? mul2(sc[j], v) : fma2(sc[j], v, part[nt][j]);
                    }
                }
            };
#pragma unroll
            for (int pr = 0; pr < 4; pr++) {             // 64 codes at a time: two pieces of 32
                uint32_t w[4];
                load_matrices(st + lm[pr], w);
                constexpr uint32_t high = 0xF0F0F0F0u;
                uint4 x[NT];
#pragma unroll
                for (int nt = 0; nt < NT; nt++) x[nt] = shared_v4(xb[nt] + x_unit + pr * x_pair);
                if (GB == 8 || GB == 4 || pr % 2 == 0) start();
#pragma unroll
                for (int nt = 0; nt < NT; nt++) mma(sum[nt], w[0] << 4 & high, w[1] << 4 & high, w[0] & high, w[1] & high, x[nt].x, x[nt].y, sum[nt]);
                if (GB == 8) finish(2 * pr), start();
#pragma unroll
                for (int nt = 0; nt < NT; nt++) mma(sum[nt], w[2] << 4 & high, w[3] << 4 & high, w[2] & high, w[3] & high, x[nt].z, x[nt].w, sum[nt]);
                if (GB == 8) finish(2 * pr + 1);
                else if (GB == 4) finish(pr);
                else if (pr % 2 == 1) finish(pr / 2);
            }
#pragma unroll
            for (int nt = 0; nt < NT; nt++) {
                const uint2 f = shared_v2(f_at + nt * 32);
#pragma unroll
                for (int j = 0; j < 2; j++) acc[nt][j] = fma2(pack2(__uint_as_float(f.x), __uint_as_float(f.y)), part[nt][j], acc[nt][j]);
            }
            slot = slot + 1 == prm.stages ? 0 : slot + 1;
            if (++u == U || i + 1 == end) {              // what this run has of the tile: [column][16 channels]
#pragma unroll
                for (int nt = 0; nt < NT; nt++) {
#pragma unroll
                    for (int j = 0; j < 2; j++) {
                        const int col = nt * 8 + 2 * t;
                        float a, b;
                        unpack2(acc[nt][j], a, b);
                        if (col < prm.cols) to[col * kRedPitch + g + j * 8] = a;
                        if (col + 1 < prm.cols) to[(col + 1) * kRedPitch + g + j * 8] = b;
                        acc[nt][j] = 0;
                    }
                }
                u = 0, tile++;
                to = red + tile * (prm.cols * kRedPitch);
            }
        }
        __syncthreads();
        if (cl > 1 && t0 == t_first) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");      // every CTA is there to be written to

        // ---- outputs.  2^share lanes put one together from the runs that its tile lies in (the fewer tiles, the more runs each), every
        // lane some of them with an activation's bytes in turn, then the lanes among themselves; and the CTAs of a cluster take turns
        // with the sums over their ranks, which the others write to them (after the last barrier nobody touches another's memory).  The order is the same every time.
        const int outs = nt_round * kTileN * prm.rows, share = lanes_of_output(nt_round, outs);       // (with those of rows behind the last)
        float *own = reinterpret_cast<float *>(smem + prm.out_off);
        auto store = [&](int o, float v, bool first) {
            const int c = o & 15, tl = tile_of_output(prm, o), m = (o >> 4) - tl * prm.rows, n = (t0 + tl) * kTileN + c;
            if (n >= prm.N || m >= rows) return;
            v += !prm.bias ? 0.0f : t0 == t_first && first ? bias0 : __ldg(prm.bias + n);
            const int64_t at = (m0 + m) * prm.ldy + n;
            if (prm.y_f32) static_cast<float *>(prm.Y)[at] = v;
            else static_cast<__nv_bfloat16 *>(prm.Y)[at] = __float2bfloat16_rn(v);
        };
        for (int i = tid; i - lane < outs << share; i += kWarps * 32) {
            const int o = i >> share, j = i & ((1 << share) - 1);
            float v = 0.0f;
            if (o < outs && total > 0) {
                const int c = o & 15, tl = tile_of_output(prm, o), m = (o >> 4) - tl * prm.rows;
                // the runs that units tl U .. tl U + U - 1 lie in
                const int w_first = ((tl * U + 1) * kWarps - 1) / total, w_last = ((tl * U + U) * kWarps - 1) / total;
                for (int w = w_first + j; w <= w_last; w += 1 << share) {
                    if (w * total / kWarps == (w + 1) * total / kWarps) continue;     // a run of nothing (fewer units than warps)
                    const float *from = (w == w_first ? red + tl * (prm.cols * kRedPitch) : head + w * (prm.cols * kRedPitch)) + m * kRedPitch + c;
                    float bytes = from[0];
                    for (int p = 1; p < PARTS; p++) bytes += from[p * prm.rows * kRedPitch];
                    v += bytes;
                }
            }
            for (int d = 1; d < 1 << share; d <<= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
            if (o < outs && j == 0) {
                if (cl > 1) {                            // to the CTA whose turn it is: [output / cl][rank]
                    uint32_t at;
                    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_addr(own + (o & ~(cl - 1)) + rank)), "r"(o & (cl - 1)));
                    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(at), "f"(v) : "memory");
                } else {
                    store(o, v, i == tid);
                }
            }
        }
        if (cl > 1) {
            cluster_barrier();
            for (int o = tid * cl + rank; o < outs; o += kWarps * 32 * cl) {
                float v = 0.0f;
                for (int r = 0; r < cl; r++) v += own[o - rank + r];
                store(o, v, o == tid * cl + rank);
            }
        }
        if (t0 + prm.tiles_round < t_last) {             // the next tiles' sums take the place of these
            if (cl > 1) cluster_barrier();
            else __syncthreads();
        }
    }
}

// ---------------------------------------------------------------------------------------------- host side

template <int NT, bool ZP, int PARTS>
const void *matvec_kernel(int gb)
{
    switch (gb) {
        case 2: return reinterpret_cast<const void *>(w4_matvec_kernel<NT, 2, ZP, PARTS>);
        case 4: return reinterpret_cast<const void *>(w4_matvec_kernel<NT, 4, ZP, PARTS>);
        default: return reinterpret_cast<const void *>(w4_matvec_kernel<NT, 8, ZP, PARTS>);
    }
}
constexpr int kMaxNt = kMaxCols / 8;
template <int PARTS>
const void *matvec_kernel(int nt, int gb, bool zp)
{
    switch (nt) {
        case 1: return zp ? matvec_kernel<1, true, PARTS>(gb) : matvec_kernel<1, false, PARTS>(gb);
        case 2: return zp ? matvec_kernel<2, true, PARTS>(gb) : matvec_kernel<2, false, PARTS>(gb);
        case 3: return zp ? matvec_kernel<3, true, PARTS>(gb) : matvec_kernel<3, false, PARTS>(gb);
        default: return zp ? matvec_kernel<4, true, PARTS>(gb) : matvec_kernel<4, false, PARTS>(gb);
    }
}
const void *matvec_kernel(int nt, int gb, bool zp, int parts)
{
    return parts == 5 ? matvec_kernel<5>(nt, gb, zp) : matvec_kernel<3>(nt, gb, zp);
}

// Per device: SM count, and the clusters of 2, 4 and 8 CTAs that are resident at once (GPCs have different numbers of SMs).
struct MatvecDevice {
    int device, sms, clusters[4];
};
constexpr size_t kMaxSmem = 227 * 1024;
std::mutex g_mu;
std::vector<MatvecDevice> g_devices;

sq_status matvec_device(MatvecDevice *out)
{
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess) return SQ_ERR_CUDA;
    std::lock_guard<std::mutex> lock(g_mu);
    for (const MatvecDevice &d : g_devices)
        if (d.device == dev) { *out = d; return SQ_OK; }
    MatvecDevice d{dev, 0, {0, 0, 0, 0}};
    cudaError_t e = cudaDeviceGetAttribute(&d.sms, cudaDevAttrMultiProcessorCount, dev);
    for (int nt = 1; nt <= kMaxNt && e == cudaSuccess; nt++)
        for (int gb = 2; gb <= 8 && e == cudaSuccess; gb *= 2)
            for (int zp = 0; zp < 2 && e == cudaSuccess; zp++)
                for (int parts = 3; parts <= 5 && e == cudaSuccess; parts += 2)
                    e = cudaFuncSetAttribute(matvec_kernel(nt, gb, zp, parts), cudaFuncAttributeMaxDynamicSharedMemorySize, int(kMaxSmem));
    d.clusters[0] = d.sms;
    for (int i = 1; i <= 3 && e == cudaSuccess; i++) {
        cudaLaunchConfig_t cfg{};
        cfg.gridDim = dim3(unsigned(d.sms / (1 << i) * (1 << i)));
        cfg.blockDim = dim3(kWarps * 32);
        cfg.dynamicSmemBytes = kMaxSmem;
        cudaLaunchAttribute at{};
        at.id = cudaLaunchAttributeClusterDimension;
        at.val.clusterDim.x = 1u << i;
        at.val.clusterDim.y = at.val.clusterDim.z = 1;
        cfg.attrs = &at;
        cfg.numAttrs = 1;
        e = cudaOccupancyMaxActiveClusters(&d.clusters[i], matvec_kernel(1, 2, false, 3), &cfg);
    }
    if (e != cudaSuccess) { note_cuda_error(e); return SQ_ERR_CUDA; }
    g_devices.push_back(d);
    *out = d;
    return SQ_OK;
}

// Shared memory of a split, and whether it fits: ring, activations with their blocks' factors (and sums), sums of as many tiles as
// there is room for (at most `tiles`).
bool lay_out(MatvecParams &p, int gb, int tiles)
{
    const uint32_t s_bytes = uint32_t(p.unit_groups * kTileN * p.s_bytes), z_bytes = p.z ? uint32_t(p.unit_groups * kTileN) : 0u;
    p.z_off = kUnitBytes + s_bytes;
    p.stage_bytes = (p.z_off + z_bytes + 127u) & ~127u;
    const size_t x_bytes = size_t(p.units_cta) * 4 * p.cols * 64, f_bytes = size_t(p.units_cta) * p.cols8 * 4,
                 xs_bytes = p.z ? gb * f_bytes : 0;
    const size_t sum = size_t(p.cols) * kRedPitch * 4, one = sum + (p.cl > 1 ? size_t(p.rows) * kTileN * 4 : 0);      // of a tile
    for (p.stages = kMaxStages; p.stages >= 2; p.stages--) {
        const size_t fixed = size_t(kWarps * p.stages) * p.stage_bytes + x_bytes + f_bytes + xs_bytes + kWarps * sum;
        if (fixed + std::min(tiles, 4) * one > kMaxSmem) continue;
        p.x_off = uint32_t(kWarps * p.stages) * p.stage_bytes;
        p.f_off = uint32_t(p.x_off + x_bytes);
        p.xs_off = uint32_t(p.f_off + f_bytes);
        p.head_off = uint32_t(p.xs_off + xs_bytes);
        p.red_off = uint32_t(p.head_off + kWarps * sum);
        p.tiles_round = int(std::min<size_t>(tiles, (kMaxSmem - fixed) / one));
        p.out_off = uint32_t(p.red_off + p.tiles_round * sum);
        return true;
    }
    return false;
}
size_t smem_bytes(const MatvecParams &p) { return p.out_off + (p.cl > 1 ? size_t(p.tiles_round) * p.rows * kTileN * 4 : 0); }

}  // namespace

sq_status launch_w4_matvec(const W4MatvecArgs &a, cudaStream_t st)
{
    MatvecDevice dev;
    sq_status r = matvec_device(&dev);
    if (r != SQ_OK) return r;
    MatvecParams p{};
    p.X = a.X; p.ldx = a.ldx; p.M = int(a.M); p.K = int(a.K); p.x_f32 = a.dt == SQ_F32;
    p.x_wide = aligned16(a.X) && (a.M == 1 || a.ldx * (p.x_f32 ? 4 : 2) % 16 == 0);
    p.act = int(a.act);
    p.y_f32 = a.y_dtype == SQ_F32;
    p.W4 = static_cast<const uint8_t *>(a.W4); p.ldw = a.ldw; p.N = int(a.N); p.row_bytes = int((a.K + 1) / 2);
    const int64_t group = std::min<int64_t>(a.group, (a.K + kUnitK - 1) / kUnitK * kUnitK);
    const int gb = int(kUnitK / std::min<int64_t>(group, kMaxBlock));
    p.unit_groups = group >= kUnitK ? 1 : int(kUnitK / group);
    p.units_group = group >= kUnitK ? int(group / kUnitK) : 1;
    p.groups = int((a.K + a.group - 1) / a.group);
    p.s = static_cast<const uint8_t *>(a.s); p.s_bytes = a.s_dtype == SQ_F32 ? 4 : 2; p.lds = a.lds * p.s_bytes;
    p.z = a.z; p.ldz = a.ldz; p.bias = a.bias;
    p.Y = a.Y; p.ldy = a.ldy;
    p.units = int((a.K + kUnitK - 1) / kUnitK);
    p.tiles = int((a.N + kTileN - 1) / kTileN);

    p.parts = p.y_f32 && (p.x_f32 || a.act != SQ_ACT_NONE) ? 5 : 3;
    // Rows of a pass: as many as 32 columns take, spread evenly; fewer where the activations would not fit.
    const int most = kMaxCols / p.parts;
    int passes = (p.M + most - 1) / most;
    double best = 0;
    MatvecParams pick{};
    for (;; passes++) {
        p.rows = (p.M + passes - 1) / passes;
        p.cols = p.rows * p.parts;
        p.per_row = 0xFFFFFFFFu / uint32_t(p.rows) + 1u;
        p.cols8 = (p.cols + 7) / 8 * 8;
        for (int ci = 0; ci < 4; ci++) {
            p.cl = 1 << ci;
            if (dev.clusters[ci] < 1 || (ci && p.cl > p.units)) continue;
            p.units_cta = (p.units + p.cl - 1) / p.cl;
            p.clusters = std::min(p.tiles, dev.clusters[ci]);
            const int tiles = (p.tiles + p.clusters - 1) / p.clusters;
            if (!lay_out(p, gb, tiles)) continue;
            // Microseconds, fitted to cl = 1, 2, 4 and 8 forced on 31 shapes: a CTA's units (more columns and shorter groups take
            // more instructions, a shallow ring waits more), converting its activations, its outputs, a cluster's
            // barriers, and starting over where the tiles' sums do not fit at once.  (The fastest of the four is missed by at most
            // 3 % on 30 of them, 9 % on the other: 6 x 4608 -> 18432 fp32, 29.4 against 27.1 us.)
            const int nt = p.cols8 / 8;
            const double unit = 0.035 + 0.02 * nt + (gb == 8 ? 0.02 : gb == 4 ? 0.007 : 0.0) * nt;
            const double cost = unit * (1.0 + 0.1 * (kMaxStages - p.stages)) * tiles * p.units_cta +
                                (p.act != SQ_ACT_NONE ? 0.05 : 0.035) * (p.parts == 5 ? 1.8 : 1.0) * p.rows * p.units_cta +
                                0.4 * ((tiles * kTileN * p.rows + kWarps * 32 - 1) / (kWarps * 32)) + (ci ? 0.7 + 0.2 * ci : 0.0) +
                                8.0 * ((tiles + p.tiles_round - 1) / p.tiles_round - 1);
            if (best == 0 || cost < best) best = cost, pick = p;
        }
        if (best != 0) break;
        if (p.rows == 1) return SQ_ERR_UNSUPPORTED;
    }
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(unsigned(pick.clusters * pick.cl), unsigned((pick.M + pick.rows - 1) / pick.rows));
    cfg.blockDim = dim3(kWarps * 32);
    cfg.dynamicSmemBytes = smem_bytes(pick);
    cfg.stream = st;
    cudaLaunchAttribute at[2] = {};
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = unsigned(pick.cl);
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = pick.cl > 1 ? 2 : 1;
    void *args[1] = {&pick};
    const cudaError_t e = cudaLaunchKernelExC(&cfg, matvec_kernel(pick.cols8 / 8, gb, p.z != nullptr, p.parts), args);
    if (e != cudaSuccess) { note_cuda_error(e); return SQ_ERR_CUDA; }
    count_launch();
    return SQ_OK;
}

sq_status launch_quantize_w4_group(const void *W, sq_dtype dt, int64_t N, int64_t K, int64_t ld, int64_t group, void *W4, int64_t ldw,
                                   void *s, sq_dtype s_dtype, int64_t lds, int8_t *z, int64_t ldz, cudaStream_t st)
{
    W4QuantParams p{};
    p.W = W; p.ld = ld; p.N = int(N); p.K = int(K);
    p.group = int(std::min<int64_t>(group, (K + kQuantK - 1) / kQuantK * kQuantK));
    p.span = std::max(p.group, kQuantK);
    const bool longer = kQuantK % p.group != 0;          // more than 512 inputs, or a number that 512 inputs are no multiple of
    if (longer) p.span = p.group;
    p.wide = (reinterpret_cast<uintptr_t>(W) & 31u) == 0 && ld * (dt == SQ_F32 ? 4 : 2) % 32 == 0;
    p.W4 = static_cast<uint8_t *>(W4); p.ldw = ldw;
    p.s = s; p.s_bf16 = s_dtype == SQ_BF16; p.lds = lds; p.z = z; p.ldz = ldz;
    p.groups = int((K + group - 1) / group);
    const int64_t block_rows = 8 * (dt == SQ_F32 ? kWarpRows<float> : kWarpRows<__nv_bfloat16>);
    const int64_t tiles_k = (K + p.span - 1) / p.span, blocks = tiles_k * ((N + block_rows - 1) / block_rows);
    if (blocks > 0x7FFFFFFF) return SQ_ERR_SHAPE;
    p.tiles_k = int(tiles_k);
    auto go = [&](auto kernel) { kernel<<<unsigned(blocks), 256, 0, st>>>(p); };
    auto lanes = [&](auto t, auto zp) {
        using Tin = decltype(t);
        constexpr bool ZP = decltype(zp)::value;
        if (longer) go(quantize_w4_group_kernel<Tin, ZP, 32, true>);
        else if (p.group == 32) go(quantize_w4_group_kernel<Tin, ZP, 2, false>);
        else if (p.group == 64) go(quantize_w4_group_kernel<Tin, ZP, 4, false>);
        else if (p.group == 128) go(quantize_w4_group_kernel<Tin, ZP, 8, false>);
        else if (p.group == 256) go(quantize_w4_group_kernel<Tin, ZP, 16, false>);
        else go(quantize_w4_group_kernel<Tin, ZP, 32, false>);
    };
    if (dt == SQ_F32) z ? lanes(float(), std::true_type()) : lanes(float(), std::false_type());
    else z ? lanes(__nv_bfloat16(), std::true_type()) : lanes(__nv_bfloat16(), std::false_type());
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) { note_cuda_error(e); return SQ_ERR_CUDA; }
    count_launch();
    return SQ_OK;
}

sq_status launch_dequantize_w4_group(const void *W4, int64_t ldw, int64_t N, int64_t K, int64_t group, const void *s, sq_dtype s_dtype,
                                     int64_t lds, const int8_t *z, int64_t ldz, void *W, sq_dtype dt, int64_t ld, cudaStream_t st)
{
    W4DequantParams p{static_cast<const uint8_t *>(W4), ldw, N, K, int(std::min<int64_t>(group, 1 << 30)), s, s_dtype == SQ_BF16, lds,
                      z, ldz, W, ld, (K + group - 1) / group};
    const int64_t by = (N + kTileRows - 1) / kTileRows;
    if (by > 65535) return SQ_ERR_SHAPE;
    const dim3 grid(unsigned((K + kTileK - 1) / kTileK), unsigned(by));
    if (dt == SQ_F32) dequantize_w4_group_kernel<float><<<grid, 256, 0, st>>>(p);
    else dequantize_w4_group_kernel<__nv_bfloat16><<<grid, 256, 0, st>>>(p);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) { note_cuda_error(e); return SQ_ERR_CUDA; }
    count_launch();
    return SQ_OK;
}

}  // namespace sq
