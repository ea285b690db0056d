// 4-bit weights with one scale (and zero-point) per output channel and group of inputs: quantization, dequantization and
// the matrix-vector product (few rows of activations).
//
//   w'[n][k] = (c[n][k] - z[g][n]) s[g][n],  g = k / group          y[m][n] = sum_g s[g][n] sum_{k in g} (c - z) a(x[m][k]) + b[n]
//
// The product is bound by reading the codes once: N K / 2 bytes, 12.8 T codes a second at copy bandwidth, for which 148 SMs have
// 2.8 lane instructions per code.  Converting a code to fp32 and one FMA per row would take more than that for a single row;
// so the codes go to the tensor cores as bf16 integers (1.5 instructions per code whatever the number of rows, up to 8):
// mma.m16n8k16 with 16 channels on its rows and the activations' rows on its 8 columns.  tcgen05 would want the expanded codes in
// shared memory, four times the bytes that came in; the tensor pipe is far from being a bound here.
#include <cuda_bf16.h>
#include <algorithm>
#include <atomic>
#include <mutex>
#include <vector>
#include "activation.cuh"

namespace sq {
namespace {

// ---------------------------------------------------------------------------------------------- quantize / dequantize

constexpr int kTileRows = 32;        // channels per block
constexpr int kTileK = 256;          // inputs per block: 8 per lane of a warp
constexpr int kRowsPerWarp = 4;      // 8 warps

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
template <typename Ts> __device__ __forceinline__ float stored_scale(float s);
template <> __device__ __forceinline__ float stored_scale<float>(float s) { return s == 0.0f ? 1.0f : s; }
template <> __device__ __forceinline__ float stored_scale<__nv_bfloat16>(float s)
{
    const float r = __bfloat162float(__float2bfloat16_rn(s));
    return r == 0.0f ? 1.0f : r;
}
__device__ __forceinline__ void store_scale(float *p, float s) { *p = s; }
__device__ __forceinline__ void store_scale(__nv_bfloat16 *p, float s) { *p = __float2bfloat16_rn(s); }

struct W4QuantParams {
    const void *W;
    int64_t ld, N, K;
    int group;
    uint8_t *W4;
    int64_t ldw;
    void *s;
    int64_t lds;
    int8_t *z;
    int64_t ldz;
    int64_t groups;
};

// Bound by reading W: a warp reads 256 consecutive inputs of a channel (four channels in flight), the lanes of a group agree on
// its extrema by shuffles, and the codes leave as 128 consecutive bytes.  Groups longer than 256 read the channel's group twice,
// the second time from cache.  Scales and zero-points are [groups][N]; a block of 32 channels gathers them in shared memory, so that
// they leave as runs of 32 channels.
template <typename Tin, typename Ts, bool ZP>
__global__ void __launch_bounds__(256) quantize_w4_group_kernel(const __grid_constant__ W4QuantParams prm)
{
    __shared__ float sm_s[8][kTileRows];
    __shared__ int8_t sm_z[8][kTileRows];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t n0 = int64_t(blockIdx.y) * kTileRows;
    const int span = prm.group > kTileK ? prm.group : kTileK;            // inputs per block
    const int64_t kb = int64_t(blockIdx.x) * span;
    const int lanes = prm.group >= kTileK ? 32 : prm.group / 8;          // lanes of a group
    const Tin *W = static_cast<const Tin *>(prm.W);

    float x[kRowsPerWarp][8];
    float lo[kRowsPerWarp], hi[kRowsPerWarp];
#pragma unroll
    for (int r = 0; r < kRowsPerWarp; r++) {
        lo[r] = 0.0f, hi[r] = 0.0f;
        const int64_t n = n0 + warp * kRowsPerWarp + r;
        if (n < prm.N) {
            load8(W + n * prm.ld, kb + lane * 8, prm.K, x[r]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; i++) x[r][i] = 0.0f;
        }
    }
#pragma unroll
    for (int r = 0; r < kRowsPerWarp; r++) {
        const int64_t n = n0 + warp * kRowsPerWarp + r;
        for (int64_t k = kb + kTileK; k < kb + span && k < prm.K; k += kTileK) {     // long groups: the rest of the extrema
            float more[8];
            if (n < prm.N) {
                load8(W + n * prm.ld, k + lane * 8, prm.K, more);
#pragma unroll
                for (int i = 0; i < 8; i++) lo[r] = fminf(lo[r], more[i]), hi[r] = fmaxf(hi[r], more[i]);
            }
        }
#pragma unroll
        for (int i = 0; i < 8; i++) lo[r] = fminf(lo[r], x[r][i]), hi[r] = fmaxf(hi[r], x[r][i]);
        for (int o = 1; o < lanes; o <<= 1) {
            lo[r] = fminf(lo[r], __shfl_xor_sync(0xFFFFFFFFu, lo[r], o));
            hi[r] = fmaxf(hi[r], __shfl_xor_sync(0xFFFFFFFFu, hi[r], o));
        }
        const float s = stored_scale<Ts>(ZP ? __fdiv_rn(__fsub_rn(hi[r], lo[r]), 15.0f) : __fdiv_rn(fmaxf(hi[r], -lo[r]), 7.0f));
        float z = 0.0f;
        if (ZP) z = -8.0f - rintf(__fdiv_rn(lo[r], s));
        const SegConst c = seg_const(s);
        const uint64_t r2 = pack2(c.r, c.r), ns2 = pack2(-c.s, -c.s);
        const float c_lo = ZP ? -8.0f : -7.0f;
        for (int64_t k = kb; k < kb + span && k < prm.K; k += kTileK) {
            if (k != kb && n < prm.N) load8(W + n * prm.ld, k + lane * 8, prm.K, x[r]);
            uint32_t word = 0;
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                float q0, q1;
                if (c.fast) {                                            // (see SegConst: the codes of the IEEE quotients)
                    unpack2(div2_rn_fast(pack2(x[r][i], x[r][i + 1]), ns2, r2), q0, q1);
                } else {
                    q0 = __fdiv_rn(x[r][i], s), q1 = __fdiv_rn(x[r][i + 1], s);
                }
                const int a = __float2int_rn(fminf(fmaxf(rintf(q0) + z, c_lo), 7.0f));
                const int b = __float2int_rn(fminf(fmaxf(rintf(q1) + z, c_lo), 7.0f));
                word |= (uint32_t(a & 15) | uint32_t(b & 15) << 4) << (4 * i);
            }
            const int64_t kk = k + lane * 8;
            if (n < prm.N && kk < prm.K) {
                if (kk + 8 > prm.K) word &= 0xFFFFFFFFu >> (4 * int(kk + 8 - prm.K));    // nothing behind the row's last code
                uint8_t *out = prm.W4 + n * prm.ldw + kk / 2;
                if (kk + 8 <= prm.K) {
                    *reinterpret_cast<uint32_t *>(out) = word;
                } else {
                    for (int64_t j = kk; j < prm.K; j += 2) *out++ = uint8_t(word), word >>= 8;
                }
            }
        }
        if (lane % lanes == 0) {
            sm_s[lane / lanes][warp * kRowsPerWarp + r] = s;
            if (ZP) sm_z[lane / lanes][warp * kRowsPerWarp + r] = int8_t(z);
        }
    }
    __syncthreads();
    const int64_t g0 = kb / prm.group;
    for (int i = threadIdx.x; i < (32 / lanes) * kTileRows; i += blockDim.x) {
        const int64_t g = g0 + i / kTileRows, n = n0 + i % kTileRows;
        if (g < prm.groups && n < prm.N) {
            store_scale(static_cast<Ts *>(prm.s) + g * prm.lds + n, sm_s[i / kTileRows][i % kTileRows]);
            if (ZP) prm.z[g * prm.ldz + n] = sm_z[i / kTileRows][i % kTileRows];
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

// The reverse, bound by writing W: a lane turns four bytes into eight values; the block's scales come through shared memory.
template <typename Tout>
__global__ void __launch_bounds__(256) dequantize_w4_group_kernel(const __grid_constant__ W4DequantParams prm)
{
    __shared__ float sm_s[8][kTileRows];
    __shared__ float sm_z[8][kTileRows];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t n0 = int64_t(blockIdx.y) * kTileRows, k0 = int64_t(blockIdx.x) * kTileK, g0 = k0 / prm.group;
    const int in_block = prm.group >= kTileK ? 1 : kTileK / prm.group;
    uint32_t word[kRowsPerWarp];
    const int64_t k = k0 + lane * 8;
#pragma unroll
    for (int r = 0; r < kRowsPerWarp; r++) {
        const int64_t n = n0 + warp * kRowsPerWarp + r;
        word[r] = 0;
        if (n < prm.N && k < prm.K) {
            const uint8_t *p = prm.W4 + n * prm.ldw + k / 2;
            if (k + 8 <= prm.K) {
                word[r] = __ldg(reinterpret_cast<const uint32_t *>(p));
            } else {
                for (int j = 0; k + 2 * j < prm.K; j++) word[r] |= uint32_t(__ldg(p + j)) << (8 * j);
            }
        }
    }
    for (int i = threadIdx.x; i < in_block * kTileRows; i += blockDim.x) {
        const int64_t g = g0 + i / kTileRows, n = n0 + i % kTileRows;
        float s = 0.0f, z = 0.0f;
        if (g < prm.groups && n < prm.N) {
            s = prm.s_bf16 ? load1(static_cast<const __nv_bfloat16 *>(prm.s) + g * prm.lds + n)
                           : __ldg(static_cast<const float *>(prm.s) + g * prm.lds + n);
            if (prm.z) z = float(prm.z[g * prm.ldz + n]);
        }
        sm_s[i / kTileRows][i % kTileRows] = s;
        sm_z[i / kTileRows][i % kTileRows] = z;
    }
    __syncthreads();
    if (k >= prm.K) return;
    const int gi = prm.group >= kTileK ? 0 : lane * 8 / prm.group;
#pragma unroll
    for (int r = 0; r < kRowsPerWarp; r++) {
        const int64_t n = n0 + warp * kRowsPerWarp + r;
        if (n >= prm.N) return;
        const float s = sm_s[gi][warp * kRowsPerWarp + r], z = sm_z[gi][warp * kRowsPerWarp + r];
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const int c = int(word[r] << (28 - 4 * i)) >> 28;
            v[i] = __fmul_rn(float(c) - z, s);
        }
        Tout *out = static_cast<Tout *>(prm.W) + n * prm.ld + k;
        if (k + 8 <= prm.K) {
            if (sizeof(Tout) == 4) {
                reinterpret_cast<float4 *>(out)[0] = make_float4(v[0], v[1], v[2], v[3]);
                reinterpret_cast<float4 *>(out)[1] = make_float4(v[4], v[5], v[6], v[7]);
            } else {
                __nv_bfloat162 b[4];
#pragma unroll
                for (int i = 0; i < 4; i++) b[i] = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
                *reinterpret_cast<uint4 *>(out) = *reinterpret_cast<const uint4 *>(b);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; i++) {
                if (k + i >= prm.K) break;
                if (sizeof(Tout) == 4) reinterpret_cast<float *>(out)[i] = v[i];
                else reinterpret_cast<__nv_bfloat16 *>(out)[i] = __float2bfloat16_rn(v[i]);
            }
        }
    }
}

// ---------------------------------------------------------------------------------------------- matrix-vector product

constexpr int kWarps = 16;
constexpr int kTileN = 16;           // channels of a warp: the MMA's rows
constexpr int kUnitK = 256;          // codes per channel and ring stage: 128 bytes
constexpr int kUnitBytes = kTileN * kUnitK / 2;
constexpr int kMaxStages = 4;         // of a warp's ring; 2 or 3 where the activations leave no room for more
constexpr int kRedPitch = 20;        // floats per column of a warp's partial sums (16 used; 20 keeps the stores off one bank)
constexpr int kMaxCols = 32;

struct MatvecParams {
    const void *X;
    int64_t ldx;
    int M, rows;                     // rows of X, rows of one pass (grid.y)
    int64_t K;
    int x_f32, x_wide, act, parts;   // parts: bf16 terms per activation (1, or 3 for fp32 values)
    const uint8_t *W4;
    int64_t ldw, N, row_bytes;
    int group;
    int64_t groups;
    const uint8_t *s;
    int s_bytes;                     // 4 or 2
    int64_t lds;                     // bytes
    const int8_t *z;
    int64_t ldz;
    const float *bias;
    void *Y;
    int y_f32;
    int64_t ldy;
    int units, cl, wk, wk_shift;     // K: units in all, CTAs of a cluster, warps of a CTA that share it
    int units_cta, units_warp;
    int64_t tiles;                   // of 16 * (16 / wk) channels
    int clusters;
    int cols;                        // columns in use: rows * parts
    int stages;
    uint32_t stage_bytes, z_off, x_off, red_off, red_bytes;
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
__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// Codes i and i + 4 of a word of eight, as bf16 integers less an offset: a nibble c with its top bit flipped is c + 8, and the
// bits 0x4300 | (c + 8) are the bf16 number 136 + c, so that subtracting 136 + z leaves c - z, exactly.
__device__ __forceinline__ uint32_t code_pair(uint32_t word, int i, uint32_t offset)
{
    uint32_t v, d;
    asm("lop3.b32 %0, %1, %2, %3, 0x6A;" : "=r"(v) : "r"(word >> (4 * i)), "r"(0x000F000Fu), "r"(0x43084308u));   // (a & b) ^ c
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(v), "r"(offset));
    return d;
}
__device__ __forceinline__ float act1(float x, int act)
{
    float a, b;
    if (act == SQ_ACT_NONE) return x;
    unpack2(act == SQ_ACT_SILU ? silu2(x, x) : gelu2(x, x), a, b);
    return a;
}
// an fp32 value as the sum of three bf16 numbers, exactly (truncations of 8 significant bits each); what is not finite keeps
// its kind in the first
__device__ __forceinline__ void split3(float x, uint32_t (&p)[3])
{
    const uint32_t bits = __float_as_uint(x);
    if ((bits & 0x7F800000u) == 0x7F800000u) {
        p[0] = x == x ? bits >> 16 : 0x7FC0u;
        p[1] = p[2] = 0;
        return;
    }
    const float r1 = x - __uint_as_float(bits & 0xFFFF0000u);
    const uint32_t b1 = __float_as_uint(r1);
    const float r2 = r1 - __uint_as_float(b1 & 0xFFFF0000u);
    p[0] = bits >> 16, p[1] = b1 >> 16, p[2] = __float_as_uint(r2) >> 16;
}

// A CTA of 16 warps holds its share of the activations in shared memory as MMA operands and goes through tiles of channels; a
// tile's K range is shared by `wk` of its warps, and by the `cl` CTAs of a cluster.  Every warp streams 16 channels x 256 codes at a
// time through a ring of its own (asynchronous copies; nothing but the warp itself waits for them), so the ring keeps going while
// the partial sums of a finished tile are added up, in a fixed order.
//
// Codes of one channel that share 16 bytes are handed to the four lanes of a row by ldmatrix, eight each; a lane's eight give the
// pairs (0, 4), (1, 5), (2, 6), (3, 7) by shifting, which is the order that the activations are laid out in: any order of K will
// do as long as both operands have it.  GB: groups of inputs per ring stage, 256 / group (1 for longer groups).  Products of codes
// and bf16 activations are exact, a group's sum is fp32, and the scale is applied to it in fp32.
template <int NT, int GB>
__global__ void __launch_bounds__(kWarps * 32, 1) w4_matvec_kernel(const __grid_constant__ MatvecParams prm)
{
    extern __shared__ __align__(128) uint8_t smem[];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    const int cl = prm.cl, wk = prm.wk, wn = kWarps / wk;
    const int rank = cl > 1 ? int(blockIdx.x) % cl : 0, cluster = int(blockIdx.x) / cl;
    const int m0 = int(blockIdx.y) * prm.rows, rows = min(prm.rows, prm.M - m0);
    const int my_k = warp & (wk - 1), my_n = warp >> prm.wk_shift;
    // this CTA's units, and this warp's
    const int c_u0 = rank * prm.units_cta, c_u1 = min(prm.units, c_u0 + prm.units_cta);
    const int u0 = min(c_u1, c_u0 + my_k * prm.units_warp), u1 = min(c_u1, u0 + prm.units_warp);

    const uint32_t ring = smem_addr(smem) + warp * prm.stages * prm.stage_bytes;

    // ---- the ring: copies of the unit (pt, pu), one stage after the other
    int64_t pt = cluster;
    int pu = u0;
    if (u0 >= u1) pt = prm.tiles;
    const int wr = lane >> 3, wc = lane & 7;             // this lane's 16-byte pieces: rows wr, wr + 4, ..
    auto issue = [&](int slot) {
        if (pt < prm.tiles) {
            const uint32_t dst = ring + slot * prm.stage_bytes;
            const int64_t n0 = (pt * wn + my_n) * kTileN;
            const int64_t off = int64_t(pu) * (kUnitK / 2) + wc * 16;
            const int bytes = int(max(int64_t(0), min(int64_t(16), prm.row_bytes - off)));
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const int r = wr + 4 * i;
                const bool in = n0 + r < prm.N && bytes > 0;
                copy16(dst + r * 128 + ((wc ^ (r & 7)) << 4), in ? prm.W4 + (n0 + r) * prm.ldw + off : prm.W4, in ? bytes : 0);
            }
            const int64_t g0 = GB > 1 ? int64_t(pu) * GB : int64_t(pu) * kUnitK / prm.group;
            const int pieces = prm.s_bytes;              // 16-byte pieces of 16 channels' scales: 4 (fp32) or 2 (bf16)
            if (lane < GB * pieces) {
                const int gi = lane / pieces, pc = lane % pieces, per = 16 / prm.s_bytes;
                const int64_t left = (prm.N - n0 - pc * per) * prm.s_bytes;
                const bool in = g0 + gi < prm.groups && left > 0;
                copy16(dst + kUnitBytes + lane * 16, in ? prm.s + (g0 + gi) * prm.lds + (n0 + pc * per) * prm.s_bytes : prm.s,
                       in ? int(min(int64_t(16), left)) : 0);
            }
            if (prm.z && lane < GB) {
                const bool in = g0 + lane < prm.groups && n0 < prm.N;
                copy16(dst + prm.z_off + lane * 16, in ? prm.z + (g0 + lane) * prm.ldz + n0 : prm.z,
                       in ? int(min(int64_t(16), prm.N - n0)) : 0);
            }
            if (++pu == u1) pu = u0, pt += prm.clusters;
        }
        copies_commit();
    };
    for (int i = 0; i < prm.stages - 1; i++) issue(i);

    // ---- activations: per 32 inputs, [column][32 bf16] with each eight as (0, 4), (1, 5), (2, 6), (3, 7); zero behind the last
    // input, so that whatever lies there in a row of codes counts for nothing
    const int eights = (c_u1 - c_u0) * (kUnitK / 8);
    for (int i = tid; i < eights * rows; i += kWarps * 32) {
        const int m = i / eights, e = i - m * eights;
        const int64_t k = int64_t(c_u0) * kUnitK + e * 8;
        float x[8];
        if (prm.x_f32) load8(static_cast<const float *>(prm.X) + (m0 + m) * prm.ldx, k, prm.K, x, prm.x_wide);
        else load8(static_cast<const __nv_bfloat16 *>(prm.X) + (m0 + m) * prm.ldx, k, prm.K, x, prm.x_wide);
        uint32_t w[3][4];
#pragma unroll
        for (int j = 0; j < 4; j++) {
            uint32_t a[3], b[3];
            split3(act1(x[j], prm.act), a);
            split3(act1(x[j + 4], prm.act), b);
#pragma unroll
            for (int p = 0; p < 3; p++) w[p][j] = a[p] | b[p] << 16;
        }
        uint8_t *dst = smem + prm.x_off + size_t(e >> 2) * (prm.cols * 64) + (e & 3) * 16;
#pragma unroll
        for (int p = 0; p < 3; p++)
            if (p < prm.parts) *reinterpret_cast<uint4 *>(dst + (p * prm.rows + m) * 64) = make_uint4(w[p][0], w[p][1], w[p][2], w[p][3]);
    }
    __syncthreads();

    // ---- tiles
    uint32_t xb[NT];                                     // this lane's activations: column g (+ 8 per MMA), codes 8 t ..
#pragma unroll
    for (int nt = 0; nt < NT; nt++) xb[nt] = smem_addr(smem) + prm.x_off + min(g + 8 * nt, prm.cols - 1) * 64 + t * 16;
    const uint32_t lm_row = (lane & 15) * 128, lm_seg = lane >> 4, lm_x = lane & 7;      // ldmatrix: rows 0-15 of two pieces
    int slot = 0, buf = 0;
    for (int64_t tile = cluster; tile < prm.tiles; tile += prm.clusters) {
        float acc[NT][4];
#pragma unroll
        for (int nt = 0; nt < NT; nt++)
#pragma unroll
            for (int i = 0; i < 4; i++) acc[nt][i] = 0.0f;
        for (int u = u0; u < u1; u++) {
            if (prm.stages == 4) copies_wait<2>();
            else if (prm.stages == 3) copies_wait<1>();
            else copies_wait<0>();
            __syncwarp();
            issue(slot == 0 ? prm.stages - 1 : slot - 1);   // the stage that was used up last
            const uint32_t st = ring + slot * prm.stage_bytes;
            const uint8_t *stp = smem + (st - smem_addr(smem));
            const uint32_t x_unit = uint32_t(u - c_u0) * 8 * (prm.cols * 64);
            constexpr int SEGS = 8 / GB;                 // 32-code pieces per group
            uint32_t w[4];
#pragma unroll
            for (int gi = 0; gi < GB; gi++) {
                float sum[NT][4];
#pragma unroll
                for (int nt = 0; nt < NT; nt++)
#pragma unroll
                    for (int i = 0; i < 4; i++) sum[nt][i] = 0.0f;
                uint32_t off0 = 0x43084308u, off1 = 0x43084308u;          // 136, 136
                if (prm.z) {
                    const int8_t *z = reinterpret_cast<const int8_t *>(stp + prm.z_off) + gi * 16;
                    const __nv_bfloat162 z0 = __float2bfloat162_rn(136.0f + float(z[g]));
                    const __nv_bfloat162 z1 = __float2bfloat162_rn(136.0f + float(z[g + 8]));
                    off0 = *reinterpret_cast<const uint32_t *>(&z0);
                    off1 = *reinterpret_cast<const uint32_t *>(&z1);
                }
#pragma unroll
                for (int s = gi * SEGS; s < (gi + 1) * SEGS; s++) {
                    if (s % 2 == 0) load_matrices(st + lm_row + (((s + lm_seg) ^ lm_x) << 4), w);
                    const uint32_t w0 = w[s % 2 * 2], w1 = w[s % 2 * 2 + 1];
                    uint32_t a[4], b[4];
#pragma unroll
                    for (int i = 0; i < 4; i++) a[i] = code_pair(w0, i, off0), b[i] = code_pair(w1, i, off1);
#pragma unroll
                    for (int nt = 0; nt < NT; nt++) {
                        uint32_t x0, x1, x2, x3;
                        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(x0), "=r"(x1), "=r"(x2), "=r"(x3)
                                     : "r"(xb[nt] + x_unit + s * (prm.cols * 64)));
                        mma(sum[nt], a[0], b[0], a[1], b[1], x0, x1);
                        mma(sum[nt], a[2], b[2], a[3], b[3], x2, x3);
                    }
                }
                float s0, s1;
                if (prm.s_bytes == 4) {
                    const float *sc = reinterpret_cast<const float *>(stp + kUnitBytes) + gi * 16;
                    s0 = sc[g], s1 = sc[g + 8];
                } else {
                    const uint16_t *sc = reinterpret_cast<const uint16_t *>(stp + kUnitBytes) + gi * 16;
                    s0 = __uint_as_float(uint32_t(sc[g]) << 16), s1 = __uint_as_float(uint32_t(sc[g + 8]) << 16);
                }
#pragma unroll
                for (int nt = 0; nt < NT; nt++) {
                    acc[nt][0] = fmaf(s0, sum[nt][0], acc[nt][0]), acc[nt][1] = fmaf(s0, sum[nt][1], acc[nt][1]);
                    acc[nt][2] = fmaf(s1, sum[nt][2], acc[nt][2]), acc[nt][3] = fmaf(s1, sum[nt][3], acc[nt][3]);
                }
            }
            slot = slot + 1 == prm.stages ? 0 : slot + 1;
        }
        // partial sums of this warp: [column][16 channels]
        float *red = reinterpret_cast<float *>(smem + prm.red_off + buf * prm.red_bytes);
        float *mine = red + warp * (prm.cols * kRedPitch);
#pragma unroll
        for (int nt = 0; nt < NT; nt++) {
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const int col = nt * 8 + 2 * t + (i & 1);
                if (col < prm.cols) mine[col * kRedPitch + g + (i >> 1) * 8] = acc[nt][i];
            }
        }
        if (cl > 1) {
            asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
        } else {
            __syncthreads();
        }
        // output o of the tile, summed by wk lanes: every lane adds a warp's columns over the cluster's CTAs and the parts of an
        // activation, then the lanes add up; the CTAs of a cluster take turns with the outputs
        const int outs = kTileN * wn * rows, turns = (outs + cl - 1) / cl;
        for (int i = tid; i - lane < turns * wk; i += kWarps * 32) {
            const int o = (i >> prm.wk_shift) * cl + rank, j = i & (wk - 1);
            float v = 0.0f;
            if (o < outs) {
                const int c = o & 15, q = o >> 4, m = q / wn, n16 = q - m * wn;
                const uint32_t at = smem_addr(red + (n16 * wk + j) * (prm.cols * kRedPitch) + m * kRedPitch + c);
                for (int r = 0; r < cl; r++) {
                    uint32_t src = at;
                    if (cl > 1) asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(src) : "r"(at), "r"(r));
                    for (int p = 0; p < prm.parts; p++) {
                        float f;
                        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(f) : "r"(src + p * prm.rows * kRedPitch * 4) : "memory");
                        v += f;
                    }
                }
            }
            for (int d = 1; d < wk; d <<= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
            if (o < outs && j == 0) {
                const int c = o & 15, q = o >> 4, m = q / wn, n16 = q - m * wn;
                const int64_t n = (tile * wn + n16) * kTileN + c;
                if (n < prm.N) {
                    if (prm.bias) v += __ldg(prm.bias + n);
                    const int64_t at = (m0 + m) * prm.ldy + n;
                    if (prm.y_f32) static_cast<float *>(prm.Y)[at] = v;
                    else static_cast<__nv_bfloat16 *>(prm.Y)[at] = __float2bfloat16_rn(v);
                }
            }
        }
        buf ^= 1;            // the next tile's partial sums: whoever still reads these has not passed that tile's barrier
    }
    if (cl > 1) asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// ---------------------------------------------------------------------------------------------- host side

template <int NT>
const void *matvec_kernel(int gb)
{
    switch (gb) {
        case 1: return reinterpret_cast<const void *>(w4_matvec_kernel<NT, 1>);
        case 2: return reinterpret_cast<const void *>(w4_matvec_kernel<NT, 2>);
        case 4: return reinterpret_cast<const void *>(w4_matvec_kernel<NT, 4>);
        default: return reinterpret_cast<const void *>(w4_matvec_kernel<NT, 8>);
    }
}
const void *matvec_kernel(int nt, int gb)
{
    switch (nt) {
        case 1: return matvec_kernel<1>(gb);
        case 2: return matvec_kernel<2>(gb);
        case 3: return matvec_kernel<3>(gb);
        default: return matvec_kernel<4>(gb);
    }
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
    for (int nt = 1; nt <= 4 && e == cudaSuccess; nt++)
        for (int gb = 1; gb <= 8 && e == cudaSuccess; gb *= 2)
            e = cudaFuncSetAttribute(matvec_kernel(nt, gb), cudaFuncAttributeMaxDynamicSharedMemorySize, int(kMaxSmem));
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
        e = cudaOccupancyMaxActiveClusters(&d.clusters[i], matvec_kernel(1, 1), &cfg);
    }
    if (e != cudaSuccess) { note_cuda_error(e); return SQ_ERR_CUDA; }
    g_devices.push_back(d);
    *out = d;
    return SQ_OK;
}

std::atomic<int> g_w4_cl{0}, g_w4_wk{0};

// Shared memory of a split, and whether it fits.
bool lay_out(MatvecParams &p, int gb)
{
    const uint32_t s_bytes = uint32_t(gb * kTileN * p.s_bytes), z_bytes = p.z ? uint32_t(gb * kTileN) : 0u;
    p.z_off = kUnitBytes + s_bytes;
    p.stage_bytes = (p.z_off + z_bytes + 127u) & ~127u;
    const size_t x_bytes = size_t(p.units_cta) * 8 * p.cols * 64;
    p.red_bytes = uint32_t(kWarps * p.cols * kRedPitch * 4);
    for (p.stages = kMaxStages; p.stages >= 2; p.stages--) {
        p.x_off = uint32_t(kWarps * p.stages) * p.stage_bytes;
        if (p.x_off + x_bytes + 2 * size_t(p.red_bytes) > kMaxSmem) continue;
        p.red_off = uint32_t(p.x_off + x_bytes);
        return true;
    }
    return false;
}

}  // namespace

void set_w4_tuning(int cl, int wk) { g_w4_cl = cl; g_w4_wk = wk; }

sq_status launch_w4_matvec(const W4MatvecArgs &a, cudaStream_t st)
{
    MatvecDevice dev;
    sq_status r = matvec_device(&dev);
    if (r != SQ_OK) return r;
    MatvecParams p{};
    p.X = a.X; p.ldx = a.ldx; p.M = int(a.M); p.K = a.K; p.x_f32 = a.dt == SQ_F32;
    p.x_wide = aligned16(a.X) && (a.M == 1 || a.ldx * (p.x_f32 ? 4 : 2) % 16 == 0);
    p.act = int(a.act);
    p.parts = p.x_f32 || p.act != SQ_ACT_NONE ? 3 : 1;
    p.W4 = static_cast<const uint8_t *>(a.W4); p.ldw = a.ldw; p.N = a.N; p.row_bytes = (a.K + 1) / 2;
    p.group = int(std::min<int64_t>(a.group, 1 << 30)); p.groups = (a.K + a.group - 1) / a.group;
    p.s = static_cast<const uint8_t *>(a.s); p.s_bytes = a.s_dtype == SQ_F32 ? 4 : 2; p.lds = a.lds * p.s_bytes;
    p.z = a.z; p.ldz = a.ldz; p.bias = a.bias;
    p.Y = a.Y; p.y_f32 = a.y_dtype == SQ_F32; p.ldy = a.ldy;
    p.units = int((a.K + kUnitK - 1) / kUnitK);
    const int gb = a.group >= kUnitK ? 1 : int(kUnitK / a.group);

    // Rows of a pass: as many as 32 columns take, spread evenly; fewer where the activations would not fit.
    const int most = kMaxCols / p.parts;
    int passes = (p.M + most - 1) / most;
    double best = 0;
    MatvecParams pick{};
    for (;; passes++) {
        p.rows = (p.M + passes - 1) / passes;
        p.cols = p.rows * p.parts;
        const int want_cl = g_w4_cl.load(std::memory_order_relaxed), want_wk = g_w4_wk.load(std::memory_order_relaxed);
        for (int ci = 0; ci < 4; ci++) {
            for (int wi = 0; wi < 5; wi++) {
                MatvecParams q = p;
                q.cl = 1 << ci; q.wk = 1 << wi; q.wk_shift = wi;
                if ((want_cl && q.cl != want_cl) || (want_wk && q.wk != want_wk)) continue;
                if (dev.clusters[ci] < 1 || (ci && q.cl > q.units)) continue;
                q.units_cta = (q.units + q.cl - 1) / q.cl;
                q.units_warp = (q.units_cta + q.wk - 1) / q.wk;
                const int tile_n = kTileN * (kWarps / q.wk);
                q.tiles = (q.N + tile_n - 1) / tile_n;
                if (!lay_out(q, gb)) continue;
                q.clusters = int(std::min<int64_t>(q.tiles, dev.clusters[ci]));
                const double rounds = double((q.tiles + q.clusters - 1) / q.clusters);
                const double cost = rounds * (0.5 * q.units_warp + (ci ? 1.0 : 0.3)) + 0.0005 * q.cols * q.units_cta * kUnitK / 16.0;
                if (best == 0 || cost < best) best = cost, pick = q;
            }
        }
        if (best != 0) break;
        if (p.rows == 1) return SQ_ERR_UNSUPPORTED;
    }
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(unsigned(pick.clusters * pick.cl), unsigned((pick.M + pick.rows - 1) / pick.rows));
    cfg.blockDim = dim3(kWarps * 32);
    cfg.dynamicSmemBytes = pick.red_off + 2 * pick.red_bytes;
    cfg.stream = st;
    cudaLaunchAttribute at{};
    if (pick.cl > 1) {
        at.id = cudaLaunchAttributeClusterDimension;
        at.val.clusterDim.x = unsigned(pick.cl);
        at.val.clusterDim.y = at.val.clusterDim.z = 1;
        cfg.attrs = &at;
        cfg.numAttrs = 1;
    }
    void *args[1] = {&pick};
    const cudaError_t e = cudaLaunchKernelExC(&cfg, matvec_kernel((pick.cols + 7) / 8, gb), args);
    if (e != cudaSuccess) { note_cuda_error(e); return SQ_ERR_CUDA; }
    count_launch();
    return SQ_OK;
}

sq_status launch_quantize_w4_group(const void *W, sq_dtype dt, int64_t N, int64_t K, int64_t ld, int64_t group, void *W4, int64_t ldw,
                                   void *s, sq_dtype s_dtype, int64_t lds, int8_t *z, int64_t ldz, cudaStream_t st)
{
    W4QuantParams p{W, ld, N, K, int(std::min<int64_t>(group, 1 << 30)), static_cast<uint8_t *>(W4), ldw, s, lds, z, ldz,
                    (K + group - 1) / group};
    const int64_t span = std::max<int64_t>(p.group, kTileK), by = (N + kTileRows - 1) / kTileRows;
    if (by > 65535) return SQ_ERR_SHAPE;
    const dim3 grid(unsigned((K + span - 1) / span), unsigned(by));
    auto go = [&](auto t, auto ts) {
        using Tin = decltype(t);
        using Ts = decltype(ts);
        if (z) quantize_w4_group_kernel<Tin, Ts, true><<<grid, 256, 0, st>>>(p);
        else quantize_w4_group_kernel<Tin, Ts, false><<<grid, 256, 0, st>>>(p);
    };
    if (dt == SQ_F32) s_dtype == SQ_F32 ? go(float(), float()) : go(float(), __nv_bfloat16());
    else s_dtype == SQ_F32 ? go(__nv_bfloat16(), float()) : go(__nv_bfloat16(), __nv_bfloat16());
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
