// The end of one block and the start of the next in one pass over the rows (m: row, b = m / rows_per_sample its sample):
//
//   u = post(y)                         none | RMS norm | layer norm, times a weight, plus a bias
//   h = r + alpha gate[b] u             the residual stream, stored rounded; everything below uses it unrounded
//   o = pre(h) w + b                    none | RMS norm | layer norm
//   o = o (1 + scale[b]) + shift[b]     -> values, or the 8-bit codes of segquant_quantize_act
//
// Bound by memory: y and r are read once, h and o (or its codes) written once.  A row stays in registers from the load to the
// store, spread over WPR warps with CH chunks of eight elements a lane, and a row group's next row is on its way while the current
// one is worked on.  One warp per row needs shuffles alone for its sums and is taken where there are rows enough to fill the GPU; few rows are
// spread over a block each, which shortens every thread's chain.  Sums are fp32; a layer norm's variance is that of the centred
// values, a second sweep over registers, so that a large mean costs no digits.
//
// What is done per channel on either side is one multiply-add: h = r + (yn P + Q), o = hn A + B with P = alpha post_w gate,
// Q = alpha post_b gate, A = w (1 + scale), B = b (1 + scale) + shift.  A block makes these vectors in shared memory for the sample that its rows
// belong to; reading up to seven vectors of two types, aligned or not, for every row instead made a kernel of some 50 KB of
// instructions, which waited for its own code (8858 x 1536 bf16, two RMS norms: 63.6 us; gated and modulated to codes 135 us).
#include <cuda_bf16.h>
#include <algorithm>
#include "quant_codes.cuh"

namespace sq {

enum : int { kOutValues = 0, kOutInt8 = 1, kOutInt8Dual = 2, kOutE4m3 = 3, kOutE4m3Dual = 4 };

struct BlockNormParams {
    const void *Y, *R;
    int64_t ldy, ldr;
    int M, C;
    int ragged;                       // C is no multiple of 8
    int post, pre;
    const void *post_w, *post_b, *w, *b;
    const void *gate, *scale, *shift;
    int64_t ld_gate, ld_scale, ld_shift;
    int rows_per_sample;              // at most M
    int p_f32;                        // type of those vectors
    int vec;                          // bit i: vector i of post_w, post_b, w, b, gate, scale, shift may be read 16 bytes at a time
    int has;                          // bits: which of P, Q, A, B there are
    int sm_at[4];                     // where they lie in shared memory
    int pitch, half;                  // floats of a vector there (eight zeros at the end), of half a one
    int own;                          // floats of a row's own vectors there (0: rows share them)
    int two_steps;                    // shared memory holds P and Q or A and B
    float alpha, eps, inv_c;
    void *H, *O;
    int64_t ldh, ldo;
    SegBounds sb;
    const float *s_pos, *s_neg;
    int lo, hi;
    uint8_t *c_pos, *c_neg;
    int64_t ldc;
};

#ifdef SQ_NORM_OUT     // the kernels of one kind of output; the kinds are compiled side by side
namespace {

constexpr int kMaxVectorBytes = 220 * 1024;       // of the vectors in shared memory

template <typename T> struct Chunk;                     // eight elements as loaded
template <> struct Chunk<float> { uint4 v[2]; };
template <> struct Chunk<__nv_bfloat16> { uint4 v[1]; };
struct Eight { float v[8]; };

__device__ __forceinline__ uint4 load_stream(const void *p)            // read once: not kept in L1
{
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
// Words of 16 bytes that hold at least one element of the row (rows start on 16-byte boundaries, so what else is in such a word
// belongs to the same allocation); the others are zero.
template <typename T>
__device__ __forceinline__ void load_chunk(const T *row, int col, int C, Chunk<T> &c)
{
    constexpr int W = int(sizeof(T)) / 2, PER = 16 / int(sizeof(T));
#pragma unroll
    for (int i = 0; i < W; i++) {
        c.v[i] = make_uint4(0u, 0u, 0u, 0u);
        if (col + i * PER < C) c.v[i] = load_stream(row + col + i * PER);
    }
}
// eight elements as four packed pairs: most of the arithmetic goes two elements per instruction
template <typename T>
__device__ __forceinline__ void expand(const Chunk<T> &c, uint64_t (&x)[4])
{
    const uint32_t *w = reinterpret_cast<const uint32_t *>(c.v);
#pragma unroll
    for (int i = 0; i < 4; i++)
        x[i] = sizeof(T) == 4 ? pack2(__uint_as_float(w[2 * i % (2 * sizeof(T))]), __uint_as_float(w[(2 * i + 1) % (2 * sizeof(T))]))
                              : pack2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xFFFF0000u));
}
__device__ __forceinline__ void singles(const uint64_t (&x)[4], float (&v)[8])
{
#pragma unroll
    for (int i = 0; i < 4; i++) unpack2(x[i], v[2 * i], v[2 * i + 1]);
}
// elements behind the row's end become zero, for the sums
__device__ __forceinline__ void cut(uint64_t (&x)[4], int left)
{
#pragma unroll
    for (int i = 0; i < 4; i++) {
        float a, b;
        unpack2(x[i], a, b);
        x[i] = pack2(2 * i < left ? a : 0.0f, 2 * i + 1 < left ? b : 0.0f);
    }
}
template <typename T>
__device__ __noinline__ void store_tail(T *p, int left, Eight x)
{
#pragma unroll
    for (int i = 0; i < 8; i++)
        if (i < left) {
            if (sizeof(T) == 4) reinterpret_cast<float *>(p)[i] = x.v[i];
            else reinterpret_cast<__nv_bfloat16 *>(p)[i] = __float2bfloat16_rn(x.v[i]);
        }
}
template <typename T>
__device__ __forceinline__ void store_whole(T *p, const uint64_t (&pairs)[4])
{
    float x[8];
    singles(pairs, x);
    if (sizeof(T) == 4) {
        reinterpret_cast<float4 *>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
        reinterpret_cast<float4 *>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
    } else {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const __nv_bfloat162 b = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t *>(&b);
        }
        *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}
template <typename T>
__device__ __forceinline__ void store_chunk(T *row, int col, int C, const uint64_t (&pairs)[4])
{
    float x[8];
    singles(pairs, x);
    if (col + 8 <= C) {
        store_whole(row + col, pairs);
    } else {
        Eight e;
#pragma unroll
        for (int i = 0; i < 8; i++) e.v[i] = x[i];
        store_tail(row + col, C - col, e);
    }
}

// ---- the vectors of a sample
enum : int { kP = 0, kQ = 1, kA = 2, kB = 3 };
__device__ __forceinline__ float vector1(const BlockNormParams &prm, const void *v, int64_t at)
{
    return prm.p_f32 ? __ldg(static_cast<const float *>(v) + at) : load1(static_cast<const __nv_bfloat16 *>(v) + at);
}
// eight channels of one of the seven vectors; `absent` where it is not there
__device__ __forceinline__ void vector8(const BlockNormParams &prm, const void *v, int64_t at, int which, int left, float absent, float (&x)[8])
{
    if (!v) {
#pragma unroll
        for (int i = 0; i < 8; i++) x[i] = absent;
    } else if (((prm.vec >> which) & 1) && left >= 8) {
        if (prm.p_f32) {
            Chunk<float> c;
#pragma unroll
            for (int i = 0; i < 2; i++) c.v[i] = __ldg(reinterpret_cast<const uint4 *>(static_cast<const float *>(v) + at) + i);
            uint64_t p[4];
            expand(c, p);
            singles(p, x);
        } else {
            Chunk<__nv_bfloat16> c;
            c.v[0] = __ldg(reinterpret_cast<const uint4 *>(static_cast<const __nv_bfloat16 *>(v) + at));
            uint64_t p[4];
            expand(c, p);
            singles(p, x);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++) x[i] = i < left ? vector1(prm, v, at + i) : 0.0f;
    }
}
// A vector in shared memory is two halves, of the first and of the last four channels of every eight, so that neighbouring lanes
// read neighbouring 16 bytes (`half`: floats of one).
__device__ __forceinline__ void put8(float *v, int half, int col, const float (&x)[8])
{
    *reinterpret_cast<float4 *>(v + col / 2) = make_float4(x[0], x[1], x[2], x[3]);
    *reinterpret_cast<float4 *>(v + half + col / 2) = make_float4(x[4], x[5], x[6], x[7]);
}
__device__ __forceinline__ void get8(const float *v, int half, int col, uint64_t (&x)[4])
{
    const ulonglong2 a = *reinterpret_cast<const ulonglong2 *>(v + col / 2), b = *reinterpret_cast<const ulonglong2 *>(v + half + col / 2);
    x[0] = a.x; x[1] = a.y; x[2] = b.x; x[3] = b.y;
}
// P and Q
__device__ __forceinline__ void make_post(const BlockNormParams &prm, float *sm, int64_t sample, int col)
{
    if (!(prm.has & (1 << kP | 1 << kQ))) return;
    const int left = prm.C - col;
    float w[8], b[8], g[8];
    vector8(prm, prm.post_w, col, 0, left, 1.0f, w);
    vector8(prm, prm.post_b, col, 1, left, 0.0f, b);
    vector8(prm, prm.gate, sample * prm.ld_gate + col, 4, left, 1.0f, g);
#pragma unroll
    for (int i = 0; i < 8; i++) {
        g[i] *= prm.alpha;
        w[i] *= g[i];
        b[i] *= g[i];
    }
    if (prm.has >> kP & 1) put8(sm + prm.sm_at[kP], prm.half, col, w);
    if (prm.has >> kQ & 1) put8(sm + prm.sm_at[kQ], prm.half, col, b);
}
// A and B
__device__ __forceinline__ void make_pre(const BlockNormParams &prm, float *sm, int64_t sample, int col)
{
    if (!(prm.has & (1 << kA | 1 << kB))) return;
    const int left = prm.C - col;
    float w[8], b[8], s[8], t[8];
    vector8(prm, prm.w, col, 2, left, 1.0f, w);
    vector8(prm, prm.b, col, 3, left, 0.0f, b);
    vector8(prm, prm.scale, sample * prm.ld_scale + col, 5, left, 0.0f, s);
    vector8(prm, prm.shift, sample * prm.ld_shift + col, 6, left, 0.0f, t);
#pragma unroll
    for (int i = 0; i < 8; i++) {
        const float f = 1.0f + s[i];
        w[i] *= f;
        b[i] = fmaf(b[i], f, t[i]);
    }
    if (prm.has >> kA & 1) put8(sm + prm.sm_at[kA], prm.half, col, w);
    if (prm.has >> kB & 1) put8(sm + prm.sm_at[kB], prm.half, col, b);
}

// Sum over the WPR warps (the L lanes) of a row, the same bits in every lane.  `red`: WPR floats of the row, another buffer each time.
template <int WPR, int L>
__device__ __forceinline__ float row_sum(float v, float *red, int warp_of_row, int row_of_block)
{
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    if (WPR == 1) return v;
    if ((threadIdx.x & 31) == 0) red[warp_of_row] = v;
    asm volatile("bar.sync %0, %1;" ::"r"(row_of_block + 1), "n"(WPR * 32) : "memory");
    v = 0.0f;
    if (WPR % 4 == 0) {
#pragma unroll
        for (int i = 0; i < WPR; i += 4) {
            const float4 f = *reinterpret_cast<const float4 *>(red + i);
            v += f.x + f.y + f.z + f.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < WPR; i++) v += red[i];
    }
    return v;
}

// x <- normalised x (elements behind the row's end are zero before, and do not count)
template <int CH, int WPR, int L>
__device__ __forceinline__ void normalise(uint64_t (&x)[CH][4], int kind, const BlockNormParams &prm, const int (&col)[CH], float *red,
                                          int warp_of_row, int row_of_block)
{
    float a, b;
    if (kind == SQ_NORM_LAYER) {
        uint64_t s = 0;
#pragma unroll
        for (int c = 0; c < CH; c++)
#pragma unroll
            for (int i = 0; i < 4; i++) s = add2(s, x[c][i]);
        unpack2(s, a, b);
        const float mean = row_sum<WPR, L>(a + b, red, warp_of_row, row_of_block) * prm.inv_c;
#pragma unroll
        for (int c = 0; c < CH; c++) {
            const float m = col[c] < prm.C ? -mean : 0.0f;
#pragma unroll
            for (int i = 0; i < 4; i++) x[c][i] = add2(x[c][i], pack2(m, m));
            if (prm.ragged) cut(x[c], prm.C - col[c]);
        }
        red += WPR;
    }
    uint64_t q = 0;
#pragma unroll
    for (int c = 0; c < CH; c++)
#pragma unroll
        for (int i = 0; i < 4; i++) q = fma2(x[c][i], x[c][i], q);
    unpack2(q, a, b);
    const float rstd = 1.0f / sqrtf(fmaf(row_sum<WPR, L>(a + b, red, warp_of_row, row_of_block), prm.inv_c, prm.eps));
#pragma unroll
    for (int c = 0; c < CH; c++)
#pragma unroll
        for (int i = 0; i < 4; i++) x[c][i] = mul2(x[c][i], pack2(rstd, rstd));
}

// Codes of a chunk that crosses a segment bound or the row's end, or whose scale is outside the fast form: element by element.
template <int CODE, int MODE>
__device__ __noinline__ void codes_tail(const BlockNormParams &prm, int col, Eight o, uint8_t *dp, uint8_t *dn)
{
    int q = 0;
#pragma unroll
    for (int i = 0; i < 8; i++) {
        if (col + i >= prm.C) return;
        while (q + 1 < prm.sb.P && col + i >= prm.sb.kb[q + 1]) q++;
        uint32_t bp, bn;
        quant1<CODE, MODE>(o.v[i], __ldg(prm.s_pos + q), MODE == kDual ? __ldg(prm.s_neg + q) : 1.0f, 0, prm.lo, prm.hi, bp, bn);
        dp[i] = uint8_t(bp);
        if (MODE == kDual) dn[i] = uint8_t(bn);
    }
}

// Threads of a block: RPB rows at a time, WPR warps each, or L = 8 or 16 lanes for rows of at most 64 and 128 channels.  A block's rows share the
// vectors of their sample in shared memory; with OWN vectors (a block per row, or samples of few rows) every thread makes and
// reads those of its own channels, so nothing has to wait.  BLOCKS: resident blocks per SM that the registers are held to.
template <typename T, int OUT, int CH, int WPR, int RPB, int BLOCKS, bool OWN, int L = 32>
__global__ void __launch_bounds__(WPR * RPB * L, BLOCKS) block_norm_kernel(const __grid_constant__ BlockNormParams prm)
{
    static_assert(OWN || RPB > 1, "rows to share with");
    static_assert(L == 32 || (WPR == 1 && CH == 1), "rows of a few lanes");
    constexpr bool CODES = OUT != kOutValues, DUAL = OUT == kOutInt8Dual || OUT == kOutE4m3Dual;
    constexpr int CODE = OUT >= kOutE4m3 ? SQ_CODE_E4M3 : SQ_CODE_INT8, MODE = DUAL ? kDual : kSingle;
    extern __shared__ __align__(16) float sm[];
    __shared__ SegConst sm_pos[CODES ? SQ_MAX_P : 1], sm_neg[CODES && DUAL ? SQ_MAX_P : 1];
    __shared__ __align__(16) float sm_red[WPR > 1 ? RPB * 4 * WPR : 1];       // four sums a row: mean and variance, twice
    const int lane = threadIdx.x & (L - 1), warp = threadIdx.x >> 5, row_of_block = threadIdx.x / (WPR * L), warp_of_row = warp % WPR;
    const int of_warp = L < 32 ? (threadIdx.x & 31) / L : 0;     // which of its warp's rows
    const int C = prm.C;
    float *vec = sm + (OWN && RPB > 1 ? row_of_block * prm.own : 0);
    const T *Y = static_cast<const T *>(prm.Y), *R = static_cast<const T *>(prm.R);
    // this block's rows, and its row group's first
    const int r0 = int(int64_t(blockIdx.x) * prm.M / gridDim.x), r1 = int((int64_t(blockIdx.x) + 1) * prm.M / gridDim.x);
    int m = r0 + row_of_block, sample = -1;
    int col[CH], at[CH];
    Chunk<T> y[CH], r[CH];
    auto fetch = [&](int row) {
#pragma unroll
        for (int c = 0; c < CH; c++) {
            if (Y) load_chunk(Y + row * prm.ldy, col[c], C, y[c]);
            if (R) load_chunk(R + row * prm.ldr, col[c], C, r[c]);
        }
    };
#pragma unroll
    for (int c = 0; c < CH; c++) {
        col[c] = ((c * WPR + warp_of_row) * L + lane) * 8;
        at[c] = col[c] < C ? col[c] : prm.pitch - 8;           // its vectors: behind the row's end zeros
        if (!Y || !R) y[c] = r[c] = Chunk<T>{};
    }
    asm volatile("griddepcontrol.launch_dependents;\n\tgriddepcontrol.wait;" ::: "memory");     // nothing is read before the kernel in front is done
    if (m < r1) fetch(m);

    uint32_t seg[CODES ? CH : 1];                              // K-segment of a chunk; bit 31: it is done element by element
    if (CODES) {
        for (int p = threadIdx.x; p < prm.sb.P; p += blockDim.x) {
            sm_pos[p] = seg_const(__ldg(prm.s_pos + p));
            if (DUAL) sm_neg[p] = seg_const(__ldg(prm.s_neg + p));
        }
        __syncthreads();
#pragma unroll
        for (int c = 0; c < CH; c++) {
            int p = 0;
            while (p + 1 < prm.sb.P && col[c] >= prm.sb.kb[p + 1]) p++;
            const bool fast = col[c] + 8 <= prm.sb.kb[p + 1] && sm_pos[p].fast && (!DUAL || sm_neg[p].fast) &&
                              !(CODE == SQ_CODE_INT8 && DUAL && prm.lo != -128);
            seg[c] = uint32_t(p) | (fast ? 0u : 0x80000000u);
        }
    }
    bool all_fast = CODES;
#pragma unroll
    for (int c = 0; c < CH; c++) all_fast = all_fast && (col[c] >= C || !(seg[CODES ? c : 0] >> 31));
    all_fast = __all_sync(0xFFFFFFFFu, all_fast);
    float *red = sm_red + (WPR > 1 ? row_of_block * 4 * WPR : 0);
    // zeros behind every vector; with vectors of its own each row has them
    if (lane < 8 && warp_of_row == 0) {
#pragma unroll
        for (int i = 0; i < 4; i++)
            if (prm.has >> i & 1) vec[prm.sm_at[i] + (lane < 4 ? 0 : prm.half) + prm.pitch / 2 - 4 + (lane & 3)] = 0.0f;
    }
    if (WPR > 1) __syncthreads();
    else __syncwarp();
    for (int start = r0, end; start < r1; start = end) {
        end = r1;
        if (!OWN) {                                            // the rows of one sample
            sample = start / prm.rows_per_sample;
            end = int(min(int64_t(r1), (int64_t(sample) + 1) * prm.rows_per_sample));
            if (start != r0) __syncthreads();                  // the last sample's vectors have been used
            for (int k = int(threadIdx.x) * 8; k < C; k += int(blockDim.x) * 8) {
                make_post(prm, vec, sample, k);
                make_pre(prm, vec, sample, k);
            }
            __syncthreads();
            if (L < 32 && start != r0) {                       // (rows that share a warp start a sample together)
                m = start + row_of_block;
                if (m < r1) fetch(m);
            }
        }
        for (; m - of_warp < end; m += RPB) {                  // whole warps
            const bool valid = L == 32 || m < end;
            if (OWN && !prm.two_steps && valid && m / prm.rows_per_sample != sample) {
                sample = m / prm.rows_per_sample;
#pragma unroll 1
                for (int c = 0; c < CH; c++) {
                    const int k = ((c * WPR + warp_of_row) * L + lane) * 8;
                    if (k < C) make_post(prm, vec, sample, k), make_pre(prm, vec, sample, k);
                }
            }
            if (OWN && RPB == 1 && prm.two_steps) sample = m / prm.rows_per_sample;
            // Branches stand around loops over the chunks, not inside them, so that the chunks of a row are worked on side by side;
            // chunks behind the row's end read zeros for its vectors and stay zero, and only stores ask where they are.
            uint64_t h[CH][4];
            if (Y) {
#pragma unroll
                for (int c = 0; c < CH; c++) expand(y[c], h[c]);
                if (prm.post != SQ_NORM_NONE) {
                    if (prm.ragged) {
#pragma unroll
                        for (int c = 0; c < CH; c++) cut(h[c], C - col[c]);
                    }
                    normalise<CH, WPR, L>(h, prm.post, prm, col, red, warp_of_row, row_of_block);
                }
                if (RPB == 1 && prm.two_steps) {
#pragma unroll 1
                    for (int c = 0; c < CH; c++) {
                        const int k = ((c * WPR + warp_of_row) * L + lane) * 8;
                        if (k < C) make_post(prm, vec, sample, k);
                    }
                }
                const float *vp = vec + prm.sm_at[kP], *vq = vec + prm.sm_at[kQ];
                const int with = prm.has & (1 << kP | 1 << kQ);
                if (with == (1 << kP | 1 << kQ)) {
#pragma unroll
                    for (int c = 0; c < CH; c++) {
                        uint64_t v[4], w[4], x[4];
                        expand(r[c], x);
                        get8(vp, prm.half, at[c], v);
                        get8(vq, prm.half, at[c], w);
#pragma unroll
                        for (int i = 0; i < 4; i++) h[c][i] = fma2(h[c][i], v[i], add2(x[i], w[i]));
                    }
                } else if (with) {
                    const bool p_only = with == 1 << kP;
                    if (p_only) {
#pragma unroll
                        for (int c = 0; c < CH; c++) {
                            uint64_t v[4], x[4];
                            expand(r[c], x);
                            get8(vp, prm.half, at[c], v);
#pragma unroll
                            for (int i = 0; i < 4; i++) h[c][i] = fma2(h[c][i], v[i], x[i]);
                        }
                    } else {
#pragma unroll
                        for (int c = 0; c < CH; c++) {
                            uint64_t v[4], x[4];
                            expand(r[c], x);
                            get8(vq, prm.half, at[c], v);
#pragma unroll
                            for (int i = 0; i < 4; i++) h[c][i] = add2(h[c][i], add2(x[i], v[i]));
                        }
                    }
                } else {
#pragma unroll
                    for (int c = 0; c < CH; c++) {
                        uint64_t x[4];
                        expand(r[c], x);
#pragma unroll
                        for (int i = 0; i < 4; i++) h[c][i] = add2(h[c][i], x[i]);
                    }
                }
            } else {
#pragma unroll
                for (int c = 0; c < CH; c++) expand(r[c], h[c]);
            }
            // the next row's loads go out before anything is stored; it is never a row that this group still has to write
            if (m + RPB < r1) fetch(m + RPB);
            auto store_row = [&](T *row) {
                if (prm.ragged) {
#pragma unroll
                    for (int c = 0; c < CH; c++)
                        if (valid && col[c] < C) store_chunk(row, col[c], C, h[c]);
                } else {
#pragma unroll
                    for (int c = 0; c < CH; c++)
                        if (valid && col[c] < C) store_whole(row + col[c], h[c]);
                }
            };
            if (prm.H) store_row(static_cast<T *>(prm.H) + m * prm.ldh);
            if (CODES || prm.O) {
                if (prm.ragged) {
#pragma unroll
                    for (int c = 0; c < CH; c++) cut(h[c], C - col[c]);
                }
                if (prm.pre != SQ_NORM_NONE)
                    normalise<CH, WPR, L>(h, prm.pre, prm, col, red + 2 * WPR * (WPR > 1), warp_of_row, row_of_block);
                if (RPB == 1 && prm.two_steps) {
#pragma unroll 1
                    for (int c = 0; c < CH; c++) {
                        const int k = ((c * WPR + warp_of_row) * L + lane) * 8;
                        if (k < C) make_pre(prm, vec, sample, k);
                    }
                }
                const float *va = vec + prm.sm_at[kA], *vb = vec + prm.sm_at[kB];
                const int with = prm.has >> kA & 3;
                if (with == 3) {
#pragma unroll
                    for (int c = 0; c < CH; c++) {
                        uint64_t v[4], w[4];
                        get8(va, prm.half, at[c], v);
                        get8(vb, prm.half, at[c], w);
#pragma unroll
                        for (int i = 0; i < 4; i++) h[c][i] = fma2(h[c][i], v[i], w[i]);
                    }
                } else if (with == 1) {
#pragma unroll
                    for (int c = 0; c < CH; c++) {
                        uint64_t v[4];
                        get8(va, prm.half, at[c], v);
#pragma unroll
                        for (int i = 0; i < 4; i++) h[c][i] = mul2(h[c][i], v[i]);
                    }
                } else if (with == 2) {
#pragma unroll
                    for (int c = 0; c < CH; c++) {
                        uint64_t v[4];
                        get8(vb, prm.half, at[c], v);
#pragma unroll
                        for (int i = 0; i < 4; i++) h[c][i] = add2(h[c][i], v[i]);
                    }
                }
                if (!CODES) {
                    store_row(static_cast<T *>(prm.O) + m * prm.ldo);
                } else {
                    uint8_t *rp = prm.c_pos + m * prm.ldc, *rn = DUAL ? prm.c_neg + m * prm.ldc : nullptr;
                    auto fast = [&](int c) {
                        const int p = int(seg[c] & 0x7FFFFFFFu);
                        const SegConst cp = sm_pos[p], cn = DUAL ? sm_neg[p] : cp;
                        float a[4], b[4];
                        unpack2(h[c][0], a[0], a[1]), unpack2(h[c][1], a[2], a[3]);
                        unpack2(h[c][2], b[0], b[1]), unpack2(h[c][3], b[2], b[3]);
                        uint32_t wp[2], wn[2];
                        quant4<CODE, MODE>(a, cp, cn, float(prm.hi), 0, wp[0], wn[0]);
                        quant4<CODE, MODE>(b, cp, cn, float(prm.hi), 0, wp[1], wn[1]);
                        if (valid && col[c] < C) {
                            *reinterpret_cast<uint2 *>(rp + col[c]) = make_uint2(wp[0], wp[1]);
                            if (DUAL) *reinterpret_cast<uint2 *>(rn + col[c]) = make_uint2(wn[0], wn[1]);
                        }
                    };
                    if (all_fast) {
#pragma unroll
                        for (int c = 0; c < CH; c++) fast(c);
                    } else {
#pragma unroll
                        for (int c = 0; c < CH; c++) {
                            if (!(seg[c] >> 31)) {
                                fast(c);
                            } else if (valid && col[c] < C) {
                                Eight e;
                                singles(h[c], e.v);
                                codes_tail<CODE, MODE>(prm, col[c], e, rp + col[c], DUAL ? rn + col[c] : nullptr);
                            }
                        }
                    }
                }
            }
            // the next row's first sums overwrite words that a slower warp may still be reading
            if (WPR > 1) asm volatile("bar.sync %0, %1;" ::"r"(row_of_block + 1), "n"(WPR * 32) : "memory");
        }
    }
}

// One shape: CH chunks a lane, WPR warps per row, RPB rows of a block at a time.  A warp per row up to 1280 bf16 (1024 fp32) channels
// where there are at least five per SM, two, four and eight up to 8192, then a block per row; fewer rows get a block each: of two and more per SM several share an SM, so
// blocks are small (300 x 12000 14.2 us against 20.7 with blocks as wide as below, 700 x 16384 29.0 against 40.1, 600 x 4096 8.6 against 9.6; 600 x 1536
// 6.2 against 5.7, 400 x 8192 11.9 against 10.6), below that as many warps as a row keeps busy (160 x 1536 3.5 us against 4.7, 290 x 8192 8.0 against 9.0).  (2048 x 5120:
// 35 us with a block per row, 20.5 with two rows a block, which share their vectors.)  Rows of up to 128
// channels take 8 or 16 lanes (32768 x 64: 14.1 -> 5.5 us).  Samples of fewer than 16 rows: every row makes its vectors (16384 x 640, a vector
// per row: 93.7 us with a block per row, 51.4 with a warp).  (8858 x 1536 bf16 to codes: one warp with six chunks a lane, held to 128 registers, 28.1 us; two with three
// 23.1 us.  32768 x 1280: one warp with five chunks 55.8 us, two with three, of which one sixth is idle, 63.2 us.)
template <typename T, int OUT>
sq_status run_shape(BlockNormParams p, cudaStream_t st)
{
    int dev = -1, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
        return SQ_ERR_CUDA;
    const int pitch = (p.C + 7) / 8 * 8 + 8;             // floats of a vector in shared memory
    p.pitch = pitch;
    int vectors = 0;
    p.half = pitch / 2;
    for (int i = 0; i < 4; i++)
        if (p.has >> i & 1) p.sm_at[i] = pitch * vectors++;
    // samples of few rows: every row has its own vectors, where shared memory has room for that
    const bool few_a_sample = p.rows_per_sample < 16;
    auto go = [&](auto kernel, int threads, int rpb, int blocks_per_sm) {
        size_t smem = size_t(vectors) * pitch * 4;
        if (rpb == 1 && smem > kMaxVectorBytes) {        // all four, over 14080 channels: two at a time then, made anew for every row
            p.two_steps = 1;
            p.sm_at[kA] = 0, p.sm_at[kB] = pitch;
            smem /= 2;
        }
        if (rpb > 1 && few_a_sample) {
            p.own = vectors * pitch;
            smem *= rpb;
        }
        if (smem > 40 * 1024) {                          // (the kernel has a few KB of its own)
            const cudaError_t e = cudaFuncSetAttribute(reinterpret_cast<const void *>(kernel), cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxVectorBytes);
            if (e != cudaSuccess) { note_cuda_error(e); return SQ_ERR_CUDA; }
        }
        const int fit = int(kMaxVectorBytes / (smem + 4096));
        const int per_sm = std::max(1, std::min(blocks_per_sm, fit));
        const int64_t blocks = std::min<int64_t>((p.M + rpb - 1) / rpb, int64_t(sms) * per_sm);
        cudaLaunchConfig_t cfg{};
        cfg.gridDim = dim3(unsigned(blocks));
        cfg.blockDim = dim3(unsigned(threads));
        cfg.dynamicSmemBytes = smem;
        cfg.stream = st;
        cudaLaunchAttribute at{};
        at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
        at.val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = &at;
        cfg.numAttrs = 1;
        void *args[1] = {&p};
        const cudaError_t e = cudaLaunchKernelExC(&cfg, reinterpret_cast<const void *>(kernel), args);
        if (e != cudaSuccess) { note_cuda_error(e); return SQ_ERR_CUDA; }
        count_launch();
        return SQ_OK;
    };
    const int chunks = (p.C + 7) / 8;
    constexpr bool HALF = sizeof(T) == 2;
#define SQ_SHARED(CH, WPR, RPB, BLOCKS, L)                                                                                  \
    return few_a_sample ? go(block_norm_kernel<T, OUT, CH, WPR, RPB, BLOCKS, true, L>, WPR * RPB * L, RPB, BLOCKS)          \
                        : go(block_norm_kernel<T, OUT, CH, WPR, RPB, BLOCKS, false, L>, WPR * RPB * L, RPB, BLOCKS)
#define SQ_ROW(CH, WPR, BLOCKS) return go(block_norm_kernel<T, OUT, CH, WPR, 1, BLOCKS, true>, WPR * 32, 1, BLOCKS)
    if (p.M >= int64_t(sms) * 5 && (!few_a_sample || size_t(vectors) * pitch * 4 * 8 <= size_t(kMaxVectorBytes))) {
        if (chunks <= 8) SQ_SHARED(1, 1, 32, 4, 8);
        if (chunks <= 16) SQ_SHARED(1, 1, 16, 4, 16);
        if (chunks <= 32) SQ_SHARED(1, 1, 8, 4, 32);
        if (chunks <= 64) SQ_SHARED(2, 1, 8, HALF ? 4 : 3, 32);
        if (chunks <= 96) SQ_SHARED(3, 1, 8, HALF ? 3 : 2, 32);
        if (chunks <= 128) SQ_SHARED(4, 1, 8, 2, 32);
        if constexpr (HALF) {
            if (chunks <= 160) SQ_SHARED(5, 1, 8, 2, 32);
        }
        if (chunks <= 192) SQ_SHARED(3, 2, 4, HALF ? 3 : 2, 32);
        if (chunks <= 256) SQ_SHARED(4, 2, 4, 2, 32);
        if (chunks <= 512) SQ_SHARED(4, 4, 2, 2, 32);
        if (chunks <= 768) SQ_SHARED(3, 8, 2, 1, 32);
        if (chunks <= 1024) SQ_SHARED(4, 8, 2, 1, 32);
    }
    if (p.M >= int64_t(sms) * 2) {
        if (chunks <= 128) SQ_ROW(1, 4, 6);
        if (chunks <= 256) SQ_ROW(2, 4, 4);
        if (chunks <= 512) SQ_ROW(2, 8, 2);
        if (chunks <= 768) SQ_ROW(3, 8, HALF ? 3 : 2);
        if (chunks <= 1024) SQ_ROW(4, 8, 2);
        SQ_ROW(4, 16, 1);
    }
    if (chunks <= 128) SQ_ROW(1, 4, 6);
    if (chunks <= 256) SQ_ROW(1, 8, 2);
    if (chunks <= 512) SQ_ROW(1, 16, 1);
    if (chunks <= 1024) SQ_ROW(1, 32, 1);
    if (chunks <= 2048) SQ_ROW(2, 32, 1);
#undef SQ_SHARED
#undef SQ_ROW
    return SQ_ERR_UNSUPPORTED;
}

}  // namespace

template <int OUT>
sq_status run_block_norm(const BlockNormParams &p, sq_dtype dt, cudaStream_t st)
{
    return dt == SQ_F32 ? run_shape<float, OUT>(p, st) : run_shape<__nv_bfloat16, OUT>(p, st);
}
template sq_status run_block_norm<SQ_NORM_OUT>(const BlockNormParams &, sq_dtype, cudaStream_t);
#else
template <int OUT> sq_status run_block_norm(const BlockNormParams &p, sq_dtype dt, cudaStream_t st);

static bool wide(const void *v, int64_t ld, size_t size) { return aligned16(v) && (size_t(ld) * size) % 16 == 0; }

sq_status launch_block_norm(const BlockNormArgs &a, cudaStream_t st)
{
    BlockNormParams p{};
    const sq_block_norm &n = *a.norm;
    const size_t ps = n.p_dtype == SQ_F32 ? 4 : 2;
    p.Y = a.Y; p.R = a.R; p.ldy = a.ldy; p.ldr = a.ldr; p.M = int(a.M); p.C = int(a.C); p.ragged = a.C % 8 != 0;
    p.post = n.post; p.pre = n.pre;
    p.post_w = n.post_w; p.post_b = n.post_b; p.w = n.w; p.b = n.b;
    p.gate = n.gate; p.scale = n.scale; p.shift = n.shift;
    p.ld_gate = n.ld_gate; p.ld_scale = n.ld_scale; p.ld_shift = n.ld_shift;
    p.rows_per_sample = int(std::min(n.rows_per_sample, a.M));
    if (a.Y) p.has |= (n.post_w || n.gate || n.alpha != 1.0f) << 0 | (n.post_b != nullptr) << 1;
    if (a.O || a.c_pos) p.has |= (n.w || n.scale) << 2 | (n.b || n.shift) << 3;
    p.vec = wide(n.post_w, 0, ps) | wide(n.post_b, 0, ps) << 1 | wide(n.w, 0, ps) << 2 | wide(n.b, 0, ps) << 3 |
            wide(n.gate, n.ld_gate, ps) << 4 | wide(n.scale, n.ld_scale, ps) << 5 | wide(n.shift, n.ld_shift, ps) << 6;
    p.alpha = n.alpha; p.eps = n.eps; p.inv_c = 1.0f / float(a.C);
    p.H = a.H; p.ldh = a.ldh; p.O = a.O; p.ldo = a.ldo;
    p.p_f32 = n.p_dtype == SQ_F32;
    if (!a.c_pos) return run_block_norm<kOutValues>(p, a.dt, st);
    p.sb = a.sb;
    p.s_pos = a.s_pos; p.s_neg = a.s_neg;
    p.c_pos = static_cast<uint8_t *>(a.c_pos); p.c_neg = static_cast<uint8_t *>(a.c_neg); p.ldc = a.ldc;
    p.hi = int(a.q_max); p.lo = a.s_neg ? -int(a.q_min_abs) : -p.hi;
    if (a.code == SQ_CODE_INT8) return a.s_neg ? run_block_norm<kOutInt8Dual>(p, a.dt, st) : run_block_norm<kOutInt8>(p, a.dt, st);
    return a.s_neg ? run_block_norm<kOutE4m3Dual>(p, a.dt, st) : run_block_norm<kOutE4m3>(p, a.dt, st);
}

#endif

}  // namespace sq
