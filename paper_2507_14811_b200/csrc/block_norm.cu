// The end of one block and the start of the next in one pass over the rows (m: row, b = m / rows_per_sample its sample):
//
//   u = post(y)                         none | RMS norm | layer norm, times a weight, plus a bias
//   h = r + alpha gate[b] u             the residual stream, stored rounded; everything below uses it unrounded
//   o = pre(h) w + b                    none | RMS norm | layer norm
//   o = o (1 + scale[b]) + shift[b]     -> values, or the 8-bit codes of segquant_quantize_act
//
// Bound by memory: y and r are read once, h and o (or its codes) written once.  A row stays in registers from the load to the
// store, spread over WPR warps with CH chunks of eight elements a lane: one warp per row needs shuffles alone for its sums, and is
// taken where there are rows enough to fill the GPU; few rows are spread over more warps, which shortens each thread's chain.  Sums
// are fp32; a layer norm's variance is that of the centred values, a second sweep over registers, so that a large mean costs no
// digits.  The vectors of a sample come through L1, which they share with nothing: rows are loaded and stored around it.
#include <cuda_bf16.h>
#include <algorithm>
#include <atomic>
#include <mutex>
#include <vector>
#include "quant_codes.cuh"

namespace sq {

enum : int { kOutValues = 0, kOutInt8 = 1, kOutInt8Dual = 2, kOutE4m3 = 3, kOutE4m3Dual = 4 };

struct BlockNormParams {
    const void *Y, *R;
    int64_t ldy, ldr, M;
    int C;
    int post, pre;
    const void *post_w, *post_b, *w, *b;
    const void *gate, *scale, *shift;
    int64_t ld_gate, ld_scale, ld_shift;
    int64_t rows_per_sample;
    int p_f32;                        // type of those vectors
    int vec;                          // bit i: vector i of post_w, post_b, w, b, gate, scale, shift may be read 16 bytes at a time
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

template <typename T> struct Chunk;                     // eight elements as loaded
template <> struct Chunk<float> { uint4 v[2]; };
template <> struct Chunk<__nv_bfloat16> { uint4 v[1]; };

__device__ __forceinline__ uint4 load_stream(const void *p)            // read once: not kept in L1
{
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
template <typename T>
__device__ __forceinline__ void load_chunk(const T *row, int col, int C, Chunk<T> &c)
{
    constexpr int W = int(sizeof(T)) / 2;
    if (col + 8 <= C) {
#pragma unroll
        for (int i = 0; i < W; i++) c.v[i] = load_stream(reinterpret_cast<const uint4 *>(row + col) + i);
    } else {
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; i++) {
            x[i] = 0.0f;
            if (col + i < C) {
                if (sizeof(T) == 4) x[i] = reinterpret_cast<const float *>(row)[col + i];
                else x[i] = __uint_as_float(uint32_t(reinterpret_cast<const uint16_t *>(row)[col + i]) << 16);
            }
        }
        if (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < W; i++)
                c.v[i] = make_uint4(__float_as_uint(x[4 * i]), __float_as_uint(x[4 * i + 1]), __float_as_uint(x[4 * i + 2]), __float_as_uint(x[4 * i + 3]));
        } else {
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; i++) w[i] = (__float_as_uint(x[2 * i]) >> 16) | (__float_as_uint(x[2 * i + 1]) & 0xFFFF0000u);
            c.v[0] = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
}
template <typename T>
__device__ __forceinline__ void expand(const Chunk<T> &c, float (&x)[8])
{
    const uint32_t *w = reinterpret_cast<const uint32_t *>(c.v);
#pragma unroll
    for (int i = 0; i < 8; i++)
        x[i] = sizeof(T) == 4 ? __uint_as_float(w[i]) : __uint_as_float((i & 1) ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
}
// eight elements of a vector over the channels, `at` elements behind its start
template <typename Tp>
__device__ __forceinline__ void load_vector_of(const Tp *v, int left, bool wide, float (&x)[8])
{
    if (wide && left >= 8) {
        constexpr int W = int(sizeof(Tp)) / 2;
        Chunk<Tp> c;
#pragma unroll
        for (int i = 0; i < W; i++) c.v[i] = __ldg(reinterpret_cast<const uint4 *>(v) + i);
        expand(c, x);
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++) x[i] = i < left ? load1(v + i) : 0.0f;
    }
}
__device__ __forceinline__ void load_vector(const BlockNormParams &prm, const void *v, int64_t at, int col, int which, float (&x)[8])
{
    const bool wide = (prm.vec >> which) & 1;
    if (prm.p_f32) load_vector_of(static_cast<const float *>(v) + at + col, prm.C - col, wide, x);
    else load_vector_of(static_cast<const __nv_bfloat16 *>(v) + at + col, prm.C - col, wide, x);
}
template <typename T>
__device__ __forceinline__ void store_chunk(T *row, int col, int C, const float (&x)[8])
{
    if (col + 8 <= C) {
        uint32_t w[2 * sizeof(T)];
        if (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < 8; i++) w[i % (2 * sizeof(T))] = __float_as_uint(x[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const __nv_bfloat162 b = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
                w[i] = *reinterpret_cast<const uint32_t *>(&b);
            }
        }
#pragma unroll
        for (int i = 0; i < int(sizeof(T)) / 2; i++)
            reinterpret_cast<uint4 *>(row + col)[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++)
            if (col + i < C) {
                if (sizeof(T) == 4) reinterpret_cast<float *>(row)[col + i] = x[i];
                else reinterpret_cast<__nv_bfloat16 *>(row)[col + i] = __float2bfloat16_rn(x[i]);
            }
    }
}

// Sum over the WPR warps of a row, the same bits in every lane.  `red`: WPR floats of the row, another buffer each time.
template <int WPR>
__device__ __forceinline__ float row_sum(float v, float *red, int warp_of_row, int row_of_block)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    if (WPR == 1) return v;
    if ((threadIdx.x & 31) == 0) red[warp_of_row] = v;
    asm volatile("bar.sync %0, %1;" ::"r"(row_of_block + 1), "n"(WPR * 32) : "memory");
    v = 0.0f;
#pragma unroll
    for (int i = 0; i < WPR; i++) v += red[i];
    return v;
}

// x <- normalised x (elements behind the row's end are zero before, and do not count)
template <int CH, int WPR>
__device__ __forceinline__ void normalise(float (&x)[CH][8], int kind, int C, float inv_c, float eps, const int (&col)[CH], float *red,
                                          int warp_of_row, int row_of_block)
{
    if (kind == SQ_NORM_LAYER) {
        float s = 0.0f;
#pragma unroll
        for (int c = 0; c < CH; c++)
#pragma unroll
            for (int i = 0; i < 8; i++) s += x[c][i];
        const float mean = row_sum<WPR>(s, red, warp_of_row, row_of_block) * inv_c;
#pragma unroll
        for (int c = 0; c < CH; c++)
#pragma unroll
            for (int i = 0; i < 8; i++) x[c][i] = col[c] + i < C ? x[c][i] - mean : 0.0f;
        red += WPR;
    }
    float q = 0.0f;
#pragma unroll
    for (int c = 0; c < CH; c++)
#pragma unroll
        for (int i = 0; i < 8; i++) q = fmaf(x[c][i], x[c][i], q);
    const float rstd = 1.0f / sqrtf(fmaf(row_sum<WPR>(q, red, warp_of_row, row_of_block), inv_c, eps));
#pragma unroll
    for (int c = 0; c < CH; c++)
#pragma unroll
        for (int i = 0; i < 8; i++) x[c][i] *= rstd;
}

template <typename T, int OUT, int CH, int WPR, int RPB>
__global__ void __launch_bounds__(WPR * RPB * 32) block_norm_kernel(const __grid_constant__ BlockNormParams prm)
{
    constexpr bool CODES = OUT != kOutValues, DUAL = OUT == kOutInt8Dual || OUT == kOutE4m3Dual;
    constexpr int CODE = OUT >= kOutE4m3 ? SQ_CODE_E4M3 : SQ_CODE_INT8, MODE = DUAL ? kDual : kSingle;
    __shared__ SegConst sm_pos[CODES ? SQ_MAX_P : 1], sm_neg[CODES && DUAL ? SQ_MAX_P : 1];
    __shared__ float sm_red[WPR > 1 ? RPB * 4 * WPR : 1];       // four sums a row: mean and variance, twice
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, row_of_block = warp / WPR, warp_of_row = warp % WPR;
    const int C = prm.C;
    int col[CH];
#pragma unroll
    for (int c = 0; c < CH; c++) col[c] = ((c * WPR + warp_of_row) * 32 + lane) * 8;
    uint32_t seg[CODES ? CH : 1];                              // K-segment of a chunk's first element; bit 31: the chunk crosses a bound
    if (CODES) {
        for (int p = threadIdx.x; p < prm.sb.P; p += blockDim.x) {
            sm_pos[p] = seg_const(__ldg(prm.s_pos + p));
            if (DUAL) sm_neg[p] = seg_const(__ldg(prm.s_neg + p));
        }
#pragma unroll
        for (int c = 0; c < CH; c++) {
            int p = 0;
            while (p + 1 < prm.sb.P && col[c] >= prm.sb.kb[p + 1]) p++;
            seg[c] = uint32_t(p) | (min(col[c] + 8, C) > prm.sb.kb[p + 1] ? 0x80000000u : 0u);
        }
        __syncthreads();
    }
    float *red = sm_red + (WPR > 1 ? row_of_block * 4 * WPR : 0);
    const T *Y = static_cast<const T *>(prm.Y), *R = static_cast<const T *>(prm.R);
    for (int64_t m = int64_t(blockIdx.x) * RPB + row_of_block; m < prm.M; m += int64_t(gridDim.x) * RPB) {
        Chunk<T> y[CH], r[CH];
#pragma unroll
        for (int c = 0; c < CH; c++) {
            if (Y && col[c] < C) load_chunk(Y + m * prm.ldy, col[c], C, y[c]);
            if (R && col[c] < C) load_chunk(R + m * prm.ldr, col[c], C, r[c]);
        }
        const int64_t sample = m / prm.rows_per_sample;
        float h[CH][8];
        if (Y) {
#pragma unroll
            for (int c = 0; c < CH; c++) {
#pragma unroll
                for (int i = 0; i < 8; i++) h[c][i] = 0.0f;
                if (col[c] < C) expand(y[c], h[c]);
            }
            if (prm.post != SQ_NORM_NONE)
                normalise<CH, WPR>(h, prm.post, C, prm.inv_c, prm.eps, col, red, warp_of_row, row_of_block);
#pragma unroll
            for (int c = 0; c < CH; c++) {
                if (col[c] >= C) continue;
                float v[8];
                if (prm.post_w) {
                    load_vector(prm, prm.post_w, 0, col[c], 0, v);
#pragma unroll
                    for (int i = 0; i < 8; i++) h[c][i] *= v[i];
                }
                if (prm.post_b) {
                    load_vector(prm, prm.post_b, 0, col[c], 1, v);
#pragma unroll
                    for (int i = 0; i < 8; i++) h[c][i] += v[i];
                }
                if (prm.gate) {
                    load_vector(prm, prm.gate, sample * prm.ld_gate, col[c], 4, v);
#pragma unroll
                    for (int i = 0; i < 8; i++) h[c][i] *= v[i];
                }
                float x[8];
#pragma unroll
                for (int i = 0; i < 8; i++) x[i] = 0.0f;
                if (R) expand(r[c], x);
#pragma unroll
                for (int i = 0; i < 8; i++) h[c][i] = fmaf(prm.alpha, h[c][i], x[i]);
                if (prm.H) store_chunk(static_cast<T *>(prm.H) + m * prm.ldh, col[c], C, h[c]);
            }
        } else {
#pragma unroll
            for (int c = 0; c < CH; c++) {
#pragma unroll
                for (int i = 0; i < 8; i++) h[c][i] = 0.0f;
                if (col[c] < C) {
                    expand(r[c], h[c]);
                    if (prm.H) store_chunk(static_cast<T *>(prm.H) + m * prm.ldh, col[c], C, h[c]);
                }
            }
        }
        if (CODES || prm.O) {
        // behind the row's end everything is zero, for the sums
#pragma unroll
        for (int c = 0; c < CH; c++)
#pragma unroll
            for (int i = 0; i < 8; i++)
                if (col[c] + i >= C) h[c][i] = 0.0f;
        if (prm.pre != SQ_NORM_NONE)
            normalise<CH, WPR>(h, prm.pre, C, prm.inv_c, prm.eps, col, red + 2 * WPR * (WPR > 1), warp_of_row, row_of_block);
#pragma unroll
        for (int c = 0; c < CH; c++) {
            if (col[c] >= C) continue;
            float v[8], o[8];
#pragma unroll
            for (int i = 0; i < 8; i++) o[i] = h[c][i];
            if (prm.w) {
                load_vector(prm, prm.w, 0, col[c], 2, v);
#pragma unroll
                for (int i = 0; i < 8; i++) o[i] *= v[i];
            }
            if (prm.b) {
                load_vector(prm, prm.b, 0, col[c], 3, v);
#pragma unroll
                for (int i = 0; i < 8; i++) o[i] += v[i];
            }
            if (prm.scale) {
                load_vector(prm, prm.scale, sample * prm.ld_scale, col[c], 5, v);
#pragma unroll
                for (int i = 0; i < 8; i++) o[i] *= 1.0f + v[i];
            }
            if (prm.shift) {
                load_vector(prm, prm.shift, sample * prm.ld_shift, col[c], 6, v);
#pragma unroll
                for (int i = 0; i < 8; i++) o[i] += v[i];
            }
            if (!CODES) {
                store_chunk(static_cast<T *>(prm.O) + m * prm.ldo, col[c], C, o);
            } else {
                const int p = int(seg[c] & 0x7FFFFFFFu);
                const SegConst cp = sm_pos[p], cn = DUAL ? sm_neg[p] : cp;
                uint32_t wp[2], wn[2] = {0, 0};
                const bool fast = !(seg[c] >> 31) && cp.fast && (!DUAL || cn.fast) && !(CODE == SQ_CODE_INT8 && DUAL && prm.lo != -128);
                if (fast) {
                    const float a[4] = {o[0], o[1], o[2], o[3]}, b[4] = {o[4], o[5], o[6], o[7]};
                    quant4<CODE, MODE>(a, cp, cn, float(prm.hi), 0, wp[0], wn[0]);
                    quant4<CODE, MODE>(b, cp, cn, float(prm.hi), 0, wp[1], wn[1]);
                } else {
                    wp[0] = wp[1] = 0;
                    int q = p;
#pragma unroll
                    for (int i = 0; i < 8; i++) {
                        if (col[c] + i >= C) break;
                        while (q + 1 < prm.sb.P && col[c] + i >= prm.sb.kb[q + 1]) q++;
                        uint32_t bp, bn;
                        quant1<CODE, MODE>(o[i], sm_pos[q].s, DUAL ? sm_neg[q].s : 1.0f, 0, prm.lo, prm.hi, bp, bn);
                        wp[i / 4] |= bp << (8 * (i & 3));
                        wn[i / 4] |= bn << (8 * (i & 3));
                    }
                }
                uint8_t *dp = prm.c_pos + m * prm.ldc + col[c], *dn = DUAL ? prm.c_neg + m * prm.ldc + col[c] : nullptr;
                if (col[c] + 8 <= C) {
                    *reinterpret_cast<uint2 *>(dp) = make_uint2(wp[0], wp[1]);
                    if (DUAL) *reinterpret_cast<uint2 *>(dn) = make_uint2(wn[0], wn[1]);
                } else {
                    for (int i = 0; col[c] + i < C; i++) {
                        dp[i] = uint8_t(wp[i / 4] >> (8 * (i & 3)));
                        if (DUAL) dn[i] = uint8_t(wn[i / 4] >> (8 * (i & 3)));
                    }
                }
            }
        }
        }
        // the next row's first sums overwrite words that a slower warp may still be reading
        if (WPR > 1) asm volatile("bar.sync %0, %1;" ::"r"(row_of_block + 1), "n"(WPR * 32) : "memory");
    }
}

// One shape: CH chunks a lane, WPR warps per row, RPB rows per block.
template <typename T, int OUT>
sq_status run_shape(const BlockNormParams &p, cudaStream_t st)
{
    int dev = -1, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
        return SQ_ERR_CUDA;
    auto go = [&](auto kernel, int rpb, int threads) {
        int per_sm = 2048 / threads;
        const int64_t blocks = std::min<int64_t>((p.M + rpb - 1) / rpb, int64_t(sms) * per_sm);
        kernel<<<unsigned(blocks), threads, 0, st>>>(p);
        const cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess) { note_cuda_error(e); return SQ_ERR_CUDA; }
        count_launch();
        return SQ_OK;
    };
    const int chunks = (p.C + 7) / 8;
#define SQ_SHAPE(CH, WPR, RPB) return go(block_norm_kernel<T, OUT, CH, WPR, RPB>, RPB, WPR * RPB * 32)
    const bool many = p.M >= int64_t(sms) * 8;
    if (many && chunks <= 32) SQ_SHAPE(1, 1, 8);
    if (many && chunks <= 64) SQ_SHAPE(2, 1, 8);
    if (many && chunks <= 128) SQ_SHAPE(4, 1, 8);
    if (many && chunks <= 192) SQ_SHAPE(6, 1, 8);
    if (chunks <= 128) SQ_SHAPE(1, 4, 1);
    if (chunks <= 256) SQ_SHAPE(2, 4, 1);
    if (chunks <= 512) SQ_SHAPE(2, 8, 1);
    if (chunks <= 1024) SQ_SHAPE(4, 8, 1);
    if (chunks <= 2048) SQ_SHAPE(4, 16, 1);
#undef SQ_SHAPE
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
    p.Y = a.Y; p.R = a.R; p.ldy = a.ldy; p.ldr = a.ldr; p.M = a.M; p.C = int(a.C);
    p.post = n.post; p.pre = n.pre;
    p.post_w = n.post_w; p.post_b = n.post_b; p.w = n.w; p.b = n.b;
    p.gate = n.gate; p.scale = n.scale; p.shift = n.shift;
    p.ld_gate = n.ld_gate; p.ld_scale = n.ld_scale; p.ld_shift = n.ld_shift;
    p.rows_per_sample = n.rows_per_sample;
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
