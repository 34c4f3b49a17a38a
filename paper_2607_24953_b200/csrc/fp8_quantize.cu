// fp4q_fp8_quantize: BF16 or FP32 -> E4M3 codes with an FP32 scale for every block of 128, both orientations in one reading.
//
// A CTA of 8 warps owns 128 x 128 elements: one block of every row, one of every column, one square block.  A warp has 16 rows, a lane 4 consecutive rows x 16
// columns, so that eight lanes make a row's block and a lane's four rows a word of the transposed codes; those cross 16 KB of shared memory
// (pieces of 16 bytes, swizzled by the column's group) and leave as 128 consecutive bytes a column.  Bound by memory, 2 or 4 bytes an element read and 1 or 2 written, and nearly as much by its instructions:
// 16384 x 4096 BF16, both orientations, 55 us, 5.0 TB/s; FP32 in square blocks 64 us, 6.3 TB/s.  BF16 with four CTAs an SM (64 registers) 52 us in a row, with three 56.
#include "common.cuh"
#include "fp8_format.cuh"
#include "row_io.cuh"

using namespace fp4q;

namespace {

struct Fp8QuantParams {
    int64_t rows, cols;
    RowsOf<__nv_bfloat16> b16;   // x as what it is
    RowsOf<float> f32;
    fp4q_fp8_tensor out;
    int64_t col_tiles;
};

template <typename T>
__device__ __forceinline__ const RowsOf<T> &source(const Fp8QuantParams &p)
{
    if constexpr (sizeof(T) == 4) return p.f32;
    else return p.b16;
}

// Magnitudes: packed pairs of BF16, or FP32.  Infinity where there is one; NaN does not count.
__device__ __forceinline__ uint32_t max_pair(uint32_t a, uint32_t b)
{
    const __nv_bfloat162 m = __hmax2(*reinterpret_cast<const __nv_bfloat162 *>(&a), *reinterpret_cast<const __nv_bfloat162 *>(&b));
    return *reinterpret_cast<const uint32_t *>(&m);
}
__device__ __forceinline__ float high(uint32_t pair) { return __uint_as_float(pair & 0xFFFF0000u); }
__device__ __forceinline__ float low(uint32_t pair) { return __uint_as_float(pair << 16); }

// Maxima of a lane's four rows and, over these, of its columns.
template <typename T>
__device__ __forceinline__ void maxima(const Raw<T> (&x)[4], float (&rows)[4], uint32_t (&cols)[Raw<T>::kWords])
{
#pragma unroll
    for (int k = 0; k < Raw<T>::kWords; k++) cols[k] = 0u;
#pragma unroll
    for (int i = 0; i < 4; i++) {
        uint32_t pair = 0u;
        float m = 0.f;
#pragma unroll
        for (int k = 0; k < Raw<T>::kWords; k++) {
            if constexpr (sizeof(T) == 2) {
                const uint32_t a = x[i].w[k] & 0x7FFF7FFFu;
                pair = max_pair(pair, a);
                cols[k] = max_pair(cols[k], a);
            } else {
                const float a = fabsf(x[i][k]);
                m = fmaxf(m, a);
                cols[k] = __float_as_uint(fmaxf(__uint_as_float(cols[k]), a));
            }
        }
        rows[i] = sizeof(T) == 2 ? fmaxf(low(pair), high(pair)) : m;
    }
}

// GRID: rows begin on 16 bytes.
template <typename T, bool SQUARE, bool GRID>
__global__ void __launch_bounds__(256, sizeof(T) == 2 ? 4 : 2) fp8_quantize_kernel(const __grid_constant__ Fp8QuantParams p)
{
    wait_for_predecessor();
    admit_successor();
    __shared__ uint4 stage[128 * 8];      // 128 columns x 128 bytes
    __shared__ float tops[8][128];
    __shared__ __align__(16) float factors[128];
    constexpr bool kPairs = sizeof(T) == 2;
    constexpr int W = Raw<T>::kWords;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, cg = lane & 7, rg = lane >> 3;
    const int64_t by = blockIdx.x / p.col_tiles, bx = blockIdx.x - by * p.col_tiles;
    const int64_t row0 = by * 128 + warp * 16 + rg * 4, col0 = bx * 128 + cg * 16;

    const int n = columns_at(col0, p.cols);
    Raw<T> x[4];
    {
        Pieces<T, GRID> on_way[4];
#pragma unroll
        for (int i = 0; i < 4; i++) on_way[i].fetch(source<T>(p), row0 + i < p.rows ? row0 + i : 0, col0, row0 + i < p.rows ? n : 0);
#pragma unroll
        for (int i = 0; i < 4; i++) x[i] = on_way[i].land(source<T>(p), row0 + i < p.rows ? row0 + i : 0, col0, row0 + i < p.rows ? n : 0);
    }

    float row_top[4];
    uint32_t col_top[W];
    maxima(x, row_top, col_top);
    float all = fmaxf(fmaxf(row_top[0], row_top[1]), fmaxf(row_top[2], row_top[3]));
    if (__any_sync(0xFFFFFFFFu, is_infinite(all))) {   // maxima of finite elements only; infinities become NaN, which they are from here on
#pragma unroll
        for (int i = 0; i < 4; i++)
#pragma unroll
            for (int k = 0; k < W; k++) {
                uint32_t &w = x[i].w[k];
                if constexpr (kPairs) {
                    if ((w & 0x7FFFu) == 0x7F80u) w |= 0x7FFFu;
                    if ((w & 0x7FFF0000u) == 0x7F800000u) w |= 0x7FFF0000u;
                } else {
                    if ((w & 0x7FFFFFFFu) == 0x7F800000u) w |= 0x7FFFFFFFu;
                }
            }
        maxima(x, row_top, col_top);
        all = fmaxf(fmaxf(row_top[0], row_top[1]), fmaxf(row_top[2], row_top[3]));
    }
    float row_factor = 0.f;   // of row cg & 3 of the lane's rows, or of the square block
    if (!SQUARE) {
        if (p.out.q) {
#pragma unroll
            for (int i = 0; i < 4; i++)
#pragma unroll
                for (int d = 1; d < 8; d <<= 1) row_top[i] = fmaxf(row_top[i], __shfl_xor_sync(0xFFFFFFFFu, row_top[i], d));
            const int i = cg & 3;
            const float m = i == 0 ? row_top[0] : i == 1 ? row_top[1] : i == 2 ? row_top[2] : row_top[3];
            row_factor = fp8_factor(m);
            if (cg < 4 && row0 + i < p.rows) p.out.scale[(row0 + i) * p.out.ld_s + bx] = fp8_scale(m);
        }
        if (p.out.q_t) {
#pragma unroll
            for (int k = 0; k < W; k++) {
                uint32_t m = col_top[k];
#pragma unroll
                for (int d = 8; d < 32; d <<= 1) {
                    const uint32_t o = __shfl_xor_sync(0xFFFFFFFFu, m, d);
                    if constexpr (kPairs) m = max_pair(m, o);
                    else m = __float_as_uint(fmaxf(__uint_as_float(m), __uint_as_float(o)));
                }
                if (rg == (k & 3)) {
                    if constexpr (kPairs) {
                        tops[warp][16 * cg + 2 * k] = low(m);
                        tops[warp][16 * cg + 2 * k + 1] = high(m);
                    } else {
                        tops[warp][16 * cg + k] = __uint_as_float(m);
                    }
                }
            }
            __syncthreads();
            if (threadIdx.x < 128) {
                float m = tops[0][threadIdx.x];
#pragma unroll
                for (int w = 1; w < 8; w++) m = fmaxf(m, tops[w][threadIdx.x]);
                factors[threadIdx.x] = fp8_factor(m);
                if (bx * 128 + threadIdx.x < p.cols) p.out.scale_t[(bx * 128 + threadIdx.x) * p.out.ld_st + by] = fp8_scale(m);
            }
        }
    } else {
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) all = fmaxf(all, __shfl_xor_sync(0xFFFFFFFFu, all, d));
        if (lane == 0) tops[0][warp] = all;
        __syncthreads();
        all = tops[0][0];
#pragma unroll
        for (int w = 1; w < 8; w++) all = fmaxf(all, tops[0][w]);
        if (threadIdx.x == 0) p.out.scale[by * p.out.ld_s + bx] = fp8_scale(all);
        row_factor = fp8_factor(all);
    }

    if (p.out.q) {
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const float f = SQUARE ? row_factor : __shfl_sync(0xFFFFFFFFu, row_factor, i, 4);
            float v[16];
#pragma unroll
            for (int e = 0; e < 16; e++) v[e] = x[i][e];
            const uint4 codes = fp8_codes(v, f, false);
            if (row0 + i < p.rows && col0 < p.cols) *reinterpret_cast<uint4 *>(p.out.q + (row0 + i) * p.out.ld_q + col0) = codes;
        }
    }
    if (!p.out.q_t) return;
    if (!SQUARE) __syncthreads();   // factors
    uint32_t *words = reinterpret_cast<uint32_t *>(stage);
#pragma unroll
    for (int e0 = 0; e0 < 16; e0 += 4) {
        float4 f = make_float4(row_factor, row_factor, row_factor, row_factor);
        if (!SQUARE) f = *reinterpret_cast<const float4 *>(factors + 16 * cg + e0);
        const float fs[4] = {f.x, f.y, f.z, f.w};
#pragma unroll
        for (int j = 0; j < 4; j++)
            words[(16 * cg + e0 + j) * 32 + ((warp ^ cg) << 2) + rg] =
                cvt_rn_e4m3x4(x[3][e0 + j] * fs[j], x[2][e0 + j] * fs[j], x[1][e0 + j] * fs[j], x[0][e0 + j] * fs[j]);
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 4; k++) {
        const int col = (threadIdx.x >> 3) + 32 * k, piece = threadIdx.x & 7;
        const uint4 v = stage[col * 8 + (piece ^ (col >> 4))];
        if (bx * 128 + col < p.cols && by * 128 + piece * 16 < p.rows)
            *reinterpret_cast<uint4 *>(p.out.q_t + (bx * 128 + col) * p.out.ld_t + by * 128 + piece * 16) = v;
    }
}

template <typename T, bool SQUARE>
fp4q_status launch(const Fp8QuantParams &p, bool grid16, dim3 grid, cudaStream_t s)
{
    return launched(grid16 ? launch_dependent(fp8_quantize_kernel<T, SQUARE, true>, grid, 256, s, p) : launch_dependent(fp8_quantize_kernel<T, SQUARE, false>, grid, 256, s, p));
}

}  // namespace

extern "C" fp4q_status fp4q_fp8_quantize(const void *x, fp4q_out x_type, int64_t rows, int64_t cols, int64_t ld_x, const fp4q_fp8_tensor *out, void *stream)
{
    if (!out) return FP4Q_ERR_NULL;
    if (rows < 0 || cols < 0 || out->rows != rows || out->cols != cols) return FP4Q_ERR_SHAPE;
    if (x_type != FP4Q_OUT_BF16 && x_type != FP4Q_OUT_F32) return FP4Q_ERR_UNSUPPORTED;
    if (out->square != 0 && out->square != 1) return FP4Q_ERR_UNSUPPORTED;
    if (rows == 0 || cols == 0) return FP4Q_OK;
    if (!x || (!out->q && !out->q_t)) return FP4Q_ERR_NULL;
    const bool square = out->square != 0;
    if ((out->q || square) && !out->scale) return FP4Q_ERR_NULL;
    if (out->q_t && !square && !out->scale_t) return FP4Q_ERR_NULL;
    if (ld_x < cols) return FP4Q_ERR_SHAPE;
    if (out->q && out->ld_q < cols) return FP4Q_ERR_SHAPE;
    if ((out->q || square) && out->ld_s < ceil_div(cols, 128)) return FP4Q_ERR_SHAPE;
    if (out->q_t && (out->ld_t < rows || (!square && out->ld_st < ceil_div(rows, 128)))) return FP4Q_ERR_SHAPE;
    if (!aligned(x, x_type == FP4Q_OUT_F32 ? 4 : 2) || !aligned(out->q, 16) || !aligned(out->q_t, 16) || (out->q && out->ld_q % 16 != 0) || (out->q_t && out->ld_t % 16 != 0) ||
        !aligned(out->scale, 4) || !aligned(out->scale_t, 4))
        return FP4Q_ERR_ALIGN;
    Fp8QuantParams p;
    p.rows = rows;
    p.cols = cols;
    p.b16 = rows_of<__nv_bfloat16>(x, ld_x);
    p.f32 = rows_of<float>(x, ld_x);
    p.out = *out;
    p.col_tiles = ceil_div(cols, 128);
    const int64_t tiles = p.col_tiles * ceil_div(rows, 128);
    if (tiles > 0x7FFFFFFF) return FP4Q_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)tiles);
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const bool grid16 = on_grid(x, ld_x, rows, x_type == FP4Q_OUT_F32 ? 4 : 2);
    if (x_type == FP4Q_OUT_F32) return square ? launch<float, true>(p, grid16, grid, s) : launch<float, false>(p, grid16, grid, s);
    return square ? launch<__nv_bfloat16, true>(p, grid16, grid, s) : launch<__nv_bfloat16, false>(p, grid16, grid, s);
}
