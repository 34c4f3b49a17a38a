// fp4q_rms_norm and its backward pass (include/fp4q.h): the norm in front of a projection, with the residual's addition before it and the projection's
// 8-bit operand behind it.
//
// A row belongs to a team of threads, each with 16 consecutive columns at a time (one 32-byte piece of BF16), which stay in registers from the row's
// only reading on: the sum of squares goes through shuffles and, for teams of several warps, shared memory; blocks of 32 or 128 elements are 2 or 8 lanes, so
// their maxima need shuffles alone.  Bound by memory: 16384 x 4096, BF16, with a residual, BF16 and 8-bit outputs 606 MB in 101 us, 6.0 TB/s; its backward pass 537 MB in 100 us.
#include "common.cuh"
#include "fp8_format.cuh"
#include "row_io.cuh"
#include "tensor_map.cuh"

#include <algorithm>
#include <atomic>
#include <type_traits>

using namespace fp4q;

namespace {

// The FP32 or BF16 weight, and E of its elements.
struct WeightOf {
    const void *p;
    int32_t bf16;
    RowsOf<float> f;
    RowsOf<__nv_bfloat16> b;
    template <bool GRID, int E>
    __device__ __forceinline__ void load(int64_t c0, int n, float (&w)[E]) const
    {
        if (!p) {
#pragma unroll
            for (int e = 0; e < E; e++) w[e] = 1.f;
        } else if (bf16) {
            const Raw<__nv_bfloat16, E> r = load_row<__nv_bfloat16, GRID, E>(b, 0, c0, n);
#pragma unroll
            for (int e = 0; e < E; e++) w[e] = r[e];
        } else {
            const Raw<float, E> r = load_row<float, GRID, E>(f, 0, c0, n);
#pragma unroll
            for (int e = 0; e < E; e++) w[e] = r[e];
        }
    }
};
WeightOf weight_of(const void *p, fp4q_out type, int64_t cols)
{
    WeightOf w;
    w.p = p;
    w.bf16 = type == FP4Q_OUT_BF16;
    w.f = rows_of<float>(p, cols);
    w.b = rows_of<__nv_bfloat16>(p, cols);
    return w;
}

// How a row is dealt to threads: `team` of them (a power of two up to 32, else whole warps), `chunks` times 16 columns each, backward 8.  A CTA has one team or, of small ones, several.
struct Deal {
    int team, threads, chunks;
    // segments: of a lane's columns, 16 or, backward, 8
    Deal(int64_t segments, bool backward)
    {
        chunks = segments <= 512 ? 1 : segments <= 1024 ? 2 : !backward || segments <= 2048 ? 4 : 16;
        const int64_t t = ceil_div(segments, chunks);
        team = 1;
        while (team < t && team < 32) team *= 2;
        if (t > 32) team = (int)round_up(t, 32);
        threads = team > 32 ? team * (int)std::max<int64_t>(1, 256 / team) : 256;
    }
};

// Where a thread works: the teams of its CTA, its own, and its place in that.
struct Place {
    int teams, team, in;
    __device__ __forceinline__ explicit Place(int size)
    {
        if (size <= 32) {   // a power of two
            const int bits = __ffs(size) - 1;
            teams = blockDim.x >> bits;
            team = threadIdx.x >> bits;
            in = threadIdx.x & (size - 1);
        } else {
            teams = (int)blockDim.x / size;
            team = teams == 1 ? 0 : (int)threadIdx.x / size;
            in = threadIdx.x - team * size;
        }
    }
};

// Sum over a team.  red: two rows of 32 floats; with teams of several warps the CTA passes one barrier.
__device__ __forceinline__ float team_sum(float v, int size, const Place &at, float (*red)[32], int which)
{
    for (int d = min(size, 32) >> 1; d > 0; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
    if (size <= 32) return v;
    const int lane = threadIdx.x & 31, warps = size >> 5;
    if (lane == 0) red[which][threadIdx.x >> 5] = v;
    __syncthreads();
    v = lane < warps ? red[which][at.team * warps + lane] : 0.f;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
    return v;
}

struct NormParams {
    int64_t rows, cols;
    int32_t team, format;
    float eps, inv_cols;
    const void *residual;
    RowsOf<__nv_bfloat16> xb, rb, hb, yb;
    RowsOf<float> xf, rf, hf, yf;
    WeightOf weight;
    int32_t y_f32;
    uint8_t *q;
    int64_t ld_q;
    void *scale;
    int64_t ld_s;
    float *rstd;
};
template <typename T>
__device__ __forceinline__ const RowsOf<T> &either(const RowsOf<__nv_bfloat16> &b, const RowsOf<float> &f)
{
    if constexpr (sizeof(T) == 4) return f;
    else return b;
}

// Codes and scale of 16 elements where a block holds infinities (or, MXFP8, NaN): maxima of finite elements only.  Whole warps come here.
__device__ __forceinline__ uint4 careful_codes(float (&v)[16], int lanes, bool mx, float &scale)
{
    float top = 0.f;
#pragma unroll
    for (int e = 0; e < 16; e++) top = fmaxf(top, finite_size(v[e]));
    for (int d = lanes >> 1; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
    if (!mx) {
        scale = fp8_scale(top);
        return fp8_codes(v, fp8_factor(top), true);
    }
#pragma unroll
    for (int e = 0; e < 16; e++) v[e] = v[e] == v[e] ? v[e] : 0.f;   // as the MXFP8 quantizers: NaN becomes 0, infinities the largest number
    const int code = mx_scale_code(top);
    scale = __int_as_float(code);
    return fp8_codes(v, inv_scale(code), false);
}

// A stream of BF16 on BF16 is added two elements at a time: the FP32 sum of two BF16 numbers is exact, or so far from a tie that it is rounded like the exact one.
template <typename TX, typename TH>
__device__ __forceinline__ void add_rows(const Raw<TX> &x, Raw<TH> &r)
{
    if constexpr (sizeof(TX) == 2 && sizeof(TH) == 2) {
#pragma unroll
        for (int k = 0; k < 8; k++) {
            const __nv_bfloat162 s = __hadd2(*reinterpret_cast<const __nv_bfloat162 *>(&x.w[k]), *reinterpret_cast<const __nv_bfloat162 *>(&r.w[k]));
            r.w[k] = *reinterpret_cast<const uint32_t *>(&s);
        }
    } else {
        float v[16];
#pragma unroll
        for (int e = 0; e < 16; e++) v[e] = x[e] + r[e];
        r.set(v);
    }
}

// Rows blockIdx.x, blockIdx.x + gridDim.x, ... of teams.  Up to 8192 columns (one chunk a thread) the weight stays in registers and the next row is on its way while this one is worked
// on.  Without a residual TX is TH.  GRID_IN, GRID_OUT: the rows of all that is read, or written, begin on 16 bytes.
template <typename TX, typename TH, int CHUNKS, bool GRID_IN, bool GRID_OUT>
__global__ void __launch_bounds__(CHUNKS == 4 ? 1024 : 512) rms_norm_kernel(const __grid_constant__ NormParams p)
{
    wait_for_predecessor();
    admit_successor();
    __shared__ float red[2][32];
    const int team = p.team, lanes = min(team, 32);
    const Place at(team);
    const int64_t cols = p.cols, step = (int64_t)gridDim.x * at.teams;
    constexpr bool kAhead = CHUNKS == 1;
    auto col_of = [&](int c) { return ((int64_t)c * team + at.in) * 16; };
    int all[CHUNKS];   // columns that exist
    float w[kAhead ? CHUNKS : 1][16];
#pragma unroll
    for (int c = 0; c < CHUNKS; c++) {
        all[c] = columns_at(col_of(c), cols);
        if (kAhead) p.weight.load<GRID_IN, 16>(col_of(c), all[c], w[kAhead ? c : 0]);
    }
    constexpr bool kSame = sizeof(TX) == sizeof(TH);
    Pieces<TX, GRID_IN> x[CHUNKS];
    Pieces<TH, GRID_IN> r[CHUNKS];
    auto load = [&](int64_t row) {
        const int64_t i = row < p.rows ? row : 0;
#pragma unroll
        for (int c = 0; c < CHUNKS; c++) {
            const int m = row < p.rows ? all[c] : 0;
            if (p.residual) {
                r[c].fetch(either<TH>(p.rb, p.rf), i, col_of(c), m);
                x[c].fetch(either<TX>(p.xb, p.xf), i, col_of(c), m);
            } else if (kSame) {
                x[c].fetch(either<TX>(p.xb, p.xf), i, col_of(c), m);
            }
        }
    };
    int64_t first = (int64_t)blockIdx.x * at.teams;
    if (kAhead) load(first + at.team);
    for (int which = 0; first < p.rows; first += step, which ^= 1) {
        const int64_t row = first + at.team;
        if (!kAhead) load(row);
        const bool exists = row < p.rows;
        const int64_t i = exists ? row : 0;
        int n[CHUNKS];
        Raw<TH> h[CHUNKS];   // as it is rounded: what the backward pass reads
#pragma unroll
        for (int c = 0; c < CHUNKS; c++) {
            n[c] = exists ? all[c] : 0;
            const Raw<TX> in = x[c].land(either<TX>(p.xb, p.xf), i, col_of(c), n[c]);
            if (p.residual) {
                h[c] = r[c].land(either<TH>(p.rb, p.rf), i, col_of(c), n[c]);
                add_rows<TX, TH>(in, h[c]);
            } else if constexpr (kSame) {
                h[c] = in;
            }
        }
        if (kAhead && first + step < p.rows) load(row + step);
        float squares = 0.f;
#pragma unroll
        for (int c = 0; c < CHUNKS; c++) {
            if (p.residual) store_row<TH, GRID_OUT>(either<TH>(p.hb, p.hf), i, col_of(c), n[c], h[c], lanes);
#pragma unroll
            for (int e = 0; e < 16; e++) squares = fmaf(h[c][e], h[c][e], squares);
        }
        const float mean = team_sum(squares, team, at, red, which) * p.inv_cols, rstd = __frcp_rn(__fsqrt_rn(mean + p.eps));
        if (p.rstd && exists && at.in == 0) p.rstd[row] = rstd;

#pragma unroll
        for (int c = 0; c < CHUNKS; c++) {
            const int col = (int)col_of(c);
            float v[16];
            if (!kAhead) p.weight.load<GRID_IN, 16>(col, n[c], w[0]);
#pragma unroll
            for (int e = 0; e < 16; e++) v[e] = __fmul_rn(__fmul_rn(h[c][e], rstd), w[kAhead ? c : 0][e]);
            if (p.yb.p && !p.y_f32) {
                Raw<__nv_bfloat16> y;
                y.set(v);
                store_row<__nv_bfloat16, GRID_OUT>(p.yb, i, col, n[c], y, lanes);
            } else if (p.yf.p) {
                Raw<float> y;
                y.set(v);
                store_row<float, GRID_OUT>(p.yf, i, col, n[c], y, lanes);
            }
            if (p.format == 0) continue;
            if (n[c] < 16) {   // what is behind the row's end: its codes are 0
#pragma unroll
                for (int e = 0; e < 16; e++)
                    if (e >= n[c]) v[e] = 0.f;
            }
            float top = 0.f;   // infinity where there is one; NaN does not count
#pragma unroll
            for (int e = 0; e < 16; e++) top = fmaxf(top, fabsf(v[e]));
            const bool mx = p.format == FP4Q_NORM_MXFP8;
            bool odd = is_infinite(top);
            if (mx) {
#pragma unroll
                for (int e = 0; e < 16; e++) odd |= v[e] != v[e];
            }
            const int block = mx ? min(team, 2) : min(team, 8);   // lanes of a block
            float scale;
            uint4 codes;
            if (__any_sync(0xFFFFFFFFu, odd)) {
                codes = careful_codes(v, block, mx, scale);
            } else {
                for (int d = block >> 1; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
                const int code = mx ? mx_scale_code(top) : 0;
                scale = mx ? __int_as_float(code) : top;
                codes = fp8_codes(v, mx ? inv_scale(code) : fp8_factor(top), false);
                if (!mx && col % 128 == 0) scale = fp8_scale(top);
            }
            if (!exists || col >= (mx ? ((int)cols + 31) / 32 * 32 : (int)cols)) continue;
            *reinterpret_cast<uint4 *>(p.q + row * p.ld_q + col) = codes;
            if (mx) {
                if (col % 32 == 0) static_cast<uint8_t *>(p.scale)[row * p.ld_s + col / 32] = (uint8_t)__float_as_int(scale);
            } else if (col % 128 == 0) {
                static_cast<float *>(p.scale)[row * p.ld_s + col / 128] = scale;
            }
        }
    }
}

// ---------------------------------------------------------------------------------------- backward

constexpr int kGradCtas = 592;          // most CTAs of a kernel that sums over rows: four an SM
constexpr int64_t kGradFused = 8192;    // columns up to which that is the kernel of dx too

// From a CTA's sums to the next one's: whole 32 bytes.
__host__ __device__ constexpr int64_t partial_pitch(int64_t cols) { return (cols + 7) / 8 * 8; }

struct GradParams {
    int64_t rows, cols;
    int32_t team;
    float inv_cols;
    const void *dh;
    RowsOf<__nv_bfloat16> dyb, hb, dhb, dxb;
    RowsOf<float> dyf, hf, dhf, dxf;
    const float *rstd;
    WeightOf weight;
    float *partial;          // [CTA][partial_pitch]: sums over its rows; NULL: none
};

// Rows blockIdx.x, blockIdx.x + gridDim.x, ... of teams, 8 columns a lane and chunk.  Up to 8192 columns the weight and the sums over rows stay in registers, and the next row is on its way
// while this one is worked on.  The operations of dx are spelled out, so that it is the same whatever else is computed.
template <typename TY, typename TH, int CHUNKS, bool GRID_IN, bool GRID_OUT, int MOST = 512>
__global__ void __launch_bounds__(MOST, CHUNKS == 1 && (sizeof(TH) == 2 || MOST < 512) ? 2 : 1) rms_norm_bwd_kernel(const __grid_constant__ GradParams p)
{
    wait_for_predecessor();
    admit_successor();
    constexpr int E = 8;
    constexpr bool kHold = CHUNKS <= 2;
    __shared__ float red[2][32];
    __shared__ float sums[kHold ? 256 * E : 1];   // of the teams of a CTA of 256 threads
    const int team = p.team, lanes = min(team, 32);
    const Place at(team);
    const int64_t cols = p.cols;
    auto col_of = [&](int c) { return ((int64_t)c * team + at.in) * E; };
    int n[CHUNKS];
    float dw[kHold ? CHUNKS : 1][E], w[kHold ? CHUNKS : 1][E];
#pragma unroll
    for (int c = 0; c < CHUNKS; c++) {
        n[c] = columns_at<E>(col_of(c), cols);
        if (kHold) {
            p.weight.load<GRID_IN, E>(col_of(c), n[c], w[kHold ? c : 0]);
#pragma unroll
            for (int e = 0; e < E; e++) dw[kHold ? c : 0][e] = 0.f;
        }
    }
    struct Row {
        Pieces<TY, GRID_IN, E> dy[CHUNKS];
        Pieces<TH, GRID_IN, E> h[CHUNKS], dh[CHUNKS];
        float r;
    };
    auto load = [&](Row &to, int64_t row) {
        const bool exists = row < p.rows;
        const int64_t i = exists ? row : 0;
#pragma unroll
        for (int c = 0; c < CHUNKS; c++) {
            const int m = exists ? n[c] : 0;
            to.dy[c].fetch(either<TY>(p.dyb, p.dyf), i, col_of(c), m);
            to.h[c].fetch(either<TH>(p.hb, p.hf), i, col_of(c), m);
            if (p.dh) to.dh[c].fetch(either<TH>(p.dhb, p.dhf), i, col_of(c), m);
        }
        to.r = exists ? load_global(p.rstd + i) : 0.f;
    };
    int64_t first = (int64_t)blockIdx.x * at.teams;
    const int64_t step = (int64_t)gridDim.x * at.teams;
    Row next;
    if (kHold && first < p.rows) load(next, first + at.team);
    for (int which = 0; first < p.rows; first += step, which ^= 1) {
        const int64_t row = first + at.team;
        const bool exists = row < p.rows;
        const int64_t i = exists ? row : 0;
        if (!kHold) load(next, row);
        Raw<TY, E> dy[CHUNKS];
        Raw<TH, E> h[CHUNKS], dh[CHUNKS];
        const float r = next.r;
#pragma unroll
        for (int c = 0; c < CHUNKS; c++) {
            const int m = exists ? n[c] : 0;
            dy[c] = next.dy[c].land(either<TY>(p.dyb, p.dyf), i, col_of(c), m);
            h[c] = next.h[c].land(either<TH>(p.hb, p.hf), i, col_of(c), m);
            if (p.dh) dh[c] = next.dh[c].land(either<TH>(p.dhb, p.dhf), i, col_of(c), m);
        }
        if (kHold && first + step < p.rows) load(next, row + step);
        float dot = 0.f;
#pragma unroll
        for (int c = 0; c < CHUNKS; c++) {
            const int k = kHold ? c : 0;
            if (!kHold) p.weight.load<GRID_IN, E>(col_of(c), n[c], w[0]);
#pragma unroll
            for (int e = 0; e < E; e++) {
                const float x = __fmul_rn(h[c][e], r);
                dot = fmaf(__fmul_rn(dy[c][e], w[k][e]), x, dot);
                if (kHold) dw[k][e] = fmaf(dy[c][e], x, dw[k][e]);   // rows that do not exist are zeros
            }
        }
        const float mean = team_sum(dot, team, at, red, which) * p.inv_cols;
#pragma unroll
        for (int c = 0; c < CHUNKS; c++) {
            const int k = kHold ? c : 0;
            float v[E];
            if (!kHold) p.weight.load<GRID_IN, E>(col_of(c), n[c], w[0]);
#pragma unroll
            for (int e = 0; e < E; e++) {
                v[e] = __fmul_rn(r, fmaf(-__fmul_rn(h[c][e], r), mean, __fmul_rn(dy[c][e], w[k][e])));
                if (p.dh) v[e] = __fadd_rn(v[e], dh[c][e]);
            }
            Raw<TH, E> dx;
            dx.set(v);
            store_row<TH, GRID_OUT, E>(either<TH>(p.dxb, p.dxf), i, col_of(c), exists ? n[c] : 0, dx, lanes);
        }
    }
    if (!kHold || !p.partial) return;
    float *to = p.partial + (int64_t)blockIdx.x * partial_pitch(cols);
    if (at.teams == 1) {
#pragma unroll
        for (int c = 0; c < CHUNKS; c++) {
            const float *d = dw[kHold ? c : 0];
            if (n[c] == 0) continue;   // columns that do not exist, up to the pitch, are zeros
            reinterpret_cast<float4 *>(to + col_of(c))[0] = make_float4(d[0], d[1], d[2], d[3]);
            reinterpret_cast<float4 *>(to + col_of(c))[1] = make_float4(d[4], d[5], d[6], d[7]);
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < E; e++) sums[threadIdx.x * E + e] = dw[0][e];
    __syncthreads();
    for (int c = threadIdx.x; c < cols; c += blockDim.x) {
        float v = 0.f;
        for (int k = 0; k < at.teams; k++) v += sums[(k * team + c / E) * E + c % E];
        to[c] = v;
    }
}

// Sums over rows of wide matrices: a CTA has 512 columns (a warp's lane 16 of them) and every gridDim.y-th row.
template <typename TY, typename TH>
__global__ void __launch_bounds__(256) rms_norm_dweight_kernel(const __grid_constant__ GradParams p)
{
    wait_for_predecessor();
    admit_successor();
    __shared__ float sums[8 * 512];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t col = (int64_t)blockIdx.x * 512 + lane * 16;
    const int n = columns_at(col, p.cols);
    float dw[16];
#pragma unroll
    for (int e = 0; e < 16; e++) dw[e] = 0.f;
    for (int64_t i = (int64_t)blockIdx.y * 8 + warp; i < p.rows; i += (int64_t)gridDim.y * 8) {
        const Raw<TY> dy = load_row<TY>(either<TY>(p.dyb, p.dyf), i, col, n);
        const Raw<TH> h = load_row<TH>(either<TH>(p.hb, p.hf), i, col, n);
        const float r = load_global(p.rstd + i);
#pragma unroll
        for (int e = 0; e < 16; e++) dw[e] = fmaf(dy[e], h[e] * r, dw[e]);
    }
#pragma unroll
    for (int e = 0; e < 16; e++) sums[warp * 512 + lane * 16 + e] = dw[e];
    __syncthreads();
    for (int c = threadIdx.x; c < 512; c += 256) {
        float v = 0.f;
#pragma unroll
        for (int k = 0; k < 8; k++) v += sums[k * 512 + c];
        if ((int64_t)blockIdx.x * 512 + c < p.cols) p.partial[(int64_t)blockIdx.y * partial_pitch(p.cols) + (int64_t)blockIdx.x * 512 + c] = v;
    }
}

// dweight (+)= the sum of `parts` rows of partial sums, 32 columns a CTA of 32 warps, which take the rows in turn.
struct SumParams {
    const float *partial;
    int64_t cols;
    int32_t parts, accumulate;
    float *dweight;
};
__global__ void __launch_bounds__(1024) column_sum_kernel(const __grid_constant__ SumParams p)
{
    wait_for_predecessor();
    admit_successor();
    __shared__ float sums[32][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t col = (int64_t)blockIdx.x * 32 + lane;
    float v = 0.f;
    if (col < p.cols)
#pragma unroll 8
        for (int k = warp; k < p.parts; k += 32) v += load_global(p.partial + (int64_t)k * partial_pitch(p.cols) + col);
    sums[warp][lane] = v;
    __syncthreads();
    v = sums[lane][warp];   // a warp has a column
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
    const int64_t mine = (int64_t)blockIdx.x * 32 + warp;
    if (lane == 0 && mine < p.cols) p.dweight[mine] = p.accumulate ? p.dweight[mine] + v : v;
}

bool plain_type(fp4q_out t) { return t == FP4Q_OUT_BF16 || t == FP4Q_OUT_F32; }
size_t size_of(fp4q_out t) { return t == FP4Q_OUT_F32 ? 4 : 2; }
// A matrix that the call reads or writes.
fp4q_status check_matrix(const void *p, int64_t ld, fp4q_out type, int64_t cols)
{
    if (!p) return FP4Q_ERR_NULL;
    if (ld < cols) return FP4Q_ERR_SHAPE;
    return aligned(p, size_of(type)) ? FP4Q_OK : FP4Q_ERR_ALIGN;
}
constexpr int64_t kMostCols = 65536;

// CTAs that an SM has room for, by their registers.  A grid of as many whose CTAs take rows in turn leaves no CTA for later (16384 x 4096: three an SM 102 us, two 128, a row each 165).
template <typename P>
int resident(void (*kernel)(const P), int threads, std::atomic<int> &known)
{
    int regs = known.load(std::memory_order_relaxed);
    if (regs == 0) {
        cudaFuncAttributes a;
        if (cudaFuncGetAttributes(&a, reinterpret_cast<const void *>(kernel)) != cudaSuccess) {
            cudaGetLastError();
            return 1;
        }
        regs = (a.numRegs + 7) / 8 * 8;
        known.store(regs, std::memory_order_relaxed);
    }
    const int warps = 4 * std::min(16, 16384 / (regs * 32));   // of four schedulers
    return std::max(1, warps / (threads / 32));
}

// in, out: the rows of all that is read, or written, begin on 16 bytes.
template <typename TX, typename TH>
fp4q_status launch_norm(const NormParams &p, const Deal &d, bool in, bool out, cudaStream_t s)
{
    const int dev = current_device();
    if (dev < 0) return FP4Q_ERR_CUDA;
    const int64_t sms = sm_count(dev);
    auto launch = [&](auto kernel, std::atomic<int> &known) {
        const int64_t ctas = ceil_div(p.rows, d.threads / d.team);
        const dim3 grid((unsigned)std::min<int64_t>(ctas, sms * resident(kernel, d.threads, known)));
        return launched(launch_dependent(kernel, grid, d.threads, s, p));
    };
    static std::atomic<int> known[5];
    if (d.chunks == 1) return in && out ? launch(rms_norm_kernel<TX, TH, 1, true, true>, known[0]) : out ? launch(rms_norm_kernel<TX, TH, 1, false, true>, known[1]) : launch(rms_norm_kernel<TX, TH, 1, false, false>, known[2]);
    return d.chunks == 2 ? launch(rms_norm_kernel<TX, TH, 2, false, false>, known[3]) : launch(rms_norm_kernel<TX, TH, 4, false, false>, known[4]);
}

template <typename TY, typename TH>
fp4q_status launch_grad(GradParams p, float *dweight, int accumulate, void *scratch, bool in, bool out, cudaStream_t s)
{
    const Deal d(ceil_div(p.cols, 8), true);
    p.team = d.team;
    const bool fused = dweight && p.cols <= kGradFused;
    p.partial = dweight ? static_cast<float *>(scratch) : nullptr;
    const int dev = current_device();
    if (dev < 0) return FP4Q_ERR_CUDA;
    const int64_t sms = sm_count(dev);
    int64_t parts = 1;
    auto launch = [&](auto kernel, std::atomic<int> &known) {
        const int64_t ctas = std::max<int64_t>(1, std::min({(int64_t)kGradCtas, ceil_div(p.rows, d.threads / d.team), sms * resident(kernel, d.threads, known)}));
        if (fused) parts = ctas;
        return launched(launch_dependent(kernel, dim3((unsigned)ctas), d.threads, s, p));
    };
    static std::atomic<int> known[10];
    auto join = [&] {
        const SumParams q = {p.partial, p.cols, (int32_t)parts, accumulate != 0, dweight};
        return launched(launch_dependent(column_sum_kernel, dim3((unsigned)ceil_div(p.cols, 32)), 1024, s, q));
    };
    if (dweight && !fused) {   // before dx, which may overwrite what this reads
        parts = std::max<int64_t>(1, std::min<int64_t>(kGradCtas / 2, ceil_div(p.rows, 8)));
        if (fp4q_status st = launched(launch_dependent(rms_norm_dweight_kernel<TY, TH>, dim3((unsigned)ceil_div(p.cols, 512), (unsigned)parts), 256, s, p))) return st;
        if (fp4q_status st = join()) return st;
    }
    if (fused || p.rows > 0) {
        fp4q_status st;
        auto one = [&](auto most, int at) {   // one chunk a thread
            constexpr int kMost = decltype(most)::value;
            return in && out ? launch(rms_norm_bwd_kernel<TY, TH, 1, true, true, kMost>, known[at])
                   : in      ? launch(rms_norm_bwd_kernel<TY, TH, 1, true, false, kMost>, known[at + 1])
                             : launch(rms_norm_bwd_kernel<TY, TH, 1, false, false, kMost>, known[at + 2]);
        };
        if (d.chunks == 1) {
            // On an FP32 stream registers for 384 threads let two CTAs of 256 to 384 threads run on an SM where those for 512 leave room for one, and three of 256 instead of two.  The more CTAs,
            // the more sums there are to join: few elements in CTAs of 256 are better off without.  8192 x 3000 51 us for 67, 1999 x 2731 18.0 for 20.9, 300 x 2731 7.3 for 8.6; 256 threads: 8192 x
            // 2048 35 for 38, 16384 x 1000 37 for 40, but 1999 x 2048 12.9 for 12.5, 1999 x 512 7.8 for 6.7, 8192 x 512 12.7 for 12.1.
            if constexpr (sizeof(TH) == 4)
                st = d.threads <= 384 && (d.threads > 256 || p.rows * p.cols >= 1 << 23) ? one(std::integral_constant<int, 384>(), 5) : one(std::integral_constant<int, 512>(), 0);
            else st = one(std::integral_constant<int, 512>(), 0);
        } else {
            st = d.chunks == 2 ? in && out ? launch(rms_norm_bwd_kernel<TY, TH, 2, true, true>, known[3]) : launch(rms_norm_bwd_kernel<TY, TH, 2, false, false>, known[4])
                 : d.chunks == 4 ? launch(rms_norm_bwd_kernel<TY, TH, 4, false, false>, known[8])
                                 : launch(rms_norm_bwd_kernel<TY, TH, 16, false, false>, known[9]);
        }
        if (st) return st;
    }
    return fused ? join() : FP4Q_OK;
}

}  // namespace

extern "C" fp4q_status fp4q_rms_norm(const fp4q_norm *n, int64_t rows, int64_t cols, void *stream)
{
    if (!n) return FP4Q_ERR_NULL;
    if (rows < 0 || cols < 0) return FP4Q_ERR_SHAPE;
    if (!plain_type(n->x_type) || (n->residual && !plain_type(n->h_type)) || (n->weight && !plain_type(n->weight_type)) || (n->y && !plain_type(n->y_type))) return FP4Q_ERR_UNSUPPORTED;
    if (n->q && n->q_format != FP4Q_NORM_MXFP8 && n->q_format != FP4Q_NORM_FP8) return FP4Q_ERR_UNSUPPORTED;
    if (!(n->eps >= 0.f) || cols > kMostCols) return FP4Q_ERR_UNSUPPORTED;
    if (rows == 0 || cols == 0) return FP4Q_OK;
    if (fp4q_status s = check_matrix(n->x, n->ld_x, n->x_type, cols)) return s;
    if (n->residual) {
        if (fp4q_status s = check_matrix(n->residual, n->ld_residual, n->h_type, cols)) return s;
        if (fp4q_status s = check_matrix(n->h, n->ld_h, n->h_type, cols)) return s;
    }
    if (n->weight && !aligned(n->weight, size_of(n->weight_type))) return FP4Q_ERR_ALIGN;
    if (n->y) {
        if (fp4q_status s = check_matrix(n->y, n->ld_y, n->y_type, cols)) return s;
    }
    const bool mx = n->q && n->q_format == FP4Q_NORM_MXFP8;
    if (n->q) {
        if (!n->scale) return FP4Q_ERR_NULL;
        if (n->ld_q < (mx ? round_up(cols, 32) : cols) || n->ld_s < ceil_div(cols, mx ? 32 : 128)) return FP4Q_ERR_SHAPE;
        if (!aligned(n->q, 16) || n->ld_q % 16 != 0 || (!mx && !aligned(n->scale, 4))) return FP4Q_ERR_ALIGN;
    }
    if (!aligned(n->rstd, 4)) return FP4Q_ERR_ALIGN;
    const Deal d(ceil_div(mx ? round_up(cols, 32) : cols, 16), false);
    NormParams p = {};
    p.rows = rows;
    p.cols = cols;
    p.team = d.team;
    p.format = n->q ? n->q_format : 0;
    p.eps = n->eps;
    p.inv_cols = 1.f / (float)cols;
    p.residual = n->residual;
    p.xb = rows_of<__nv_bfloat16>(n->x, n->ld_x);
    p.xf = rows_of<float>(n->x, n->ld_x);
    if (n->residual) {
        p.rb = rows_of<__nv_bfloat16>(n->residual, n->ld_residual);
        p.rf = rows_of<float>(n->residual, n->ld_residual);
        p.hb = rows_of<__nv_bfloat16>(n->h, n->ld_h);
        p.hf = rows_of<float>(n->h, n->ld_h);
    }
    p.yb = rows_of<__nv_bfloat16>(n->y, n->ld_y);
    p.yf = rows_of<float>(n->y, n->ld_y);
    p.y_f32 = n->y_type == FP4Q_OUT_F32;
    p.weight = weight_of(n->weight, n->weight_type, cols);
    p.q = n->q;
    p.ld_q = n->ld_q;
    p.scale = n->scale;
    p.ld_s = n->ld_s;
    p.rstd = n->rstd;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const bool x32 = n->x_type == FP4Q_OUT_F32, h32 = n->residual ? n->h_type == FP4Q_OUT_F32 : x32;
    const size_t xs = size_of(n->x_type), hs = size_of(n->h_type);
    const bool in = on_grid(n->x, n->ld_x, rows, xs) && on_grid(n->residual, n->ld_residual, rows, hs) && aligned(n->weight, 16);
    const bool out = (!n->residual || on_grid(n->h, n->ld_h, rows, hs)) && on_grid(n->y, n->ld_y, rows, size_of(n->y_type));
    if (x32) return h32 ? launch_norm<float, float>(p, d, in, out, s) : launch_norm<float, __nv_bfloat16>(p, d, in, out, s);
    return h32 ? launch_norm<__nv_bfloat16, float>(p, d, in, out, s) : launch_norm<__nv_bfloat16, __nv_bfloat16>(p, d, in, out, s);
}

extern "C" size_t fp4q_rms_norm_bwd_scratch_bytes(int64_t rows, int64_t cols)
{
    if (rows < 0 || cols <= 0 || cols > kMostCols) return 0;
    return (size_t)round_up(std::max<int64_t>(1, std::min<int64_t>(kGradCtas, rows)) * partial_pitch(cols) * 4, 256);
}

extern "C" fp4q_status fp4q_rms_norm_bwd(const fp4q_norm_grad *n, int64_t rows, int64_t cols, void *scratch, size_t scratch_bytes, void *stream)
{
    if (!n) return FP4Q_ERR_NULL;
    if (rows < 0 || cols < 0) return FP4Q_ERR_SHAPE;
    if (!plain_type(n->dy_type) || !plain_type(n->h_type) || (n->weight && !plain_type(n->weight_type)) || cols > kMostCols) return FP4Q_ERR_UNSUPPORTED;
    if (cols == 0 || (rows == 0 && !n->dweight)) return FP4Q_OK;
    if (rows > 0) {
        if (fp4q_status s = check_matrix(n->dy, n->ld_dy, n->dy_type, cols)) return s;
        if (fp4q_status s = check_matrix(n->h, n->ld_h, n->h_type, cols)) return s;
        if (fp4q_status s = check_matrix(n->dx, n->ld_dx, n->h_type, cols)) return s;
        if (n->dh) {
            if (fp4q_status s = check_matrix(n->dh, n->ld_dh, n->h_type, cols)) return s;
        }
        if (!n->rstd) return FP4Q_ERR_NULL;
        if (!aligned(n->rstd, 4)) return FP4Q_ERR_ALIGN;
    }
    if ((n->weight && !aligned(n->weight, size_of(n->weight_type))) || !aligned(n->dweight, 4)) return FP4Q_ERR_ALIGN;
    if (n->dweight) {
        if (!scratch || scratch_bytes < fp4q_rms_norm_bwd_scratch_bytes(rows, cols)) return FP4Q_ERR_WORKSPACE;
        if (!aligned(scratch, 256)) return FP4Q_ERR_ALIGN;
    }
    if (rows > 0x7FFFFFFF) return FP4Q_ERR_UNSUPPORTED;
    GradParams p = {};
    p.rows = rows;
    p.cols = cols;
    p.inv_cols = 1.f / (float)cols;
    p.dh = n->dh;
    p.dyb = rows_of<__nv_bfloat16>(n->dy, n->ld_dy);
    p.dyf = rows_of<float>(n->dy, n->ld_dy);
    p.hb = rows_of<__nv_bfloat16>(n->h, n->ld_h);
    p.hf = rows_of<float>(n->h, n->ld_h);
    p.dhb = rows_of<__nv_bfloat16>(n->dh, n->ld_dh);
    p.dhf = rows_of<float>(n->dh, n->ld_dh);
    p.dxb = rows_of<__nv_bfloat16>(n->dx, n->ld_dx);
    p.dxf = rows_of<float>(n->dx, n->ld_dx);
    p.rstd = n->rstd;
    p.weight = weight_of(n->weight, n->weight_type, cols);
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const bool y32 = n->dy_type == FP4Q_OUT_F32, h32 = n->h_type == FP4Q_OUT_F32;
    const size_t hs = size_of(n->h_type);
    const bool in = on_grid(n->dy, n->ld_dy, rows, size_of(n->dy_type)) && on_grid(n->h, n->ld_h, rows, hs) && on_grid(n->dh, n->ld_dh, rows, hs) && aligned(n->weight, 16);
    const bool out = on_grid(n->dx, n->ld_dx, rows, hs);
    if (y32) return h32 ? launch_grad<float, float>(p, n->dweight, n->accumulate, scratch, in, out, s) : launch_grad<float, __nv_bfloat16>(p, n->dweight, n->accumulate, scratch, in, out, s);
    return h32 ? launch_grad<__nv_bfloat16, float>(p, n->dweight, n->accumulate, scratch, in, out, s)
               : launch_grad<__nv_bfloat16, __nv_bfloat16>(p, n->dweight, n->accumulate, scratch, in, out, s);
}
