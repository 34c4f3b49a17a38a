// fp4q_rms_norm and its backward pass (include/fp4q.h): the norm in front of a projection, with the residual's addition before it and the projection's
// 8-bit operand behind it.
//
// A row belongs to a team of threads, each with 16 consecutive columns at a time (one 32-byte piece of BF16), which stay in registers from the row's
// only reading on: the sum of squares goes through shuffles and, for teams of several warps, shared memory; blocks of 32 or 128 elements are 2 or 8 lanes, so
// their maxima need shuffles alone.  Bound by memory; rows of up to 512 columns share a CTA.
#include "common.cuh"
#include "fp8_format.cuh"
#include "row_io.cuh"

#include <algorithm>

using namespace fp4q;

namespace {

// The FP32 or BF16 weight, 16 of its elements.
struct WeightOf {
    const void *p;
    int32_t bf16;
    RowsOf<float> f;
    RowsOf<__nv_bfloat16> b;
    template <bool FAST = false>
    __device__ __forceinline__ void load(int64_t c0, int n, float (&w)[16]) const
    {
        if (!p) {
#pragma unroll
            for (int e = 0; e < 16; e++) w[e] = 1.f;
        } else if (bf16) {
            const Raw16<__nv_bfloat16> r = load_row16<__nv_bfloat16, FAST>(b, 0, c0, n);
#pragma unroll
            for (int e = 0; e < 16; e++) w[e] = r[e];
        } else {
            const Raw16<float> r = load_row16<float, FAST>(f, 0, c0, n);
#pragma unroll
            for (int e = 0; e < 16; e++) w[e] = r[e];
        }
    }
};
WeightOf weight_of(const void *p, fp4q_out type, int64_t cols)
{
    WeightOf w;
    w.p = p;
    w.bf16 = type == FP4Q_OUT_BF16;
    w.f = rows_of<float>(p, 1, cols, cols);
    w.b = rows_of<__nv_bfloat16>(p, 1, cols, cols);
    return w;
}

// How a row is dealt to threads: `team` of them (a power of two up to 32, else whole warps and all of the CTA's), `chunks` times 16 columns each.
struct Deal {
    int team, threads, chunks;
    explicit Deal(int64_t segments)
    {
        chunks = segments <= 512 ? 1 : segments <= 1024 ? 2 : 4;
        const int64_t t = ceil_div(segments, chunks);
        team = 1;
        while (team < t && team < 32) team *= 2;
        if (t > 32) team = (int)round_up(t, 32);
        threads = team > 32 ? team : 256;
    }
};

// Sum over a team.  red: two rows of 32 floats; a team of several warps is the CTA and passes one barrier.
__device__ __forceinline__ float team_sum(float v, int team, float (*red)[32], int which)
{
    for (int d = min(team, 32) >> 1; d > 0; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
    if (team <= 32) return v;
    if ((threadIdx.x & 31) == 0) red[which][threadIdx.x >> 5] = v;
    __syncthreads();
    v = (threadIdx.x & 31) < (team >> 5) ? red[which][threadIdx.x & 31] : 0.f;
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
__device__ __forceinline__ void add_rows(const Raw16<TX> &x, Raw16<TH> &r)
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

// Where a thread works: the teams of its CTA, its own, and its place in that.
struct Place {
    int teams = 1, team = 0, in;
    __device__ __forceinline__ explicit Place(int size)
    {
        in = threadIdx.x;
        if (size <= 32) {   // a power of two
            const int bits = __ffs(size) - 1;
            teams = blockDim.x >> bits;
            team = threadIdx.x >> bits;
            in = threadIdx.x & (size - 1);
        }
    }
};

// Rows blockIdx.x, blockIdx.x + gridDim.x, ... of teams.  Up to 8192 columns (one chunk a thread) the weight stays in registers and the next row is on its way while this one is worked
// on.  Without a residual TX is TH.  FAST: all matrices' rows begin on 16 bytes, and cols is a multiple of 16.
template <typename TX, typename TH, int CHUNKS, bool FAST>
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
        all[c] = columns16(col_of(c), cols);
        if (kAhead) p.weight.load<FAST>(col_of(c), all[c], w[kAhead ? c : 0]);
    }
    Raw16<TX> x[CHUNKS];
    Raw16<TH> r[CHUNKS];
    auto load = [&](int64_t row) {
        const int64_t i = row < p.rows ? row : 0;
#pragma unroll
        for (int c = 0; c < CHUNKS; c++) {
            const int m = row < p.rows ? all[c] : 0;
            if (p.residual) {
                x[c] = load_row16<TX, FAST>(either<TX>(p.xb, p.xf), i, col_of(c), m);
                r[c] = load_row16<TH, FAST>(either<TH>(p.rb, p.rf), i, col_of(c), m);
            } else {
                r[c] = load_row16<TH, FAST>(either<TH>(p.xb, p.xf), i, col_of(c), m);
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
        Raw16<TH> h[CHUNKS];   // as it is rounded: what the backward pass reads
#pragma unroll
        for (int c = 0; c < CHUNKS; c++) {
            n[c] = exists ? all[c] : 0;
            h[c] = r[c];
            if (p.residual) add_rows<TX, TH>(x[c], h[c]);
        }
        if (kAhead && first + step < p.rows) load(row + step);
        float squares = 0.f;
#pragma unroll
        for (int c = 0; c < CHUNKS; c++) {
            if (p.residual) store_row16<TH, FAST>(either<TH>(p.hb, p.hf), i, col_of(c), n[c], h[c], lanes);
#pragma unroll
            for (int e = 0; e < 16; e++) squares = fmaf(h[c][e], h[c][e], squares);
        }
        const float mean = team_sum(squares, team, red, which) * p.inv_cols, rstd = __frcp_rn(__fsqrt_rn(mean + p.eps));
        if (p.rstd && exists && at.in == 0) p.rstd[row] = rstd;

#pragma unroll
        for (int c = 0; c < CHUNKS; c++) {
            const int col = (int)col_of(c);
            float v[16];
            if (!kAhead) p.weight.load<FAST>(col, n[c], w[0]);
#pragma unroll
            for (int e = 0; e < 16; e++) v[e] = __fmul_rn(__fmul_rn(h[c][e], rstd), w[kAhead ? c : 0][e]);
            if (p.yb.p && !p.y_f32) {
                Raw16<__nv_bfloat16> y;
                y.set(v);
                store_row16<__nv_bfloat16, FAST>(p.yb, i, col, n[c], y, lanes);
            } else if (p.yf.p) {
                Raw16<float> y;
                y.set(v);
                store_row16<float, FAST>(p.yf, i, col, n[c], y, lanes);
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
            if (!exists || (FAST && !mx ? n[c] == 0 : col >= (mx ? ((int)cols + 31) / 32 * 32 : (int)cols))) continue;
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

constexpr int kGradCtas = 296;          // of the kernel that sums over rows: two an SM
constexpr int64_t kGradFused = 8192;    // columns up to which that is the kernel of dx too

struct GradParams {
    int64_t rows, cols;
    int32_t team;
    float inv_cols;
    const void *dh;
    RowsOf<__nv_bfloat16> dyb, hb, dhb, dxb;
    RowsOf<float> dyf, hf, dhf, dxf;
    const float *rstd;
    WeightOf weight;
    float *partial;          // [CTA][cols]: sums over its rows; NULL: none
};

// Rows blockIdx.x, blockIdx.x + gridDim.x, ... of teams.  The operations of dx are spelled out, so that it is the same with SUMS and without.  With SUMS a CTA has many rows: the next
// one's elements are on their way while this one's are worked on.
template <typename TY, typename TH, int CHUNKS, bool SUMS, bool FAST>
__global__ void __launch_bounds__(CHUNKS == 4 ? 1024 : 512) rms_norm_bwd_kernel(const __grid_constant__ GradParams p)
{
    wait_for_predecessor();
    admit_successor();
    __shared__ float red[2][32];
    __shared__ float sums[SUMS ? 4096 : 1];   // of the teams of a CTA of 256 threads
    const int team = p.team, lanes = min(team, 32);
    const Place at(team);
    const int teams = at.teams;
    const int64_t cols = p.cols;
    auto col_of = [&](int c) { return ((int64_t)c * team + at.in) * 16; };
    int n[CHUNKS];
#pragma unroll
    for (int c = 0; c < CHUNKS; c++) n[c] = columns16(col_of(c), cols);
    float dw[SUMS ? CHUNKS : 1][16], w[SUMS ? CHUNKS : 1][16];
    if (SUMS) {
#pragma unroll
        for (int c = 0; c < CHUNKS; c++) {
            p.weight.load<FAST>(col_of(c), n[c], w[c]);
#pragma unroll
            for (int e = 0; e < 16; e++) dw[c][e] = 0.f;
        }
    }
    struct Row {
        Raw16<TY> dy[CHUNKS];
        Raw16<TH> h[CHUNKS], dh[CHUNKS];
        float r;
    };
    auto load = [&](Row &to, int64_t row) {
        const bool exists = row < p.rows;
        const int64_t i = exists ? row : 0;
#pragma unroll
        for (int c = 0; c < CHUNKS; c++) {
            const int m = exists ? n[c] : 0;
            to.dy[c] = load_row16<TY, FAST>(either<TY>(p.dyb, p.dyf), i, col_of(c), m);
            to.h[c] = load_row16<TH, FAST>(either<TH>(p.hb, p.hf), i, col_of(c), m);
            if (p.dh) to.dh[c] = load_row16<TH, FAST>(either<TH>(p.dhb, p.dhf), i, col_of(c), m);
        }
        to.r = exists ? load_global(p.rstd + i) : 0.f;
    };
    int which = 0;
    const int64_t mine = (int64_t)blockIdx.x * teams, step = (int64_t)gridDim.x * teams;
    Row next;
    if (SUMS && mine < p.rows) load(next, mine + at.team);
    for (int64_t first = mine; first < p.rows; first += step, which ^= 1) {
        const int64_t row = first + at.team;
        const bool exists = row < p.rows;
        Row now;
        if (SUMS) {
            now = next;
            if (first + step < p.rows) load(next, row + step);
        } else {
            load(now, row);
        }
        float dot = 0.f;
#pragma unroll
        for (int c = 0; c < CHUNKS; c++) {
            float wc[16];
            if (!SUMS) p.weight.load<FAST>(col_of(c), n[c], wc);
#pragma unroll
            for (int e = 0; e < 16; e++) {
                const float x = __fmul_rn(now.h[c][e], now.r);
                dot = fmaf(__fmul_rn(now.dy[c][e], SUMS ? w[SUMS ? c : 0][e] : wc[e]), x, dot);
                if (SUMS) dw[SUMS ? c : 0][e] = fmaf(now.dy[c][e], x, dw[SUMS ? c : 0][e]);   // rows that do not exist are zeros
            }
        }
        const float mean = team_sum(dot, team, red, which) * p.inv_cols;
#pragma unroll
        for (int c = 0; c < CHUNKS; c++) {
            float wc[16], v[16];
            if (!SUMS) p.weight.load<FAST>(col_of(c), n[c], wc);
#pragma unroll
            for (int e = 0; e < 16; e++) {
                const float g = __fmul_rn(now.dy[c][e], SUMS ? w[SUMS ? c : 0][e] : wc[e]);
                v[e] = __fmul_rn(now.r, fmaf(-__fmul_rn(now.h[c][e], now.r), mean, g));
                if (p.dh) v[e] = __fadd_rn(v[e], now.dh[c][e]);
            }
            Raw16<TH> dx;
            dx.set(v);
            store_row16<TH, FAST>(either<TH>(p.dxb, p.dxf), exists ? row : 0, col_of(c), exists ? n[c] : 0, dx, lanes);
        }
    }
    if (!SUMS) return;
    float *to = p.partial + (int64_t)blockIdx.x * cols;
    if (teams == 1) {
#pragma unroll
        for (int c = 0; c < CHUNKS; c++)
#pragma unroll
            for (int e = 0; e < 16; e++)
                if (col_of(c) + e < cols) to[col_of(c) + e] = dw[SUMS ? c : 0][e];
        return;
    }
#pragma unroll
    for (int e = 0; e < 16; e++) sums[threadIdx.x * 16 + e] = dw[0][e];
    __syncthreads();
    for (int c = threadIdx.x; c < cols; c += blockDim.x) {
        float v = 0.f;
        for (int k = 0; k < teams; k++) v += sums[(k * team + (c >> 4)) * 16 + (c & 15)];
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
    const int n = columns16(col, p.cols);
    float dw[16];
#pragma unroll
    for (int e = 0; e < 16; e++) dw[e] = 0.f;
    for (int64_t i = (int64_t)blockIdx.y * 8 + warp; i < p.rows; i += (int64_t)gridDim.y * 8) {
        const Raw16<TY> dy = load_row16<TY>(either<TY>(p.dyb, p.dyf), i, col, n);
        const Raw16<TH> h = load_row16<TH>(either<TH>(p.hb, p.hf), i, col, n);
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
        if ((int64_t)blockIdx.x * 512 + c < p.cols) p.partial[(int64_t)blockIdx.y * p.cols + (int64_t)blockIdx.x * 512 + c] = v;
    }
}

// dweight (+)= the sum of `parts` rows of partial sums, 32 columns a CTA.
struct SumParams {
    const float *partial;
    int64_t cols;
    int32_t parts, accumulate;
    float *dweight;
};
__global__ void __launch_bounds__(256) column_sum_kernel(const __grid_constant__ SumParams p)
{
    wait_for_predecessor();
    admit_successor();
    __shared__ float sums[8][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t col = (int64_t)blockIdx.x * 32 + lane;
    float v = 0.f;
    if (col < p.cols)
#pragma unroll 8
        for (int k = warp; k < p.parts; k += 8) v += load_global(p.partial + (int64_t)k * p.cols + col);
    sums[warp][lane] = v;
    __syncthreads();
    if (warp != 0 || col >= p.cols) return;
    v = 0.f;
#pragma unroll
    for (int k = 0; k < 8; k++) v += sums[k][lane];
    p.dweight[col] = p.accumulate ? p.dweight[col] + v : v;
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
constexpr int kNormThreads = 148 * 2 * 256;   // of a grid whose CTAs take rows in turn: all of them run at once (16384 x 4096 104 us; 4 x 256 an SM 105, one row each 165)

template <typename TX, typename TH>
fp4q_status launch_norm(const NormParams &p, const Deal &d, bool fast, cudaStream_t s)
{
    const int64_t ctas = ceil_div(p.rows, d.threads / d.team);
    const dim3 grid((unsigned)std::min<int64_t>(ctas, kNormThreads / d.threads));
    return launched(d.chunks == 1   ? fast ? launch_dependent(rms_norm_kernel<TX, TH, 1, true>, grid, d.threads, s, p) : launch_dependent(rms_norm_kernel<TX, TH, 1, false>, grid, d.threads, s, p)
                    : d.chunks == 2 ? launch_dependent(rms_norm_kernel<TX, TH, 2, false>, grid, d.threads, s, p)
                                    : launch_dependent(rms_norm_kernel<TX, TH, 4, false>, grid, d.threads, s, p));
}

int64_t grad_ctas(int64_t rows, int teams) { return std::max<int64_t>(1, std::min<int64_t>(kGradCtas, ceil_div(rows, teams))); }

template <typename TY, typename TH>
fp4q_status launch_grad(GradParams p, float *dweight, int accumulate, void *scratch, bool fast, cudaStream_t s)
{
    const Deal d(ceil_div(p.cols, 16));
    p.team = d.team;
    const int teams = d.threads / d.team;
    const bool fused = dweight && p.cols <= kGradFused;
    p.partial = dweight ? static_cast<float *>(scratch) : nullptr;
    int64_t parts = grad_ctas(p.rows, teams);
    if (fused) {
        if (fp4q_status st = launched(fast ? launch_dependent(rms_norm_bwd_kernel<TY, TH, 1, true, true>, dim3((unsigned)parts), d.threads, s, p)
                                              : launch_dependent(rms_norm_bwd_kernel<TY, TH, 1, true, false>, dim3((unsigned)parts), d.threads, s, p))) return st;
    } else if (p.rows > 0) {
        const int64_t ctas = ceil_div(p.rows, teams);
        const dim3 grid((unsigned)std::min<int64_t>(ctas, 0x7FFFFFFF));
        if (fp4q_status st = launched(d.chunks == 1   ? launch_dependent(rms_norm_bwd_kernel<TY, TH, 1, false, false>, grid, d.threads, s, p)
                                      : d.chunks == 2 ? launch_dependent(rms_norm_bwd_kernel<TY, TH, 2, false, false>, grid, d.threads, s, p)
                                                      : launch_dependent(rms_norm_bwd_kernel<TY, TH, 4, false, false>, grid, d.threads, s, p)))
            return st;
    }
    if (!dweight) return FP4Q_OK;
    if (!fused) {
        parts = std::max<int64_t>(1, std::min<int64_t>(kGradCtas, ceil_div(p.rows, 8)));
        if (fp4q_status st = launched(launch_dependent(rms_norm_dweight_kernel<TY, TH>, dim3((unsigned)ceil_div(p.cols, 512), (unsigned)parts), 256, s, p))) return st;
    }
    const SumParams q = {p.partial, p.cols, (int32_t)parts, accumulate != 0, dweight};
    return launched(launch_dependent(column_sum_kernel, dim3((unsigned)ceil_div(p.cols, 32)), 256, s, q));
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
    const Deal d(ceil_div(mx ? round_up(cols, 32) : cols, 16));
    NormParams p = {};
    p.rows = rows;
    p.cols = cols;
    p.team = d.team;
    p.format = n->q ? n->q_format : 0;
    p.eps = n->eps;
    p.inv_cols = 1.f / (float)cols;
    p.residual = n->residual;
    p.xb = rows_of<__nv_bfloat16>(n->x, rows, cols, n->ld_x);
    p.xf = rows_of<float>(n->x, rows, cols, n->ld_x);
    if (n->residual) {
        p.rb = rows_of<__nv_bfloat16>(n->residual, rows, cols, n->ld_residual);
        p.rf = rows_of<float>(n->residual, rows, cols, n->ld_residual);
        p.hb = rows_of<__nv_bfloat16>(n->h, rows, cols, n->ld_h);
        p.hf = rows_of<float>(n->h, rows, cols, n->ld_h);
    }
    p.yb = rows_of<__nv_bfloat16>(n->y, rows, cols, n->ld_y);
    p.yf = rows_of<float>(n->y, rows, cols, n->ld_y);
    p.y_f32 = n->y_type == FP4Q_OUT_F32;
    p.weight = weight_of(n->weight, n->weight_type, cols);
    p.q = n->q;
    p.ld_q = n->ld_q;
    p.scale = n->scale;
    p.ld_s = n->ld_s;
    p.rstd = n->rstd;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const bool x32 = n->x_type == FP4Q_OUT_F32, h32 = n->residual ? n->h_type == FP4Q_OUT_F32 : x32;
    const bool fast = cols % 16 == 0 && on_grid(n->x, n->ld_x, rows, size_of(n->x_type)) && (!n->residual || (on_grid(n->residual, n->ld_residual, rows, size_of(n->h_type)) && on_grid(n->h, n->ld_h, rows, size_of(n->h_type)))) &&
                      aligned(n->weight, 16) && (!n->y || on_grid(n->y, n->ld_y, rows, size_of(n->y_type)));
    if (x32) return h32 ? launch_norm<float, float>(p, d, fast, s) : launch_norm<float, __nv_bfloat16>(p, d, fast, s);
    return h32 ? launch_norm<__nv_bfloat16, float>(p, d, fast, s) : launch_norm<__nv_bfloat16, __nv_bfloat16>(p, d, fast, s);
}

extern "C" size_t fp4q_rms_norm_bwd_scratch_bytes(int64_t rows, int64_t cols)
{
    if (rows < 0 || cols <= 0 || cols > kMostCols) return 0;
    return (size_t)round_up(std::max<int64_t>(1, std::min<int64_t>(kGradCtas, rows)) * cols * 4, 256);
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
    p.dyb = rows_of<__nv_bfloat16>(n->dy, rows, cols, n->ld_dy);
    p.dyf = rows_of<float>(n->dy, rows, cols, n->ld_dy);
    p.hb = rows_of<__nv_bfloat16>(n->h, rows, cols, n->ld_h);
    p.hf = rows_of<float>(n->h, rows, cols, n->ld_h);
    p.dhb = rows_of<__nv_bfloat16>(n->dh, rows, cols, n->ld_dh);
    p.dhf = rows_of<float>(n->dh, rows, cols, n->ld_dh);
    p.dxb = rows_of<__nv_bfloat16>(n->dx, rows, cols, n->ld_dx);
    p.dxf = rows_of<float>(n->dx, rows, cols, n->ld_dx);
    p.rstd = n->rstd;
    p.weight = weight_of(n->weight, n->weight_type, cols);
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const bool y32 = n->dy_type == FP4Q_OUT_F32, h32 = n->h_type == FP4Q_OUT_F32;
    const size_t hs = size_of(n->h_type);
    const bool fast = cols % 16 == 0 && on_grid(n->dy, n->ld_dy, rows, size_of(n->dy_type)) && on_grid(n->h, n->ld_h, rows, hs) && on_grid(n->dh, n->ld_dh, rows, hs) &&
                      on_grid(n->dx, n->ld_dx, rows, hs) && aligned(n->weight, 16);
    if (y32) return h32 ? launch_grad<float, float>(p, n->dweight, n->accumulate, scratch, fast, s) : launch_grad<float, __nv_bfloat16>(p, n->dweight, n->accumulate, scratch, fast, s);
    return h32 ? launch_grad<__nv_bfloat16, float>(p, n->dweight, n->accumulate, scratch, fast, s) : launch_grad<__nv_bfloat16, __nv_bfloat16>(p, n->dweight, n->accumulate, scratch, fast, s);
}
