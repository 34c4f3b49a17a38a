// Orthogonalised updates: momentum, normalisation and Newton-Schulz steps for a stack of weight gradients (include/fp4q.h).
//
//   X <- U / (|U| + eps);  per step, with A = X X^T on the shorter side:  X <- a X + (b A + c A A) X
//
// A step is three products: A = X X^T and P = a I + b A + c A A are symmetric, so only the tiles on and below the diagonal are computed and
// written to both places; X' = P X.  A matrix that is taller than wide keeps its layout: A = X^T X and X' = X P, with operands read across
// their rows.
//
// Precision.  The products' operands are FP16: values of X, A and P lie in a narrow range (singular values of at most about 1.3), so the
// three bits that FP16 has more than BF16 cost nothing.  X itself is kept as a sum of two FP16 numbers (22 bits): A's product takes the upper
// one, and a times the lower one is added to P's product with the upper one.  P's diagonal, which has a in it, is rounded once, by up to 2^-11 of itself,
// and carries what A's rounding makes of b A + c A A.  Where a matrix's singular values are all alike A and P are little but their diagonals, and these
// errors do not average out.  The term a X carries directions of small singular values from step to step, multiplied by a = 3.4 each time,
// and rounding X as a whole puts noise into those that a gradient does not have (rank 100, 768 x 2048: the update is off by 1.8e-2 with one
// FP16 number and 1.4e-1 with a BF16 one, 1.3e-3 with the sum of two).  Matrices of a short side have few elements over which the roundings of
// A, P and the products' X average out and little work: there A and P are sums of two numbers as well, and the three products are made of three each
// (kSplitSide).  Beside the result's rounding to BF16, 1.7e-3 of its norm, they are off by 5e-7; others by 1.4e-3 (777 x 1003) to 2.8e-3 (385 x 30000) on random
// matrices, and by up to 4e-3 where all singular values are alike (orthogonal 400 x 400, an identity of 385).  Scales: X 2^10, A and P 2^9, so that elements of large matrices
// stay above FP16's smallest normal number and the largest singular values that the entry point admits below its largest.  A matrix whose norm is far
// below eps keeps X small for some steps: it has a power of two more in X's scale, of which every step takes back what X may have grown by, so that X
// is held to 22 bits, or 2^-33 of the norm that it starts with or may have grown to, whatever that norm is.
#include "gemm16.cuh"

#include <algorithm>
#include <cmath>

using namespace fp4q;

namespace {

constexpr int kNsThreads = 256, kNsMaxBlocks = 1024;
constexpr int kLogScaleX = 10;
constexpr float kScaleX = 1 << kLogScaleX, kScaleA = 512.0f;
constexpr int kMaxSteps = 64;
constexpr int kMaxLift = 100;   // what is smaller is beyond the result's type
constexpr int64_t kSplitSide = 384;

struct MomentumParams {
    const void *g;
    float *m;                    // NULL: none
    int64_t ld_g, ld_m;
    int64_t rows;
    int32_t cols, g_f32, vec_g, vec_m;
    uint32_t units_row, units;   // units of eight columns in a row and in a matrix
    float beta;
    int32_t nesterov;
    double eps;
    double *partial;             // [count, gridDim.x]
    int32_t *lift;               // [count]
    __half *up, *lo;             // normalised: upper and lower parts
    int64_t pitch;
    uint32_t *counters;          // of the products' tiles, to be zeroed
    int32_t n_counters;
};

struct Eight {
    float v[8];
};
__device__ __forceinline__ Eight load_eight(const float *p, bool vec, int left)
{
    Eight r;
    if (vec && left >= 8) {
        const float4 a = *reinterpret_cast<const float4 *>(p), b = *reinterpret_cast<const float4 *>(p + 4);
        return Eight{{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}};
    }
#pragma unroll
    for (int e = 0; e < 8; e++) r.v[e] = e < left ? p[e] : 0.f;
    return r;
}
__device__ __forceinline__ Eight load_eight(const __nv_bfloat16 *p, bool vec, int left)
{
    Eight r;
    if (vec && left >= 8) {
        const uint4 w = *reinterpret_cast<const uint4 *>(p);
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int e = 0; e < 4; e++) { r.v[2 * e] = __uint_as_float(u[e] << 16); r.v[2 * e + 1] = __uint_as_float(u[e] & 0xFFFF0000u); }
        return r;
    }
#pragma unroll
    for (int e = 0; e < 8; e++) r.v[e] = e < left ? __bfloat162float(p[e]) : 0.f;
    return r;
}
__device__ __forceinline__ void store_eight(float *p, bool vec, int left, const Eight &x)
{
    if (vec && left >= 8) {
        *reinterpret_cast<float4 *>(p) = make_float4(x.v[0], x.v[1], x.v[2], x.v[3]);
        *reinterpret_cast<float4 *>(p + 4) = make_float4(x.v[4], x.v[5], x.v[6], x.v[7]);
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; e++)
        if (e < left) p[e] = x.v[e];
}

// The block's sum, in an order that depends on nothing but the block's size; every thread gets it.
__device__ __forceinline__ double block_sum(double v)
{
    __shared__ double part[kNsThreads / 32];
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
    __syncthreads();
    double s = 0.0;
#pragma unroll
    for (int w = 0; w < kNsThreads / 32; w++) s += part[w];
    return s;
}

// FINISH = false: the momentum, and each block's share of |U|^2.  FINISH = true: the norm, and X = U / (|U| + eps) in two halves.
// The sum of squares is held in 64 bits: gradients of 1e-25 and 1e25 have squares that FP32 does not.
// UNROLL: units of eight columns that a thread has under way: one in stacks (64 of 768 x 2048, BF16 gradients: 157 and 180 us, with two 199 and 200;
// 1 GB each), two in a single matrix, whose blocks are fewer (11008 x 4096: 105 and 87 with one, 86 and 85 with two; 541 MB).  Six blocks an SM, 40 registers, in
// the stacks' first pass (128 of 768 x 2048 313 us; 347 with 42 registers and five blocks).
template <bool FINISH, int UNROLL>
__global__ void __launch_bounds__(kNsThreads, !FINISH && UNROLL == 1 ? 6 : 1) momentum_kernel(const MomentumParams p)
{
    wait_for_predecessor();
    const int64_t row0 = (int64_t)blockIdx.y * p.rows;
    double sum = 0.0;
    int lift = 0;
    float inv0 = 0.f, inv1 = 0.f;   // 1 / (|U| + eps), scaled, as a power of two and the rest, rounded by 2^-24 as one factor of the matrix: it may lie outside of what FP32 holds
    if (FINISH) {
        for (int i = threadIdx.x; i < (int)gridDim.x; i += kNsThreads) sum += load_global(p.partial + (int64_t)blockIdx.y * gridDim.x + i);
        const double norm = sqrt(block_sum(sum));
        // A norm below eps leaves X small: it is scaled by so much more that its own norm lies between a quarter and one (from the numbers' exponents).
        lift = norm > 0.0 ? max(0, min(kMaxLift, (__double2hiint(norm + p.eps) >> 20) - (__double2hiint(norm) >> 20) - 1)) : 0;
        const double inv = __hiloint2double((1023 + kLogScaleX + lift) << 20, 0) / (norm + p.eps);
        int e;
        frexp(inv, &e);
        e = max(-200, min(200, e)) / 2;
        inv0 = ldexpf(1.f, e);
        inv1 = (float)ldexp(inv, -e);
    }
    const uint32_t step = gridDim.x * kNsThreads;
    for (uint32_t base = blockIdx.x * kNsThreads + threadIdx.x; base < p.units; base += UNROLL * step) {
        Eight g[UNROLL], m[UNROLL];
        int64_t row[UNROLL];
        int col[UNROLL];
#pragma unroll
        for (int j = 0; j < UNROLL; j++) {
            const uint32_t u = base + j * step;
            const uint32_t r = u / p.units_row;
            row[j] = u < p.units ? row0 + r : -1;
            col[j] = (int)(u - r * p.units_row) * 8;
            if (row[j] < 0) continue;
            const int left = p.cols - col[j];
            if (!FINISH || !p.m || p.nesterov)
                g[j] = p.g_f32 ? load_eight(static_cast<const float *>(p.g) + row[j] * p.ld_g + col[j], p.vec_g, left)
                               : load_eight(static_cast<const __nv_bfloat16 *>(p.g) + row[j] * p.ld_g + col[j], p.vec_g, left);
            if (p.m) m[j] = load_eight(p.m + row[j] * p.ld_m + col[j], p.vec_m, left);
        }
#pragma unroll
        for (int j = 0; j < UNROLL; j++) {
            if (row[j] < 0) continue;
            Eight u = g[j];
            if (p.m) {
                if (!FINISH) {
#pragma unroll
                    for (int e = 0; e < 8; e++) m[j].v[e] = fmaf(p.beta, m[j].v[e], g[j].v[e]);
                    store_eight(p.m + row[j] * p.ld_m + col[j], p.vec_m, p.cols - col[j], m[j]);
                }
#pragma unroll
                for (int e = 0; e < 8; e++) u.v[e] = p.nesterov ? fmaf(p.beta, m[j].v[e], g[j].v[e]) : m[j].v[e];
            }
            if (!FINISH) {
#pragma unroll
                for (int e = 0; e < 8; e++) sum += (double)u.v[e] * u.v[e];
            } else {
                uint32_t up[4], lo[4];
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    const float x = u.v[2 * e] * inv0 * inv1, y = u.v[2 * e + 1] * inv0 * inv1;
                    up[e] = pack_half(x, y);
                    const float2 h = unpack_half(up[e]);
                    lo[e] = pack_half(x - h.x, y - h.y);
                }
                const int64_t at = row[j] * p.pitch + col[j];
                *reinterpret_cast<uint4 *>(p.up + at) = make_uint4(up[0], up[1], up[2], up[3]);
                *reinterpret_cast<uint4 *>(p.lo + at) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
            }
        }
    }
    if (FINISH && blockIdx.x == 0 && threadIdx.x == 0) p.lift[blockIdx.y] = lift;
    if (!FINISH && blockIdx.x == 0 && blockIdx.y == 0)
        for (int i = threadIdx.x; i < p.n_counters; i += kNsThreads) p.counters[i] = 0u;
    if (!FINISH) {
        sum = block_sum(sum);
        if (threadIdx.x == 0) p.partial[(int64_t)blockIdx.y * gridDim.x + blockIdx.x] = sum;
    }
}

// Rounds of tiles of 128 x 128 in single CTAs or 256 x 256 in pairs, in us: a round takes its boxes, which get 115 GB/s an SM and 15 TB/s in all from L2, and
// 2 or 4 us.
double rounds_us(int64_t tiles, int64_t stages, int64_t edge)
{
    const int64_t slots = edge == 256 ? 74 : 148, sms = edge == 256 ? 2 : 1;
    const double box = std::max(32768.0 / 115e3, 32768.0 * (double)(sms * std::min(tiles, slots)) / 15e6);
    return (double)ceil_div(tiles, slots) * ((double)stages * box + 2.0 * sms);
}
// A's product in tiles of `edge`, its contraction of `stages` boxes cut into parts: the number of parts with the least estimated time.  Parts take
// their way through memory, where whoever comes last reads them one after the other.  (Parts for 4751 x 63: 70 -> 20 us.)  No accumulator takes more than
// kMostElems elements: the tensor cores cut it off towards zero, by 5e-9 of a sum of squares for each (16 x 2^20 in one: the update off by 8.5e-3).  It costs
// stacks of some hundred short and very long matrices their 64 x 64 tiles, which are not cut (130 of 16 x 250000 22.4 -> 31.2 ms).
constexpr int64_t kMostElems = 32768;
struct GramPlan {
    int64_t tiles, parts = 1;
    double us = 1e30;
    GramPlan(int64_t count, int64_t side, int64_t stages, int64_t most, int64_t edge)
    {
        const int64_t across = ceil_div(side, edge), slots = edge == 256 ? 74 : 148, least = ceil_div(stages, most);
        tiles = count * across * (across + 1) / 2;
        for (int64_t n = least; n == least || (n <= 32 && stages / n >= 16 && tiles * n <= 4 * slots); n++) {
            const double t = rounds_us(tiles * n, ceil_div(stages, n), edge) + (n > 1 ? 3.0 + 0.6 * (double)n : 0.0);
            if (t < us) { us = t; parts = n; }
        }
    }
};

// Where things lie in the scratch memory.
struct Scratch {
    int64_t pitch_x, pitch_a, side;
    bool split;
    int edge;                            // tiles of A's product: 64, 128 or 256 (pairs)
    int64_t tiles, part_stages;
    size_t counters, accumulators, partial, lift, x[2], lo[2], a[2], poly[2], bytes;   // upper and lower parts; X and the next X: lower parts in one place unless they are operands
    Scratch(int64_t count, int64_t rows, int64_t cols)
    {
        side = rows < cols ? rows : cols;
        pitch_x = round_up(cols, 16);
        pitch_a = round_up(side, 16);
        const size_t x_bytes = (size_t)round_up(count * rows * pitch_x * 2, 256), a_bytes = (size_t)round_up(count * side * pitch_a * 2, 256);
        split = side <= kSplitSide;
        partial = 0;
        bytes = (size_t)round_up(count * kNsMaxBlocks * 8, 256);
        auto place = [&](size_t n) { const size_t at = bytes; bytes += n; return at; };
        lift = place((size_t)round_up(count * 4, 256));
        x[0] = place(x_bytes); x[1] = place(x_bytes);
        lo[0] = place(x_bytes); lo[1] = split ? place(x_bytes) : lo[0];
        a[0] = place(a_bytes); a[1] = split ? place(a_bytes) : a[0];
        poly[0] = place(a_bytes); poly[1] = split ? place(a_bytes) : poly[0];
        const int64_t stages = (split ? 2 : 1) * ceil_div(rows < cols ? cols : rows, kBox16);
        const int64_t most = (split ? 2 : 1) * kMostElems / kBox16;
        const GramPlan one(count, side, stages, most, 128), two(count, side, stages, most, 256);
        const bool pairs = two.us < one.us;
        // 64 x 64 tiles, 0.17 us a stage, where all of them run at once and no parts are faster (which take about 3 us more than estimated): they are
        // all computed, and not cut.  All five steps, in larger tiles and in these: 256 x 256 129 and 104 us, 300 x 1500 167 and 143, 85 of 2382 x 45
        // 370 and 311; 200 x 5000 182 and 232.
        const bool small = stages <= most && count * ceil_div(side, 64) * ceil_div(side, 64) <= 148 && 0.17 * (double)stages < std::min(one.us, two.us) + 2.0;
        edge = small ? 64 : pairs ? 256 : 128;
        tiles = pairs ? two.tiles : one.tiles;
        const int64_t parts = edge == 64 ? 1 : pairs ? two.parts : one.parts;
        part_stages = parts >= 2 ? round_up(ceil_div(stages, parts), split ? 2 : 1) : 0;
        counters = place(part_stages ? (size_t)round_up(tiles * 2 * 8 * 4, 256) : 0);
        accumulators = place(part_stages ? (size_t)(tiles * parts * (edge == 256 ? Cfg16<2, 256>::kPlaceBytes : Cfg16<1, 128>::kPlaceBytes)) : 0);
    }
};

const int64_t kMaxSide = 1 << 20, kMaxCount = 65535;

bool sizes_ok(int64_t count, int64_t rows, int64_t cols)
{
    const int64_t side = rows < cols ? rows : cols, across = ceil_div(side, 128);   // tiles of A and parts of them are counted in 32 bits, too
    return count <= kMaxCount && rows <= kMaxSide && cols <= kMaxSide && rows * ceil_div(cols, 8) < (1ll << 31) && count * rows <= 0x7FFFFFFF &&
           count * rows * round_up(cols, 16) <= (1ll << 40) && count * ceil_div(rows, 128) * ceil_div(cols, 64) <= 0x7FFFFFFF - 4096 &&
           count * (across * (across + 1) / 2) * ceil_div(rows < cols ? cols : rows, kMostElems) <= 0x7FFFFFFF - 4096;
}

// The largest singular value x that X can have after each step, from at most 1, and the largest eigenvalues of b A + c A A and a I + b A + c A A, with
// q = x x: both polynomials are largest at an end of q's range or where their slope is zero.  Whether FP16 holds all that they reach.  grown[s]:
// powers of two by which a singular value may have grown before step s.
bool steps_fit(const float *coefficients, int32_t steps, int32_t *grown)
{
    double top = 1.0;
    grown[0] = 0;
    for (int32_t s = 0; s < steps; s++) {
        const double a = coefficients[3 * s], b = coefficients[3 * s + 1], c = coefficients[3 * s + 2], end = top * top;
        const double root = std::sqrt(std::max(0.0, 9.0 * b * b - 20.0 * a * c));   // a + 3 b q + 5 c q q = 0; b + 2 c q = 0 first
        const double at[4] = {end, c != 0.0 ? -b / (2.0 * c) : end, c != 0.0 ? (-3.0 * b + root) / (10.0 * c) : b != 0.0 ? -a / (3.0 * b) : end,
                              c != 0.0 ? (-3.0 * b - root) / (10.0 * c) : end};
        double next = 0.0, factor = std::fabs(a);
        for (const double q : at) {
            if (q < 0.0 || q > end) continue;
            const double poly = b * q + c * q * q, all = std::fabs(a + poly), y = std::sqrt(q) * all;
            if (!(std::fabs(poly) <= 100.0) || !(all <= 100.0) || !(y <= 10.0)) return false;
            next = std::max(next, y);
            factor = std::max(factor, all);
        }
        if (!(factor <= 100.0)) return false;
        grown[s + 1] = grown[s] + std::max(0, (int32_t)std::ceil(std::log2(std::max(factor, 1e-3) * 1.01)));
        top = std::max(next * 1.01, 1e-3);   // roundings
    }
    return true;
}

// Upper and lower parts of an operand.
struct Parts {
    Operand16 up, lo;
    Parts(const void *u, const void *l, int64_t cols, int64_t rows, int64_t count, int64_t pitch)
        : up{u, cols, rows, count, pitch, rows * pitch}, lo{l, cols, rows, count, pitch, rows * pitch} {}
};

// Boxes of an epilogue: what it reads or writes, and mirrored.
fp4q_status boxes16(CUtensorMap *up, CUtensorMap *lo, const Parts &x, bool two, bool mirrored = false)
{
    const int cols = mirrored ? 32 : 64, rows = mirrored ? 64 : 32;
    const CUtensorMapSwizzle swizzle = mirrored ? CU_TENSOR_MAP_SWIZZLE_NONE : CU_TENSOR_MAP_SWIZZLE_128B;
    return make_map16(up, x.up, cols, rows, swizzle) && (!two || make_map16(lo, x.lo, cols, rows, swizzle)) ? FP4Q_OK : FP4Q_ERR_CUDA;
}

template <int CTAS, int BN>
struct Steps {
    static constexpr int kBM = Cfg16<CTAS, BN, false, true>::kTileRows;
    static_assert(kBM == BN, "symmetric products have square tiles");
    // 64 x 64 tiles are all computed, which is as fast and saves the mirrored stores: they all run at once.
    static constexpr int kSym = BN == 64 ? TILES_BATCH : TILES_SYM;
    static int64_t symmetric_tiles(Gemm16Params &p)
    {
        p.a_box = kBM / CTAS;
        p.m_tiles = p.n_tiles = (int32_t)ceil_div(p.n, BN);
        return (int64_t)p.batch * p.m_tiles * (kSym == TILES_BATCH ? 2 * p.m_tiles : p.m_tiles + 1) / 2;
    }
    static fp4q_status gram(const Parts &x, const Parts &a, bool tall, Gemm16Params p, cudaStream_t stream)
    {
        Maps16 maps = {};
        int64_t tiles = symmetric_tiles(p);
        if (p.partial) tiles *= ceil_div((p.split ? 2 : 1) * ceil_div(p.k, kBox16), p.part_stages);
        if (fp4q_status s = boxes16(&maps.out, &maps.out2, a, p.split)) return s;
        if (fp4q_status s = boxes16(&maps.mirror, &maps.mirror2, a, p.split, true)) return s;
        return tall ? launch_gemm16<CTAS, BN, true, true, EPI16_GRAM, kSym>(x.up, x.up, x.lo, x.lo, maps, p, tiles, stream)
                    : launch_gemm16<CTAS, BN, false, false, EPI16_GRAM, kSym>(x.up, x.up, x.lo, x.lo, maps, p, tiles, stream);
    }
    static fp4q_status poly(const Parts &a, const Parts &poly, Gemm16Params p, cudaStream_t stream)
    {
        Maps16 maps = {};
        const int64_t tiles = symmetric_tiles(p);
        if (fp4q_status s = boxes16(&maps.in, &maps.in2, a, p.split)) return s;
        if (fp4q_status s = boxes16(&maps.out, &maps.out2, poly, p.split)) return s;
        if (fp4q_status s = boxes16(&maps.mirror, &maps.mirror2, poly, p.split, true)) return s;
        return launch_gemm16<CTAS, BN, false, false, EPI16_POLY, kSym>(a.up, a.up, a.lo, a.lo, maps, p, tiles, stream);
    }
    static fp4q_status update(const Parts &x, const Parts &poly, const Parts &next, bool tall, Gemm16Params p, cudaStream_t stream)
    {
        Maps16 maps = {};
        p.a_box = kBM / CTAS;
        p.m_tiles = (int32_t)ceil_div(p.m, kBM);
        p.n_tiles = (int32_t)ceil_div(p.n, BN);
        const int64_t tiles = (int64_t)p.batch * p.m_tiles * p.n_tiles;
        if (!p.split && !make_map16(&maps.in2, x.lo, 64, 32)) return FP4Q_ERR_CUDA;
        if (p.o) {
            if (p.boxed > 0 && !make_map16(&maps.out, Operand16{p.o, p.boxed, p.m, p.batch, p.ld_o, p.m * p.ld_o}, 64, 32)) return FP4Q_ERR_CUDA;
        } else if (fp4q_status s = boxes16(&maps.out, &maps.out2, next, true)) {
            return s;
        }
        return tall ? launch_gemm16<CTAS, BN, false, false, EPI16_UPDATE, TILES_BATCH>(x.up, poly.up, x.lo, poly.lo, maps, p, tiles, stream)
                    : launch_gemm16<CTAS, BN, false, true, EPI16_UPDATE, TILES_BATCH>(poly.up, x.up, poly.lo, x.lo, maps, p, tiles, stream);
    }
};

}  // namespace

extern "C" size_t fp4q_newton_schulz_scratch_bytes(int64_t count, int64_t rows, int64_t cols)
{
    if (count <= 0 || rows <= 0 || cols <= 0 || !sizes_ok(count, rows, cols)) return 0;
    return Scratch(count, rows, cols).bytes;
}

extern "C" fp4q_status fp4q_newton_schulz(const void *g, fp4q_out g_type, int64_t count, int64_t rows, int64_t cols, int64_t ld_g, float *momentum, int64_t ld_m,
                                          float beta, int nesterov, const float *coefficients, int32_t steps, float eps, float scale, void *out_bf16,
                                          int64_t ld_o, void *scratch, size_t scratch_bytes, void *ws, size_t ws_bytes, void *stream)
{
    if (count < 0 || rows < 0 || cols < 0 || ld_g < cols || ld_o < cols || (momentum && ld_m < cols)) return FP4Q_ERR_SHAPE;
    if (g_type != FP4Q_OUT_BF16 && g_type != FP4Q_OUT_F32) return FP4Q_ERR_UNSUPPORTED;
    if (!coefficients) return FP4Q_ERR_NULL;
    int32_t grown[kMaxSteps + 1];
    if (steps < 1 || steps > kMaxSteps || !(eps >= 0.0f) || !steps_fit(coefficients, steps, grown)) return FP4Q_ERR_UNSUPPORTED;
    if (count == 0 || rows == 0 || cols == 0) return FP4Q_OK;
    if (!sizes_ok(count, rows, cols)) return FP4Q_ERR_UNSUPPORTED;
    if (!g || !out_bf16) return FP4Q_ERR_NULL;
    const size_t g_bytes = g_type == FP4Q_OUT_F32 ? 4 : 2;
    if (!aligned(g, g_bytes) || !aligned(momentum, 4) || !aligned(out_bf16, 2)) return FP4Q_ERR_ALIGN;
    const Scratch at(count, rows, cols);
    if (!ws || ws_bytes < sizeof(Workspace) || !scratch || scratch_bytes < at.bytes) return FP4Q_ERR_WORKSPACE;
    if (!aligned(ws, 256) || !aligned(scratch, 256)) return FP4Q_ERR_ALIGN;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    uint8_t *base = static_cast<uint8_t *>(scratch);
    auto half_at = [&](size_t offset) { return reinterpret_cast<__half *>(base + offset); };

    MomentumParams q = {};
    q.g = g; q.m = momentum; q.ld_g = ld_g; q.ld_m = ld_m; q.rows = rows; q.cols = (int32_t)cols;
    q.g_f32 = g_type == FP4Q_OUT_F32;
    q.vec_g = aligned(g, 16) && ld_g * g_bytes % 16 == 0;
    q.vec_m = momentum && aligned(momentum, 16) && ld_m % 4 == 0;
    q.units_row = (uint32_t)ceil_div(cols, 8);
    q.units = (uint32_t)(rows * q.units_row);
    q.beta = beta; q.nesterov = nesterov != 0; q.eps = eps;
    q.partial = reinterpret_cast<double *>(base + at.partial);
    q.lift = reinterpret_cast<int32_t *>(base + at.lift);
    q.counters = reinterpret_cast<uint32_t *>(base + at.counters);
    q.n_counters = at.part_stages ? (int32_t)(at.tiles * (at.edge == 256 ? 16 : 8)) : 0;
    q.up = half_at(at.x[0]); q.lo = half_at(at.lo[0]); q.pitch = at.pitch_x;
    const int64_t want = ceil_div(q.units, kNsThreads * (count > 1 ? 1 : 2)), share = ceil_div(16 * 148, count);
    const dim3 grid((unsigned)std::min<int64_t>(std::min(want, share), kNsMaxBlocks), (unsigned)count);
    if (fp4q_status st = launched(launch_dependent(count > 1 ? momentum_kernel<false, 1> : momentum_kernel<false, 2>, grid, kNsThreads, s, q, true))) return st;
    if (fp4q_status st = launched(launch_dependent(count > 1 ? momentum_kernel<true, 1> : momentum_kernel<true, 2>, grid, kNsThreads, s, q, true))) return st;

    const bool tall = rows > cols;
    const int64_t side = at.side;
    Gemm16Params p = {};
    p.batch = (int32_t)count;
    p.a_box = 128;
    p.status = static_cast<uint32_t *>(ws);
    p.split = at.split;
    p.lift = q.lift;
    p.admit = 1;
    const Parts part_a(half_at(at.a[0]), half_at(at.a[1]), side, side, count, at.pitch_a), part_p(half_at(at.poly[0]), half_at(at.poly[1]), side, side, count, at.pitch_a);
    // P and X': 64 x 64 tiles where one round of them does, each with less to load and a shorter epilogue; else what is estimated to be faster
    // (all steps with pairs for all that takes several rounds, and so: 200 of 128 x 128 220 and 164 us, 86 of 6358 x 29 618 and 557; 4 of 900 x 1000 197 and
    // 201).
    const int64_t s64 = ceil_div(side, 64), s128 = ceil_div(side, 128), s256 = ceil_div(side, 256), stages = (at.split ? 2 : 1) * s64;
    auto edge_of = [&](int64_t tiles64, int64_t tiles128, int64_t tiles256) {
        if (count * tiles64 <= 148) return 64;
        return rounds_us(count * tiles128, stages, 128) <= rounds_us(count * tiles256, stages, 256) ? 128 : 256;
    };
    const int edge_poly = edge_of(s64 * s64, s128 * (s128 + 1) / 2, s256 * (s256 + 1) / 2),
              edge_update = edge_of(ceil_div(rows, 64) * ceil_div(cols, 64), ceil_div(rows, 128) * ceil_div(cols, 128), ceil_div(rows, 256) * ceil_div(cols, 256));
    for (int32_t i = 0; i < steps; i++) {
        const float *c = coefficients + 3 * i;
        const int now = i & 1, next = now ^ 1;
        p.grown = grown[i];
        p.grown_next = grown[i + 1];
        const Parts part_x(half_at(at.x[now]), half_at(at.lo[now]), cols, rows, count, at.pitch_x);
        const Parts part_next(half_at(at.x[next]), half_at(at.lo[next]), cols, rows, count, at.pitch_x);
        Gemm16Params gp = p;
        gp.m = gp.n = (int32_t)side;
        gp.k = (int32_t)(tall ? rows : cols);
        gp.fa = kScaleA / (kScaleX * kScaleX);
        Gemm16Params pp = gp;
        if (at.part_stages) {
            gp.part_stages = (int32_t)at.part_stages;
            gp.partial = reinterpret_cast<float *>(base + at.accumulators);
            gp.counters = reinterpret_cast<uint32_t *>(base + at.counters);
        }
        pp.k = (int32_t)side;
        pp.fa = c[0] * kScaleA;
        pp.fb = c[1];
        pp.fc = c[2] / kScaleA;
        Gemm16Params up = p;
        up.m = (int32_t)rows;
        up.n = (int32_t)cols;
        up.k = (int32_t)side;
        up.fb = c[0];
        up.fc = 1.0f / kScaleA;
        if (i == steps - 1) {
            up.admit = 0;
            up.o = static_cast<__nv_bfloat16 *>(out_bf16);
            up.ld_o = ld_o;
            up.o_scale = scale / kScaleX;
            up.boxed = aligned(out_bf16, 16) && ld_o % 8 == 0 ? (int32_t)(cols / 8 * 8) : 0;
        }
        fp4q_status st = at.edge == 256   ? Steps<2, 256>::gram(part_x, part_a, tall, gp, s)
                         : at.edge == 128 ? Steps<1, 128>::gram(part_x, part_a, tall, gp, s)
                                          : Steps<1, 64>::gram(part_x, part_a, tall, gp, s);
        if (!st)
            st = edge_poly == 256   ? Steps<2, 256>::poly(part_a, part_p, pp, s)
                 : edge_poly == 128 ? Steps<1, 128>::poly(part_a, part_p, pp, s)
                                    : Steps<1, 64>::poly(part_a, part_p, pp, s);
        if (!st)
            st = edge_update == 256   ? Steps<2, 256>::update(part_x, part_p, part_next, tall, up, s)
                 : edge_update == 128 ? Steps<1, 128>::update(part_x, part_p, part_next, tall, up, s)
                                      : Steps<1, 64>::update(part_x, part_p, part_next, tall, up, s);
        if (st) return st;
    }
    return FP4Q_OK;
}
