// Products of 8-bit tensors with a scale for every block of 128 contraction elements: C[M,N] = sum over blocks b of sA sB (A_b B_b^T), codes E4M3,
// scales FP32 (include/fp4q.h).
//
// A stage of the operand ring is one block: rows of 128 bytes.  Four tcgen05.mma (kind::f8f6f4, 32 elements each) make the block's product in an accumulator of its
// own in tensor memory; the epilogue's warps take it from there, times its scales, into sums in registers, while the next block's MMAs run into
// another accumulator.  The accumulator that the tensor cores cut off towards zero is thus never longer than 128 elements; the sums are rounded to nearest.
// Bound by that path of the accumulators, 1100 cycles a block of a pair's tile where its MMAs take 512: 16384 x 11008 x 4096 800 us (1.85 PFLOP/s; 690 in a short run), the weight gradient of 4096 x 4096 over
// 16384 rows 411.  One token: bound by the weight's bytes, 4096 x 11008 12.3 us.
#include "fp8_format.cuh"
#include "gemm16.cuh"

#include <cuda_fp8.h>

#include <algorithm>

using namespace fp4q;

namespace {

constexpr int kBlock8 = 128;   // contraction elements, and bytes, of a block

// Which operand's scales differ inside a tile: those of A's rows (B's are one number for 128 columns), those of B's rows, or both.
enum { SCALE_ROWS = 0, SCALE_COLS = 1, SCALE_BOTH = 2 };

// The scale of row r and block b: p[(r >> shift) * row + b * block].
struct Scales8 {
    const float *p;
    int64_t row, block;
    int32_t shift;
    int32_t fours;                   // four blocks of a row lie in 16 aligned bytes
    __device__ __forceinline__ float at(int r, int b) const { return load_global(p + (int64_t)(r >> shift) * row + b * block); }
    // Blocks b .. b + 3 of row r, those below `end`; b is a multiple of four.
    __device__ __forceinline__ float4 four(int r, int b, int end) const
    {
        if (fours && b + 4 <= end) return load_global(reinterpret_cast<const float4 *>(p + (int64_t)(r >> shift) * row + b));
        return make_float4(at(r, b), b + 1 < end ? at(r, b + 1) : 0.f, b + 2 < end ? at(r, b + 2) : 0.f, b + 3 < end ? at(r, b + 3) : 0.f);
    }
};

struct Gemm8Params {
    int32_t m, n, blocks;            // rows of A and B, blocks of the contraction
    int32_t m_tiles, n_tiles, split; // split: CTAs of a cluster, which share a tile's contraction
    int32_t whole, pieces;           // persistent: tiles that are computed as one, and pieces in all; the tiles behind these are two pieces each, of half of the columns
    int32_t boxed;                   // columns that leave in boxes, whole 16 bytes; the rest of a row leaves by itself
    Scales8 sa, sb;
    void *c;                         // row-major, [m, n] or, with SCALE_COLS, its transpose: [n, m]
    int64_t ldc;
    int32_t f32, accumulate, wide;
    uint32_t *status;
    const uint8_t *qa, *qb;          // codes, for sums that are not finite: rows of A and B, k of each
    int64_t lda, ldb, k;
};
struct Maps8 {
    CUtensorMap a, b;
};

// By the lanes for which `issue` holds, without a branch (see tcgen05_mma_f16).  PAIR: the copy is counted on a barrier of the pair's leader.
template <bool PAIR>
__device__ __forceinline__ void tma_load_if(uint32_t dst, const CUtensorMap *map, int32_t x, int32_t y, uint32_t bar, bool issue)
{
    if (PAIR)
        asm volatile("{\n .reg .pred q;\n setp.ne.b32 q, %5, 0;\n"
                     "@q cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];\n}"
                     ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar), "r"((uint32_t)issue) : "memory");
    else
        asm volatile("{\n .reg .pred q;\n setp.ne.b32 q, %5, 0;\n"
                     "@q cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];\n}"
                     ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar), "r"((uint32_t)issue) : "memory");
}
template <int CTAS>
__device__ __forceinline__ void tcgen05_mma_f8(uint32_t d_tmem, uint32_t a_lo, uint32_t b_lo, uint32_t hi, uint32_t idesc, bool accumulate, bool issue)
{
    if (CTAS == 2)
        asm volatile("{\n .reg .pred p, q;\n .reg .b64 a, b;\n setp.ne.b32 p, %5, 0;\n setp.ne.b32 q, %6, 0;\n mov.b64 a, {%1, %3};\n mov.b64 b, {%2, %3};\n"
                     "@q tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], a, b, %4, p;\n}"
                     ::"r"(d_tmem), "r"(a_lo), "r"(b_lo), "r"(hi), "r"(idesc), "r"((uint32_t)accumulate), "r"((uint32_t)issue) : "memory");
    else
        asm volatile("{\n .reg .pred p, q;\n .reg .b64 a, b;\n setp.ne.b32 p, %5, 0;\n setp.ne.b32 q, %6, 0;\n mov.b64 a, {%1, %3};\n mov.b64 b, {%2, %3};\n"
                     "@q tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], a, b, %4, p;\n}"
                     ::"r"(d_tmem), "r"(a_lo), "r"(b_lo), "r"(hi), "r"(idesc), "r"((uint32_t)accumulate), "r"((uint32_t)issue) : "memory");
}
// E4M3 x E4M3 -> FP32, both operands along the contraction; 128 rows of A for each CTA.
template <int CTAS>
__device__ __forceinline__ uint32_t instr_desc8(int cols)
{
    return (1u << 4) | ((uint32_t)(cols >> 3) << 17) | ((uint32_t)((128 * CTAS) >> 4) << 24);
}

// Columns of an accumulator's row; the values are there after landed().
__device__ __forceinline__ void load_acc(uint32_t from, uint32_t (&v)[16]) { FP4Q_TMEM_LD_X16(from, v); }
__device__ __forceinline__ void landed(uint32_t (&v)[16])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]), "+r"(v[8]), "+r"(v[9]), "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]),
                   "+r"(v[14]), "+r"(v[15])
                 :: "memory");
}

__device__ __forceinline__ void load_scales_16(uint32_t at, float (&f)[16])   // in shared memory, on 16 bytes; stays behind the barrier before it
{
#pragma unroll
    for (int e = 0; e < 16; e += 4) asm volatile("ld.shared.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(f[e]), "=f"(f[e + 1]), "=f"(f[e + 2]), "=f"(f[e + 3]) : "r"(at + 4 * e));
}
__device__ __forceinline__ float load_scale(uint32_t at)
{
    float f;
    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(f) : "r"(at));
    return f;
}

// sum += a block's product times its scales, for COLS columns of a thread's row.  row: the row's scale; cols: where those of the columns lie in shared memory.  read: called when the
// accumulator has been read.  The scales are put together while the accumulator's values are on their way.  (Additions in pairs, fma.rn.f32x2, would halve the instructions, but
// every value is then moved into an aligned pair first: 8192 x 4096 x 4096 194 us for 147.)
template <int MODE, int COLS, typename F>
__device__ __forceinline__ void add_block(float (&sum)[COLS], uint32_t from, float row, uint32_t cols, F read)
{
#pragma unroll
    for (int c = 0; c < COLS; c += 16) {
        uint32_t x[16];
        float f[16];
        load_acc(from + c, x);
        if (MODE != SCALE_ROWS) load_scales_16(cols + 4 * c, f);
        if (MODE == SCALE_BOTH)
#pragma unroll
            for (int e = 0; e < 16; e += 2)   // in pairs, as they were loaded
                asm("{\n .reg .b64 a, b;\n mov.b64 a, {%0, %1};\n mov.b64 b, {%2, %2};\n mul.rn.f32x2 a, a, b;\n mov.b64 {%0, %1}, a;\n}" : "+f"(f[e]), "+f"(f[e + 1]) : "f"(row));
        landed(x);
        if (c + 16 == COLS) read();
#pragma unroll
        for (int e = 0; e < 16; e++) sum[c + e] = fmaf(__uint_as_float(x[e]), MODE == SCALE_ROWS ? row : f[e], sum[c + e]);
    }
}

// Scales are FP32 numbers, and the product of two need not be one.  Above FP32's range it is infinite, and the sum it enters infinite or, where the block's product is 0, NaN: sums that
// are not finite are looked at before they leave, and computed again, from the codes, if scales are why.  (The loops over blocks know nothing of it: a look at every set of scales there, with
// a way out, cost 5 to 20 %; this 0 to 2.)  Below the normal range a product of scales keeps fewer bits, which moves a block's share of a sum by |x| 2^-150 < 2^-125 at most.

// sum + x a b, with nothing on the way out of FP32's range that is in it at the end; |x| is 0 or from 2^-18 to 2^25.
__device__ __forceinline__ float add_scaled(float sum, float x, float a, float b)
{
    const float f = a * b;
    if (!is_infinite(f)) return fmaf(x, f, sum);
    return fmaf((x * 0x1p64f) * ((a * 0x1p-64f) * (b * 0x1p-64f)), 0x1p64f, sum);   // neither is below 1
}
// + the product of 16 codes of each operand.
__device__ __forceinline__ float add_codes(float x, const uint4 &a, const uint4 &b)
{
    const uint32_t u[4] = {a.x, a.y, a.z, a.w}, v[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
    for (int i = 0; i < 16; i++) {
        const auto value = [](uint32_t w, int at) { return __half2float(__half(__nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)(w >> at), __NV_E4M3))); };
        x = fmaf(value(u[i / 4], 8 * (i % 4)), value(v[i / 4], 8 * (i % 4)), x);
    }
    return x;
}
// Codes k .. k + 15 of a row, which begins on 16 bytes, those below n.
__device__ __forceinline__ uint4 codes_at(const uint8_t *row, int64_t k, int64_t n)
{
    if (k + 16 <= n) return load_global(reinterpret_cast<const uint4 *>(row + k));
    uint32_t w[4] = {0u, 0u, 0u, 0u};
    for (int i = 0; k + i < n; i++) w[i / 4] |= (uint32_t)load_global(row + k + i) << (8 * (i % 4));
    return make_uint4(w[0], w[1], w[2], w[3]);
}
// The sum of row m of A and row n of B, which was not finite.
__device__ __noinline__ float careful_sum(const Gemm8Params &p, int m, int n, float was)
{
    bool scales = false;
    for (int b = 0; b < p.blocks; b++) scales |= is_infinite(p.sa.at(m, b) * p.sb.at(n, b));
    if (!scales) return was;
    float sum = 0.f;
    const uint8_t *a = p.qa + m * p.lda, *w = p.qb + n * p.ldb;
    for (int b = 0; b < p.blocks; b++) {
        const int64_t end = min((int64_t)(b + 1) * kBlock8, p.k);
        float x = 0.f;
        for (int64_t k = (int64_t)b * kBlock8; k < end; k += 16) x = add_codes(x, codes_at(a, k, end), codes_at(w, k, end));
        sum = add_scaled(sum, x, p.sa.at(m, b), p.sb.at(n, b));
    }
    return sum;
}
__device__ __noinline__ void careful_sums(const Gemm8Params &p, int m, int n, int count, float *sums)   // columns n .. n + count - 1
{
    if (m >= p.m) return;
    float top = 0.f;   // a product of finite scales is infinite if both are above 1
    for (int b = 0; b < p.blocks; b++) top = fmaxf(top, fabsf(p.sa.at(m, b)));
    if (!(top > 1.f)) return;
    for (int e = 0; e < count && n + e < p.n; e++)
        if (!(fabsf(sums[e]) <= 0x1.fffffep127f)) sums[e] = careful_sum(p, m, n + e, sums[e]);
}
// Four sums next to one another in the output: along B's rows or, transposed, A's.
__device__ __noinline__ float4 careful_four(const Gemm8Params &p, int m, int n, bool transposed, float4 v)
{
    if (transposed) {
        careful_sums(p, m, n, 1, &v.x);
        careful_sums(p, m + 1, n, 1, &v.y);
        careful_sums(p, m + 2, n, 1, &v.z);
        careful_sums(p, m + 3, n, 1, &v.w);
    } else {
        careful_sums(p, m, n, 4, &v.x);
    }
    return v;
}
template <int COLS>
__device__ __forceinline__ void check_sums(const Gemm8Params &p, int m, int n, float (&sum)[COLS])
{
    float zero[4] = {0.f, 0.f, 0.f, 0.f};   // or NaN
#pragma unroll
    for (int i = 0; i < COLS; i++) zero[i % 4] = fmaf(sum[i], 0.f, zero[i % 4]);
    if (zero[0] + zero[1] + zero[2] + zero[3] == 0.f) return;
    float sums[COLS];
#pragma unroll
    for (int i = 0; i < COLS; i++) sums[i] = sum[i];
    careful_sums(p, m, n, COLS, sums);
#pragma unroll
    for (int i = 0; i < COLS; i++) sum[i] = sums[i];
}

// Columns col .. col + 15 of a row, of which those below n exist.
__device__ __forceinline__ void store_row16(const Gemm8Params &p, int64_t row, int col, int n, const float *v)
{
    const int left = n - col;
    if (left <= 0) return;
    if (p.f32) {
        float *c = static_cast<float *>(p.c) + row * p.ldc + col;
        if (left >= 16) {
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
                float4 w = make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]);
                if (p.accumulate) {
                    const float4 o = *reinterpret_cast<const float4 *>(c + e);
                    w.x += o.x; w.y += o.y; w.z += o.z; w.w += o.w;
                }
                *reinterpret_cast<float4 *>(c + e) = w;
            }
        } else {
#pragma unroll
            for (int e = 0; e < 16; e++)
                if (e < left) c[e] = p.accumulate ? c[e] + v[e] : v[e];
        }
    } else {
        __nv_bfloat16 *c = static_cast<__nv_bfloat16 *>(p.c) + row * p.ldc + col;
        if (left >= 16) {
            uint32_t w[8];
#pragma unroll
            for (int j = 0; j < 8; j++) w[j] = pack_bf16(v[2 * j], v[2 * j + 1]);
            if (p.wide) store_32_bytes(c, w);
            else {
                *reinterpret_cast<uint4 *>(c) = make_uint4(w[0], w[1], w[2], w[3]);
                *reinterpret_cast<uint4 *>(c + 8) = make_uint4(w[4], w[5], w[6], w[7]);
            }
        } else {
#pragma unroll
            for (int e = 0; e < 16; e++)
                if (e < left) c[e] = __float2bfloat16_rn(v[e]);
        }
    }
}
__device__ __forceinline__ void store_one(const Gemm8Params &p, int64_t row, int col, float v)
{
    if (p.f32) {
        float *c = static_cast<float *>(p.c) + row * p.ldc + col;
        *c = p.accumulate ? *c + v : v;
    } else {
        static_cast<__nv_bfloat16 *>(p.c)[row * p.ldc + col] = __float2bfloat16_rn(v);
    }
}

// Columns col .. col + 3 of a row, of which those below n exist; col is a multiple of four.
__device__ __forceinline__ void store_four(const Gemm8Params &p, int64_t row, int col, int n, float4 v)
{
    if (col + 4 > n) {
        const float w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int e = 0; e < 4; e++)
            if (col + e < n) store_one(p, row, col + e, w[e]);
    } else if (p.f32) {
        float4 *c = reinterpret_cast<float4 *>(static_cast<float *>(p.c) + row * p.ldc + col);
        if (p.accumulate) {
            const float4 o = *c;
            v.x += o.x; v.y += o.y; v.z += o.z; v.w += o.w;
        }
        *c = v;
    } else {
        *reinterpret_cast<uint2 *>(static_cast<__nv_bfloat16 *>(p.c) + row * p.ldc + col) = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
    }
}

// A box of 32 rows x 128 bytes, COLS columns from col on, leaves an epilogue warp, which has two of them in turn at box_at, side by side on 8 KB.  w: the lane's row of it, value(e): its elements.
template <int COLS, typename F>
__device__ __forceinline__ void send_box(const Gemm8Params &p, const CUtensorMap *map, uint32_t &box_at, const uint32_t *w, int row0, int col, int lane, F value)
{
    if (row0 >= p.m || col >= p.n) return;
    if (col < p.boxed) {
        // The store before the last has read its box.
        if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
        __syncwarp();
        Box16(box_at, lane).put(w);
        fence_async_shared();
        __syncwarp();
        if (lane == 0) {
            if (p.accumulate) tma_reduce_add_2d(map, col, row0, box_at);
            else tma_store_2d(map, col, row0, box_at);
            bulk_commit();
        }
        box_at ^= 4096u;
    }
    if (col + COLS > p.boxed && p.boxed < p.n && row0 + lane < p.m) {
#pragma unroll
        for (int e = 0; e < COLS; e++)
            if (col + e >= p.boxed && col + e < p.n) store_one(p, row0 + lane, col + e, value(e));
    }
    __syncwarp();
}

// The scales of AHEAD blocks from b on, for ROWS rows from m0 on and COLS columns from n0 on: those of rows already times the one of the columns, and the other way round.  All of
// a warp's loads are on their way before the first is written.
template <int MODE, int AHEAD, int ROWS, int COLS>
__device__ __forceinline__ void load_scales(const Gemm8Params &p, int m0, int n0, int b, int b1, float *to)
{
    constexpr int kR = (ROWS + 31) / 32, kC = (COLS + 31) / 32;
    const int lane = threadIdx.x & 31;
    float other[AHEAD], r[AHEAD][kR ? kR : 1], c[AHEAD][kC ? kC : 1];
#pragma unroll
    for (int i = 0; i < AHEAD; i++) {
        const bool there = b + i < b1;
        other[i] = !there || MODE == SCALE_BOTH ? 1.f : MODE == SCALE_ROWS ? p.sb.at(n0, b + i) : p.sa.at(m0, b + i);
#pragma unroll
        for (int j = 0; j < kR; j++) r[i][j] = there && m0 + lane + 32 * j < p.m ? p.sa.at(m0 + lane + 32 * j, b + i) : 0.f;
#pragma unroll
        for (int j = 0; j < kC; j++) c[i][j] = there && lane + 32 * j < COLS && n0 + lane + 32 * j < p.n ? p.sb.at(n0 + lane + 32 * j, b + i) : 0.f;
    }
#pragma unroll
    for (int i = 0; i < AHEAD; i++) {
#pragma unroll
        for (int j = 0; j < kR; j++) to[i * ROWS + lane + 32 * j] = r[i][j] * other[i];
#pragma unroll
        for (int j = 0; j < kC; j++)
            if (lane + 32 * j < COLS) to[AHEAD * ROWS + i * COLS + lane + 32 * j] = c[i][j] * other[i];
    }
}

// ---------------------------------------------------------------------------------------- one tile a cluster

// A tile of 128 x BN whose contraction is shared by the CTAs of a cluster.  Warps: 0 TMA producer, 1 MMA issuer, 2 scales, 4 and up epilogue.
template <int BN, int MODE>
struct Cfg8 {
    static_assert(BN == 16 || BN == 32 || BN == 64 || BN == 128, "tile shapes");
    static constexpr int kEpiWarps = BN == 128 ? 8 : 4, kThreads = 128 + 32 * kEpiWarps;
    static constexpr int kCols = BN == 128 ? 64 : BN;                      // of an epilogue warp
    static constexpr int kABytes = 128 * kBlock8, kBBytes = BN * kBlock8, kStageBytes = kABytes + kBBytes;
    static constexpr int kStages = BN == 128 ? 6 : BN == 64 ? 4 : 5;       // up to 64 columns: two CTAs an SM
    static constexpr int kOperands = kStages * kStageBytes;
    static constexpr int kAccs = BN == 128 ? 2 : 4, kTmemCols = kAccs * BN < 32 ? 32 : kAccs * BN;
    static constexpr int kRowScales = MODE == SCALE_COLS ? 0 : 128, kColScales = MODE == SCALE_ROWS ? 0 : BN;
    static constexpr int kAhead = 4, kScales = kAhead * (kRowScales + kColScales);   // of four blocks; there are two such sets
    // Where the cluster adds up its CTAs' sums they lie in the operands' place: lines along what is consecutive in the output (SCALE_COLS: the tile's 128 rows), 4 more a line than
    // it has, so that neither side's accesses meet in a bank.
    static constexpr int kLine = MODE == SCALE_COLS ? 128 : BN, kLines = MODE == SCALE_COLS ? BN : 128, kPitch = kLine + 4;
    static constexpr int kSmem = 1024 + kOperands + 2 * kScales * 4 + 256;
    static_assert(kStages <= 8, "barriers");
    static_assert(kPitch * kLines * 4 <= kOperands && kSmem <= 227 * 1024, "shared memory budget");
};

template <int BN, int MODE>
__global__ void __launch_bounds__(Cfg8<BN, MODE>::kThreads, BN == 128 ? 1 : 2) gemm8_tile_kernel(const __grid_constant__ Maps8 maps, const __grid_constant__ Gemm8Params p)
{
    using C = Cfg8<BN, MODE>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint8_t *smem_a = smem, *smem_b = smem + C::kStages * C::kABytes;
    float *scales = reinterpret_cast<float *>(smem + C::kOperands);
    uint64_t *bars = reinterpret_cast<uint64_t *>(scales + 2 * C::kScales);
    // [0..7] full, [8..15] empty, [16..19] accumulator full, [20..23] accumulator empty, [24..25] scales full, [26..27] scales empty
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(bars + 28);
    volatile uint32_t *abort_flag = tmem_slot + 1;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t bar_full = smem_u32(bars), bar_empty = smem_u32(bars + 8), bar_acc_full = smem_u32(bars + 16), bar_acc_empty = smem_u32(bars + 20),
                   bar_sc_full = smem_u32(bars + 24), bar_sc_empty = smem_u32(bars + 26);
    const int rank = p.split > 1 ? (int)cluster_ctarank() : 0;

    if (warp == 0) {
        if (lane < 28) mbar_init(smem_u32(bars + lane), (lane >= 20 && lane < 24) || lane >= 26 ? C::kEpiWarps : 1);
        if (lane == 0) *abort_flag = 0u;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    } else if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(C::kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        tcgen05_fence_before();
    } else if (warp == 2 && lane == 0) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.a) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.b) : "memory");
    }
    __syncthreads();
    tcgen05_fence_after();
    const uint32_t tmem = *tmem_slot;
    wait_for_predecessor();   // from here on global memory is read and written

    const uint32_t limit_word = load_global(p.status + 2), withhold = blockIdx.x == 0 ? load_global(p.status + 3) : 0u;
    const uint64_t limit = limit_word != 0u ? limit_word : kWaitLimit;
    const int tile = blockIdx.x / p.split, m0 = tile / p.n_tiles * 128, n0 = tile % p.n_tiles * BN;
    const int b0 = (int)((int64_t)p.blocks * rank / p.split), b1 = (int)((int64_t)p.blocks * (rank + 1) / p.split);   // this CTA's blocks
    constexpr int kSums = C::kCols;
    float sum[kSums];

    if (warp == 0) {
        const bool issuer = elect_one();
        const uint32_t a0 = smem_u32(smem_a), bb0 = smem_u32(smem_b);
        Ring16<C::kStages> ring;
        uint32_t loads = 0;
        for (int b = b0; b < b1; b++, ring.next()) {
            if (!warp_wait(bar_empty + 8 * ring.slot, ring.phase ^ 1u, abort_flag, p.status, limit, 0x100u + ring.slot)) break;
            const uint32_t bar = bar_full + 8 * ring.slot;
            expect_tx_if(bar, C::kStageBytes, issuer);
            tma_load_if<false>(a0 + ring.slot * C::kABytes, &maps.a, b * kBlock8, m0, bar, issuer && (withhold == 0u || ++loads != withhold));
            tma_load_if<false>(bb0 + ring.slot * C::kBBytes, &maps.b, b * kBlock8, n0, bar, issuer);
        }
    } else if (warp == 1) {
        const bool issuer = elect_one();
        const uint32_t idesc = instr_desc8<1>(BN), a_desc = (uint32_t)smem_desc_sw128(smem_u32(smem_a)), b_desc = (uint32_t)smem_desc_sw128(smem_u32(smem_b));
        constexpr uint32_t desc_hi = (1024 >> 4) | (1u << 14) | (2u << 29);
        Ring16<C::kStages> ring;
        Ring16<C::kAccs> acc;
        for (int b = b0; b < b1; b++, ring.next(), acc.next()) {
            if (!warp_wait(bar_acc_empty + 8 * acc.slot, acc.phase ^ 1u, abort_flag, p.status, limit, 0x200u)) break;
            if (!warp_wait(bar_full + 8 * ring.slot, ring.phase, abort_flag, p.status, limit, 0x300u + ring.slot)) break;
            tcgen05_fence_after();
#pragma unroll
            for (int j = 0; j < 4; j++)
                tcgen05_mma_f8<1>(tmem + acc.slot * BN, a_desc + ((ring.slot * C::kABytes + 32 * j) >> 4), b_desc + ((ring.slot * C::kBBytes + 32 * j) >> 4), desc_hi, idesc, j > 0, issuer);
            tcgen05_commit_if<1>(bar_empty + 8 * ring.slot, issuer);
            tcgen05_commit_if<1>(bar_acc_full + 8 * acc.slot, issuer);
        }
    } else if (warp == 2) {
        // The scales of four blocks at a time: those of rows already times the one of the columns, and the other way round.
        Ring16<2> set;
        for (int b = b0; b < b1; b += C::kAhead, set.next()) {
            if (!warp_wait(bar_sc_empty + 8 * set.slot, set.phase ^ 1u, abort_flag, p.status, limit, 0x400u)) break;
            float *to = scales + set.slot * C::kScales;
            load_scales<MODE, C::kAhead, C::kRowScales, C::kColScales>(p, m0, n0, b, b1, to);
            __syncwarp();
            if (lane == 0) mbar_arrive(bar_sc_full + 8 * set.slot);
        }
    } else if (warp >= 4) {
        const int quarter = warp & 3, half = (warp - 4) >> 2;
#pragma unroll
        for (int i = 0; i < kSums; i++) sum[i] = 0.f;
        Ring16<C::kAccs> acc;
        Ring16<2> set;
        for (int b = b0; b < b1; b++, acc.next()) {
            const int i = (b - b0) % C::kAhead;
            if (i == 0 && !warp_wait(bar_sc_full + 8 * set.slot, set.phase, abort_flag, p.status, limit, 0x500u)) break;
            if (!warp_wait(bar_acc_full + 8 * acc.slot, acc.phase, abort_flag, p.status, limit, 0x600u)) break;
            tcgen05_fence_after();
            const uint32_t from = smem_u32(scales + set.slot * C::kScales);
            const float row = C::kRowScales ? load_scale(from + 4 * (i * C::kRowScales + 32 * quarter + lane)) : 1.f;
            add_block<MODE, C::kCols>(sum, tmem + acc.slot * BN + half * C::kCols + ((uint32_t)(32 * quarter) << 16), row, from + 4 * (C::kAhead * C::kRowScales + i * C::kColScales + half * C::kCols), [&] {
                tcgen05_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar_acc_empty + 8 * acc.slot);
            });
            __syncwarp();
            if (i == C::kAhead - 1 || b == b1 - 1) {
                if (lane == 0) mbar_arrive(bar_sc_empty + 8 * set.slot);
                set.next();
            }
        }
        const int in = 32 * quarter + lane;   // row of the tile
        if (p.split == 1) {
            if (m0 + in < p.m && *abort_flag == 0u) {
                check_sums(p, m0 + in, n0 + half * C::kCols, sum);
#pragma unroll
                for (int c = 0; c < C::kCols; c += 16) {
                    float v[16];
#pragma unroll
                    for (int e = 0; e < 16; e++) v[e] = sum[c + e];
                    const int col = n0 + half * C::kCols + c;
                    if (MODE != SCALE_COLS) store_row16(p, m0 + in, col, p.n, v);
                    else
#pragma unroll
                        for (int e = 0; e < 16; e++)
                            if (col + e < p.n) store_one(p, col + e, m0 + in, v[e]);
                }
            }
        } else {
            // All MMAs of this CTA are done, so its operands' place is free.
            float *mine = reinterpret_cast<float *>(smem);
            if (MODE == SCALE_COLS) {
#pragma unroll
                for (int c = 0; c < C::kCols; c++) mine[(half * C::kCols + c) * C::kPitch + in] = sum[c];
            } else {
#pragma unroll
                for (int c = 0; c < C::kCols; c += 4) *reinterpret_cast<float4 *>(mine + in * C::kPitch + half * C::kCols + c) = make_float4(sum[c], sum[c + 1], sum[c + 2], sum[c + 3]);
            }
        }
    }
    __syncwarp();
    if (p.split > 1) {
        cluster_arrive();
        cluster_wait();
        // This CTA's share of the tile: the sums of all CTAs, in their order.
        if (*abort_flag == 0u) {
            constexpr int kFours = C::kLine / 4 * C::kLines;
            const int e0 = (int)((int64_t)kFours * rank / p.split), e1 = (int)((int64_t)kFours * (rank + 1) / p.split);
            for (int e = e0 + threadIdx.x; e < e1; e += C::kThreads) {
                const int line = e / (C::kLine / 4), at = e % (C::kLine / 4) * 4;
                const int64_t row = MODE == SCALE_COLS ? n0 + line : m0 + line;      // of the output
                const int col = MODE == SCALE_COLS ? m0 + at : n0 + at, rows = MODE == SCALE_COLS ? p.n : p.m, cols = MODE == SCALE_COLS ? p.m : p.n;
                if (row >= rows || col >= cols) continue;
                const uint32_t from = smem_u32(smem) + (line * C::kPitch + at) * 4;
                float4 x[8];   // on their way together
#pragma unroll
                for (int r = 0; r < 8; r++)
                    if (r < p.split)
                        asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(x[r].x), "=f"(x[r].y), "=f"(x[r].z), "=f"(x[r].w) : "r"(cluster_addr(from, r)) : "memory");
                float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int r = 0; r < 8; r++)
                    if (r < p.split) { v.x += x[r].x; v.y += x[r].y; v.z += x[r].z; v.w += x[r].w; }
                if (!((v.x + v.y) * 0.f + (v.z + v.w) * 0.f == 0.f))   // (a sum of two may be infinite where they are not)
                    v = careful_four(p, MODE == SCALE_COLS ? col : (int)row, MODE == SCALE_COLS ? (int)row : col, MODE == SCALE_COLS, v);
                store_four(p, row, col, cols, v);
            }
        }
        __syncwarp();
        cluster_arrive();
        cluster_wait();
    }
    // Where a wait has run out, copies and MMAs may still be under way: they take microseconds, a millisecond is left to them.
    if (*abort_flag != 0u)
        for (int i = 0; i < 64; i++) __nanosleep(16000);
    tcgen05_fence_before();
    __syncthreads();
    if (warp == 1) {
        tcgen05_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(C::kTmemCols) : "memory");
    }
}

// ---------------------------------------------------------------------------------------- persistent: many tiles

// A wait that mostly need not wait: one look, which is sooner done than a suspending poll.  (64 looks before it are slower: 8192 x 4096 x 4096 138 -> 146 us.)
// CLUSTER: another CTA's arrivals complete the barrier (1 % of a forward product of 16384 rows).
template <bool CLUSTER>
__device__ __forceinline__ bool seen_or_wait(uint32_t bar, uint32_t parity, volatile uint32_t *abort_flag, uint32_t *status, uint64_t limit, uint32_t where)
{
    return __all_sync(0xFFFFFFFFu, mbar_look<CLUSTER>(bar, parity)) || warp_wait<CLUSTER>(bar, parity, abort_flag, status, limit, where);
}

// Single CTAs with tiles of 128 x 128, or pairs (cta_group::2) with tiles of 256 x 256 of which each CTA has 128 rows and loads half of B's: 32 KB of operands then feed
// 2 x 128 x 256 x 128 operations, in 512 cycles of the tensor core, which is what L2 delivers at best.  Warps: 0 TMA producer, 1 MMA issuer, 2 scales, 3 caller, 4 and up epilogue, each
// with 32 rows x half of the columns: with 128 sums a thread they need more registers than 12 warps' share, which the others give.
// What counts is how soon an accumulator is read and handed back, since a pair has two and a block's MMAs take 512 cycles.  Waiting for an mbarrier takes a warp some 300 cycles even where it has completed, and the
// polls of eight of them hold up everything else that goes through shared memory: only the caller polls, and lets the epilogue go through named barriers, one for each half of its
// warps and accumulator.
template <int CTAS, int MODE>
struct CfgP {
    static constexpr int kBN = 128 * CTAS, kThreads = 384;
    static constexpr int kCols = 64 * CTAS;
    static constexpr int kABytes = 128 * kBlock8, kBBytes = 128 * kBlock8, kStageBytes = kABytes + kBBytes;   // of a CTA
    // Two boxes an epilogue warp at the price of a stage: 8192 x 8192 x 1024 89.6 -> 84.8 us, 16384 x 11008 x 4096 688 -> 679.
    static constexpr int kStages = 4, kBoxes = 2;
    static constexpr int kOperands = kStages * kStageBytes;
    static constexpr int kAccs = 4 / CTAS, kTmemCols = 512;
    static constexpr int kCalled = 128 + 32;                               // threads of a named barrier: half of the epilogue, and the caller
    static constexpr int kColScales = MODE == SCALE_BOTH ? kBN : 0;        // else one for each block of 128 columns
    static constexpr int kAhead = 4, kScales = kAhead * (128 + kBN);
    static constexpr int kStaging = 4096 * kBoxes, kAlign = kStaging;      // of an epilogue warp: boxes of 32 rows x 128 bytes, on a multiple of both boxes' size, wherever shared memory begins
    static constexpr int kSmem = kAlign + kOperands + 8 * kStaging + 2 * kScales * 4 + 512;
    static constexpr int kFewRegs = 104, kManyRegs = 200;                  // 88 are too few for the scales' warp with both: 438 -> 421 us
    static_assert(128 * kFewRegs + 256 * kManyRegs <= 384 * 168, "registers: what the epilogue takes is what the other warps give");
    static_assert(kBoxes == 2 && kAlign % 1024 == 0 && kOperands % kAlign == 0, "one box from the other: bit 12 of its address");
    static_assert(kSmem <= 227 * 1024 && kStages <= 8, "shared memory budget, barriers");
};
struct MapsP {
    CUtensorMap a, b, b_half, out;
};

// What an epilogue warp of the persistent kernel works with.
template <int ACCS>
struct Epilogue8 {
    uint32_t tmem, scales, lead_empty, acc_empty, sc_empty, box_at;
    volatile uint32_t *abort_flag;
    int quarter, half, lane, rank;
    Ring16<ACCS> acc;
    Ring16<2> set;
};

// A warp's part of a tile, 32 rows x COLS columns.  false: a wait of another warp has run out.
template <int CTAS, int MODE, int COLS>
__device__ __forceinline__ bool tile_out(const Gemm8Params &p, const MapsP &maps, Epilogue8<CfgP<CTAS, MODE>::kAccs> &w, int m0, int n0)
{
    using C = CfgP<CTAS, MODE>;
    float sum[COLS];
#pragma unroll
    for (int i = 0; i < COLS; i++) sum[i] = 0.f;
    float row = 0.f, top = 0.f;   // top: the largest factor of the row's sums.  (Short contractions: 16384 x 4096 over 256 57 us without it, 55 with.  Where the columns' scales differ, too, it costs 6 %.)
    for (int b = 0; b < p.blocks; b++, w.acc.next()) {
        const int i = b % C::kAhead;
        const uint32_t from = w.scales + w.set.slot * C::kScales * 4;
        asm volatile("bar.sync %0, %1;" ::"r"(1 + w.half * C::kAccs + w.acc.slot), "n"(C::kCalled) : "memory");
        const uint32_t aborted = *w.abort_flag;
        auto goes_on = [&] {
            if (__all_sync(0xFFFFFFFFu, aborted == 0u)) return true;
            w.acc.next();   // whoever of this half did not see it yet waits at the next barrier, and sees it behind that
            asm volatile("bar.arrive %0, %1;" ::"r"(1 + w.half * C::kAccs + w.acc.slot), "n"(C::kCalled) : "memory");
            return false;
        };
        auto row_scale = [&](int i) {
            const float f = load_scale(from + 4 * (i * 128 + 32 * w.quarter + w.lane));
            return MODE == SCALE_ROWS ? f * load_scale(from + 4 * (C::kAhead * 128 + i * CTAS + w.half * COLS / 128)) : f;
        };
        // Where the columns' scales make the additions the longest part, nothing is waited for ahead of them: the flag is looked at behind them, and the next block's scale is loaded
        // beside them.  Weight gradient of 4096 x 4096 over 16384 rows 412 -> 362 us for the two together, nothing for either alone; with one scale for all columns slower, 682 -> 691.
        if (MODE == SCALE_ROWS && !goes_on()) return false;
        tcgen05_fence_after();
        float next = 0.f;
        if (MODE == SCALE_ROWS || i == 0) row = row_scale(i);
        if (MODE == SCALE_BOTH) next = row_scale(min(i + 1, C::kAhead - 1));
        if (MODE == SCALE_ROWS) top = fmaxf(top, fabsf(row));
        add_block<MODE, COLS>(sum, w.tmem + w.acc.slot * C::kBN + w.half * COLS + ((uint32_t)(32 * w.quarter) << 16), row, from + 4 * (C::kAhead * 128 + i * C::kColScales + w.half * COLS), [&] {
            tcgen05_fence_before();
            __syncwarp();
            if (w.lane == 0) {
                // Of the default scope, as in the other products' pairs, on the assumption that is written beside this function.  Released to the cluster, the arrival
                // would wait for all that the warp has under way: 16384 x 11008 x 4096 663 -> 1268 us.
                if (w.rank != 0) mbar_arrive_cluster(w.lead_empty + 8 * w.acc.slot);
                else mbar_arrive(w.acc_empty + 8 * w.acc.slot);
            }
        });
        if (MODE == SCALE_BOTH) {
            row = next;
            if (!goes_on()) return false;
        }
        __syncwarp();
        if (i == C::kAhead - 1 || b == p.blocks - 1) {
            if (w.lane == 0) mbar_arrive(w.sc_empty + 8 * w.set.slot);
            w.set.next();
        }
    }
    if (MODE == SCALE_BOTH || top > 0x1.fffffep127f) check_sums(p, m0 + 32 * w.quarter + w.lane, n0 + w.half * COLS, sum);
    // Boxes of 32 rows x 128 bytes; a row's last bytes that are no whole 16 by themselves.
    const int row0 = m0 + 32 * w.quarter, col0 = n0 + w.half * COLS, lane = w.lane;
    if (p.f32) {
#pragma unroll
        for (int c = 0; c < COLS; c += 32) {
            float v[32];
#pragma unroll
            for (int e = 0; e < 32; e++) v[e] = sum[c + e];
            send_box<32>(p, &maps.out, w.box_at, reinterpret_cast<const uint32_t *>(v), row0, col0 + c, lane, [&](int e) { return v[e]; });
        }
    } else {
#pragma unroll
        for (int c = 0; c < COLS; c += 64) {
            uint32_t v[32];
#pragma unroll
            for (int e = 0; e < 32; e++) v[e] = pack_bf16(sum[c + 2 * e], sum[c + 2 * e + 1]);
            send_box<64>(p, &maps.out, w.box_at, v, row0, col0 + c, lane, [&](int e) { return __uint_as_float((e & 1) ? v[e >> 1] & 0xFFFF0000u : v[e >> 1] << 16); });
        }
    }
    return true;
}

template <int CTAS, int MODE>
__global__ void __launch_bounds__(384, 1) gemm8_kernel(const __grid_constant__ MapsP maps, const __grid_constant__ Gemm8Params p)
{
    using C = CfgP<CTAS, MODE>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + C::kAlign - 1) & ~(uintptr_t)(C::kAlign - 1));
    uint8_t *smem_a = smem, *smem_b = smem + C::kStages * C::kABytes, *smem_boxes = smem + C::kOperands;
    float *scales = reinterpret_cast<float *>(smem_boxes + 8 * C::kStaging);
    uint64_t *bars = reinterpret_cast<uint64_t *>(scales + 2 * C::kScales);
    // [0..7] full, [8..15] empty, [16..19] accumulator full, [20..23] accumulator empty, [24..25] scales full, [26..27] scales empty
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(bars + 28);
    volatile uint32_t *abort_flag = tmem_slot + 1;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t bar_full = smem_u32(bars), bar_empty = smem_u32(bars + 8), bar_acc_full = smem_u32(bars + 16), bar_acc_empty = smem_u32(bars + 20),
                   bar_sc_full = smem_u32(bars + 24), bar_sc_empty = smem_u32(bars + 26);
    const int rank = CTAS == 2 ? (int)cluster_ctarank() : 0;

    if (warp == 0) {
        if (lane < 28) mbar_init(smem_u32(bars + lane), lane >= 20 && lane < 24 ? 8 * CTAS : lane >= 26 ? 8 : 1);
        if (lane == 0) *abort_flag = 0u;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    } else if (warp == 1) {
        if (CTAS == 2) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(C::kTmemCols) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(C::kTmemCols) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        }
        tcgen05_fence_before();
    } else if (warp == 2 && lane == 0) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.a) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.b) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.out) : "memory");
    }
    __syncthreads();
    if (CTAS == 2) { cluster_arrive(); cluster_wait(); }
    tcgen05_fence_after();
    const uint32_t tmem = *tmem_slot;
    wait_for_predecessor();   // from here on global memory is read and written

    const uint32_t limit_word = load_global(p.status + 2), withhold = blockIdx.x == 0 ? load_global(p.status + 3) : 0u;
    const uint64_t limit = limit_word != 0u ? limit_word : kWaitLimit;
    const int step = gridDim.x / CTAS, blocks = p.blocks;
    // Bands of kRaster16 rows of tiles, whose A rows stay in L2 while the columns go by.
    auto place = [&](int piece, int &m0, int &n0) {
        const int second = CTAS == 2 ? max(piece - p.whole, 0) : 0, tile = piece - second + second / 2;
        const int per_band = kRaster16 * p.n_tiles, band = tile / per_band, top = band * kRaster16, h = min(kRaster16, p.m_tiles - top), rem = tile - band * per_band;
        n0 = rem / h * C::kBN + second % 2 * (C::kBN / 2);
        m0 = (top + rem % h) * (128 * CTAS) + rank * 128;
    };

    if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::kFewRegs));
        if (warp == 0) {
            const bool issuer = elect_one();
            const uint32_t a0 = smem_u32(smem_a), b0 = smem_u32(smem_b), lead = CTAS == 2 ? cluster_addr(bar_full, 0) : bar_full;
            Ring16<C::kStages> ring;
            uint32_t loads = 0, issued = 0;
            bool ok = true;
            for (int tile = blockIdx.x / CTAS; ok && tile < p.pieces; tile += step) {
                int m0, n0;
                place(tile, m0, n0);
                const bool part = CTAS == 2 && tile >= p.whole;
                const CUtensorMap *const map_b = part ? &maps.b_half : &maps.b;
                const uint32_t bytes = part ? (C::kABytes + C::kBBytes / 2) * CTAS : C::kStageBytes * CTAS;
                if (CTAS == 2) n0 += rank * (part ? 64 : 128);
                for (int b = 0; b < blocks; b++, ring.next()) {
                    if (!warp_wait(bar_empty + 8 * ring.slot, ring.phase ^ 1u, abort_flag, p.status, limit, 0x100u + ring.slot)) { ok = false; break; }
                    issued++;
                    const uint32_t bar = lead + 8 * ring.slot, at = ring.slot * C::kABytes;
                    expect_tx_if(bar_full + 8 * ring.slot, bytes, issuer && rank == 0);
                    tma_load_if<CTAS == 2>(a0 + at, &maps.a, b * kBlock8, m0, bar, issuer && (withhold == 0u || ++loads != withhold));
                    tma_load_if<CTAS == 2>(b0 + at, map_b, b * kBlock8, n0, bar, issuer);
                }
            }
            // The MMAs' last reports reach this CTA's barriers while it is still there.
            for (uint32_t i = 0; ok && i < C::kStages; i++, ring.next())
                if (issued >= C::kStages - i) ok = warp_wait(bar_empty + 8 * ring.slot, ring.phase ^ 1u, abort_flag, p.status, limit, 0x700u + ring.slot);
        } else if (warp == 1 && rank == 0) {
            const bool issuer = elect_one();
            const uint32_t a_desc = (uint32_t)smem_desc_sw128(smem_u32(smem_a)), b_desc = (uint32_t)smem_desc_sw128(smem_u32(smem_b));
            constexpr uint32_t desc_hi = (1024 >> 4) | (1u << 14) | (2u << 29);
            Ring16<C::kStages> ring;
            Ring16<C::kAccs> acc;
            bool ok = true;
            for (int tile = blockIdx.x / CTAS; ok && tile < p.pieces; tile += step) {
                const uint32_t idesc = instr_desc8<CTAS>(CTAS == 1 || tile < p.whole ? C::kBN : C::kBN / 2);
                for (int b = 0; b < blocks; b++, ring.next(), acc.next()) {
                    ok = seen_or_wait<false>(bar_full + 8 * ring.slot, ring.phase, abort_flag, p.status, limit, 0x300u + ring.slot) &&
                         seen_or_wait<CTAS == 2>(bar_acc_empty + 8 * acc.slot, acc.phase ^ 1u, abort_flag, p.status, limit, 0x200u);
                    if (!ok) break;
                    tcgen05_fence_after();
#pragma unroll
                    for (int j = 0; j < 4; j++)
                        tcgen05_mma_f8<CTAS>(tmem + acc.slot * C::kBN, a_desc + ((ring.slot * C::kABytes + 32 * j) >> 4), b_desc + ((ring.slot * C::kBBytes + 32 * j) >> 4), desc_hi, idesc, j > 0,
                                             issuer);
                    tcgen05_commit_if<CTAS>(bar_acc_full + 8 * acc.slot, issuer);
                    tcgen05_commit_if<CTAS>(bar_empty + 8 * ring.slot, issuer);
                }
            }
        } else if (warp == 2) {
            // The scales of four blocks at a time, loaded while the set before waits for its place.
            constexpr int kR = 4, kC = C::kColScales / 32;
            Ring16<2> set;
            bool ok = true;
            for (int tile = blockIdx.x / CTAS; ok && tile < p.pieces; tile += step) {
                int m0, n0;
                place(tile, m0, n0);
                for (int b = 0; b < blocks; b += C::kAhead, set.next()) {
                    float4 r[kR], c[kC ? kC : 1];
                    const float4 none = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                    for (int j = 0; j < kR; j++) r[j] = m0 + lane + 32 * j < p.m ? p.sa.four(m0 + lane + 32 * j, b, blocks) : none;
#pragma unroll
                    for (int j = 0; j < kC; j++) c[j] = n0 + lane + 32 * j < p.n ? p.sb.four(n0 + lane + 32 * j, b, blocks) : none;
                    float one = 0.f;   // lane: a block of the contraction and one of the columns
                    if (MODE == SCALE_ROWS && lane < C::kAhead * CTAS && b + lane / CTAS < blocks && n0 + 128 * (lane % CTAS) < p.n) one = p.sb.at(n0 + 128 * (lane % CTAS), b + lane / CTAS);
                    ok = warp_wait(bar_sc_empty + 8 * set.slot, set.phase ^ 1u, abort_flag, p.status, limit, 0x400u);
                    if (!ok) break;
                    float *to = scales + set.slot * C::kScales;
#pragma unroll
                    for (int j = 0; j < kR; j++) {
                        float *at = to + lane + 32 * j;
                        at[0] = r[j].x; at[128] = r[j].y; at[256] = r[j].z; at[384] = r[j].w;
                    }
#pragma unroll
                    for (int j = 0; j < kC; j++) {
                        float *at = to + C::kAhead * 128 + lane + 32 * j;
                        at[0] = c[j].x; at[C::kColScales] = c[j].y; at[2 * C::kColScales] = c[j].z; at[3 * C::kColScales] = c[j].w;
                    }
                    if (MODE == SCALE_ROWS && lane < C::kAhead * CTAS) to[C::kAhead * 128 + lane] = one;
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar_sc_full + 8 * set.slot);
                }
            }
        } else if (warp == 3) {
            Ring16<C::kAccs> acc;
            Ring16<2> set;
            bool ok = true;
            for (int tile = blockIdx.x / CTAS; ok && tile < p.pieces; tile += step)
                for (int b = 0; ok && b < blocks; b++, acc.next()) {
                    if (b % C::kAhead == 0) {
                        ok = warp_wait(bar_sc_full + 8 * set.slot, set.phase, abort_flag, p.status, limit, 0x500u);
                        set.next();
                    }
                    ok = ok && warp_wait(bar_acc_full + 8 * acc.slot, acc.phase, abort_flag, p.status, limit, 0x600u);
                    // Where a wait has run out, the abort flag is set: the epilogue is called all the same, and leaves.
                    asm volatile("bar.arrive %0, %1;" ::"r"(1 + acc.slot), "n"(C::kCalled) : "memory");
                    asm volatile("bar.arrive %0, %1;" ::"r"(1 + C::kAccs + acc.slot), "n"(C::kCalled) : "memory");
                }
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(C::kManyRegs));
        const int quarter = warp & 3, half = (warp - 4) >> 2;
        Epilogue8<C::kAccs> e = {tmem, smem_u32(scales), CTAS == 2 ? cluster_addr(bar_acc_empty, 0) : bar_acc_empty, bar_acc_empty, bar_sc_empty, smem_u32(smem_boxes) + (warp - 4) * C::kStaging, abort_flag,
                                 quarter, half, lane, rank};
        for (int tile = blockIdx.x / CTAS; tile < p.pieces; tile += step) {
            int m0, n0;
            place(tile, m0, n0);
            bool ok;
            if (CTAS == 1 || tile < p.whole) ok = tile_out<CTAS, MODE, C::kCols>(p, maps, e, m0, n0);
            else ok = tile_out<CTAS, MODE, 64>(p, maps, e, m0, n0);
            if (!ok) break;
        }
        boxes_free(lane);   // the stores have read shared memory; what they write is there when the grid has completed
    }
    // Shared memory and tensor memory stay until all roles, of both CTAs of a pair, have done with them.  Where a wait has run out, copies and MMAs may still be under
    // way: they take microseconds, a millisecond is left to them.
    __syncwarp();
    if (*abort_flag != 0u) {
        if (CTAS == 2 && lane == 0)   // the other CTA is told
            asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(cluster_addr(smem_u32(const_cast<const uint32_t *>(abort_flag)), 1 - rank)), "r"(1u) : "memory");
        for (int i = 0; i < 64; i++) __nanosleep(16000);
    }
    tcgen05_fence_before();
    __syncthreads();
    if (CTAS == 2) { cluster_arrive(); cluster_wait(); }
    if (warp == 1) {
        tcgen05_fence_after();
        if (CTAS == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(C::kTmemCols) : "memory");
        else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(C::kTmemCols) : "memory");
    }
}

// ---------------------------------------------------------------------------------------- host side

const int64_t kMaxDim8 = 0x7FFFFFFF - 4096;

// An operand: codes [rows, cols], rows along the contraction.
struct Operand8 {
    const uint8_t *q;
    int64_t rows, cols, ld;
    Scales8 scales;
};
bool make_map8(CUtensorMap *map, const Operand8 &o, int box_rows)
{
    const cuuint64_t dims[2] = {(cuuint64_t)o.cols, (cuuint64_t)o.rows};
    const cuuint64_t strides[1] = {(cuuint64_t)o.ld};
    const cuuint32_t box[2] = {(cuuint32_t)kBlock8, (cuuint32_t)box_rows};
    return encode_tiled(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<uint8_t *>(o.q), dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B);
}

void codes_of(const Operand8 &a, const Operand8 &b, Gemm8Params &p)
{
    p.qa = a.q;
    p.qb = b.q;
    p.lda = a.ld;
    p.ldb = b.ld;
    p.k = a.cols;
}

template <typename K>
bool allow_smem(K kernel, int bytes, std::atomic<bool> (&set)[kMaxDevices], int dev)
{
    if (set[dev].load(std::memory_order_relaxed)) return true;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) {
        cudaGetLastError();
        return false;
    }
    set[dev].store(true, std::memory_order_relaxed);
    return true;
}

// What launches a tile kernel in clusters of `split`; attr: two of them.
template <int BN, int MODE>
cudaLaunchConfig_t tile_config(int64_t ctas, int split, cudaLaunchAttribute *attr, cudaStream_t stream)
{
    using C = Cfg8<BN, MODE>;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ctas);
    cfg.blockDim = dim3(C::kThreads);
    cfg.dynamicSmemBytes = C::kSmem;
    cfg.stream = stream;
    cfg.attrs = attr;
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)split;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.numAttrs = split > 1 ? 2 : 1;
    return cfg;
}

// Clusters of `split` CTAs of the 128 x 128 tile kernel that run at once: they do not cross the GPU's partitions, so fewer CTAs of large ones do (16 clusters of eight ran one behind the other: 200 x 1024 x
// 2816 13.8 us, in clusters of six 8.3).
template <int MODE>
int clusters_at_once(int split, int dev)
{
    static std::atomic<int> known[kMaxDevices][9];
    int n = known[dev][split].load(std::memory_order_relaxed);
    if (n == 0) {
        cudaLaunchAttribute attr[2];
        cudaLaunchConfig_t cfg = tile_config<128, MODE>(split, split, attr, nullptr);
        n = sm_count(dev) / split;
        int found = 0;
        if (split > 1) {
            if (cudaOccupancyMaxActiveClusters(&found, gemm8_tile_kernel<128, MODE>, &cfg) == cudaSuccess && found > 0) n = found;
            else cudaGetLastError();
        }
        known[dev][split].store(n, std::memory_order_relaxed);
    }
    return n;
}

template <int BN, int MODE>
fp4q_status launch_tiles(const Operand8 &a, const Operand8 &b, Gemm8Params p, int split, cudaStream_t stream)
{
    using C = Cfg8<BN, MODE>;
    Maps8 maps;
    if (!make_map8(&maps.a, a, 128) || !make_map8(&maps.b, b, BN)) return FP4Q_ERR_CUDA;
    const int dev = current_device();
    static std::atomic<bool> set[kMaxDevices];
    if (dev < 0 || !allow_smem(gemm8_tile_kernel<BN, MODE>, C::kSmem, set, dev)) return FP4Q_ERR_CUDA;
    p.n_tiles = (int32_t)ceil_div(p.n, BN);
    p.split = split;
    codes_of(a, b, p);
    const int64_t ctas = ceil_div(p.m, 128) * p.n_tiles * split;
    if (ctas > 0x7FFFFFFF) return FP4Q_ERR_UNSUPPORTED;
    cudaLaunchAttribute attr[2];
    const cudaLaunchConfig_t cfg = tile_config<BN, MODE>(ctas, split, attr, stream);
    return launched(cudaLaunchKernelEx(&cfg, gemm8_tile_kernel<BN, MODE>, maps, p));
}

template <int CTAS, int MODE>
fp4q_status launch_persistent(const Operand8 &a, const Operand8 &b, Gemm8Params p, cudaStream_t stream)
{
    using C = CfgP<CTAS, MODE>;
    MapsP maps;
    if (!make_map8(&maps.a, a, 128) || !make_map8(&maps.b, b, 128)) return FP4Q_ERR_CUDA;
    const int64_t bytes = p.f32 ? 4 : 2;
    {
        const cuuint64_t dims[2] = {(cuuint64_t)p.boxed, (cuuint64_t)p.m};
        const cuuint64_t strides[1] = {(cuuint64_t)(p.ldc * bytes)};
        const cuuint32_t box[2] = {(cuuint32_t)(128 / bytes), 32u};
        if (!encode_tiled(&maps.out, p.f32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_UINT16, 2, p.c, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B,
                          CU_TENSOR_MAP_L2_PROMOTION_L2_256B))
            return FP4Q_ERR_CUDA;
    }
    const int dev = current_device();
    static std::atomic<bool> set[kMaxDevices];
    if (dev < 0 || !allow_smem(gemm8_kernel<CTAS, MODE>, C::kSmem, set, dev)) return FP4Q_ERR_CUDA;
    codes_of(a, b, p);
    p.m_tiles = (int32_t)ceil_div(p.m, 128 * CTAS);
    p.n_tiles = (int32_t)ceil_div(p.n, C::kBN);
    const int64_t tiles = (int64_t)p.m_tiles * p.n_tiles, slots = sm_count(dev) / CTAS;
    if (tiles > 0x3FFFFFFF) return FP4Q_ERR_UNSUPPORTED;
    // A last round for which half of the pairs suffice is computed in halves of tiles, whose blocks take 0.7 of a whole one's time: weight gradient of 4096 x 4096 over 16384 rows 486 -> 458 us (before its
    // additions were faster), 4096 x 4096 x 4096 78 -> 75.  (Halves of a single CTA's tiles take as long as the whole.)
    const int64_t last = tiles % slots;
    p.whole = (int32_t)(CTAS == 2 && 2 * last <= slots ? tiles - last : tiles);
    p.pieces = (int32_t)(2 * tiles - p.whole);
    if (p.whole != tiles && !make_map8(&maps.b_half, b, 64)) return FP4Q_ERR_CUDA;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[2];
    cfg.gridDim = dim3((unsigned)(CTAS * std::min<int64_t>(p.pieces, slots)));
    cfg.blockDim = dim3(C::kThreads);
    cfg.dynamicSmemBytes = C::kSmem;
    cfg.stream = stream;
    cfg.attrs = attr;
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = CTAS;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.numAttrs = CTAS == 2 ? 2 : 1;
    return launched(cudaLaunchKernelEx(&cfg, gemm8_kernel<CTAS, MODE>, maps, p));
}

// How a product is computed, by estimated time.  Rounds of tiles: a block takes 0.365 us in a single CTA's tile of the persistent kernel (0.47 where both operands' scales differ inside a tile), 0.55 (0.71) in a
// pair's, four times as large, and a tile 1.3 or 2.2 us beside its blocks; 0.40 (0.58) and 2 us in a tile of a CTA to itself, whose contraction a cluster may share for about 3 us.
// (4096 x 4096 x 4096: pairs 70 us, single CTAs 82; 1999 x 2731 over 1003 16.4 and 17.6; 512 x 4096 x 4096 19 and 12.5; 128 x 4096 x 4096 in clusters of four 9, single CTAs 12.5;
// a weight gradient of 256 x 256 over 16384 rows in clusters of eight 15, single CTAs 72.)
struct Plan8 {
    int pairs = 0, split = 1;   // pairs: 2, single CTAs: 1, clusters of `split` CTAs with a tile: 0
    Plan8(int64_t m, int64_t n, int64_t blocks, bool both, bool boxes, int dev)
    {
        const double each = both ? 0.58 : 0.40;
        double least = 1e30;
        auto consider = [&](double us, int p, int s) {
            if (us < least) { least = us; pairs = p; split = s; }
        };
        const int64_t tiles = ceil_div(m, 128) * ceil_div(n, 128);
        for (int64_t s = 1; s <= 8 && (s == 1 || s * 2 <= blocks); s++)
            consider((double)ceil_div(tiles, both ? clusters_at_once<SCALE_BOTH>((int)s, dev) : clusters_at_once<SCALE_ROWS>((int)s, dev)) * ((double)ceil_div(blocks, s) * each + 2.0) +
                         (s > 1 ? 2.5 + 0.15 * (double)s : 0.0), 0, (int)s);
        if (!boxes) return;
        const int64_t sms = sm_count(dev), slots = sms / 2;
        consider((double)ceil_div(tiles, sms) * ((double)blocks * (both ? 0.47 : 0.365) + 1.3), 1, 1);
        const int64_t large = ceil_div(m, 256) * ceil_div(n, 256), last = large % slots;
        consider(((double)(large / slots) + (last == 0 ? 0.0 : 2 * last <= slots ? 0.7 : 1.0)) * ((double)blocks * (both ? 0.71 : 0.55) + 2.2), 2, 1);
    }
};

// SCALE_ROWS: C[m, n] with A in 1D blocks and B in square ones; both: both in 1D blocks.
fp4q_status product8(const Operand8 &a, const Operand8 &b, Gemm8Params p, bool both, cudaStream_t stream)
{
    p.m = (int32_t)a.rows;
    p.n = (int32_t)b.rows;
    p.blocks = (int32_t)ceil_div(a.cols, kBlock8);
    p.sa = a.scales;
    p.sb = b.scales;
    const int dev = current_device();
    if (dev < 0) return FP4Q_ERR_CUDA;
    if (!both && a.rows <= 64) {   // few tokens: B's rows become the tile's 128 rows, of which an SM has room for two tiles; B is read at memory's pace when all SMs read
        std::swap(p.m, p.n);
        std::swap(p.sa, p.sb);
        const int64_t tiles = ceil_div(b.rows, 128), sms = sm_count(dev);
        // CTAs of a tile: one an SM for few tiles, as far as clusters reach all SMs, two an SM for more, which clusters of over four leave idle.  One token, contractions of 4096 and 11008: 24 tiles
        // by 5 5.8 and 9.0 us, by 7 6.5 and 9.3; 32 by 4 6.2 and 10.1, by 5 6.8 and 10.4; 40 by 4 7.4 and 11.9, by 7 10.5 and 15.3; 64 by 3 8.7 and 15.2, by 4 8.2 and 13.4, by 5 11.6 and
        // 19.0; 148 by 2 11.6 and 36.1, by 1 12.2 and 37.1.
        int64_t each = tiles <= 32 ? 7 * sms / 8 / tiles : std::min<int64_t>(4, 2 * sms / tiles);
        if (each == 7) each = 6;   // 17 tiles by 7 6.2 and 8.9 us, by 6 5.6 and 8.2
        const int split = (int)std::max<int64_t>(1, std::min<int64_t>({8, each, p.blocks / 2}));
        return a.rows <= 16 ? launch_tiles<16, SCALE_COLS>(b, a, p, split, stream) : a.rows <= 32 ? launch_tiles<32, SCALE_COLS>(b, a, p, split, stream) : launch_tiles<64, SCALE_COLS>(b, a, p, split, stream);
    }
    // Before the kernels' clusters are asked for, their shared memory is allowed.
    static std::atomic<bool> rows_set[kMaxDevices], both_set[kMaxDevices];
    if (!(both ? allow_smem(gemm8_tile_kernel<128, SCALE_BOTH>, Cfg8<128, SCALE_BOTH>::kSmem, both_set, dev) : allow_smem(gemm8_tile_kernel<128, SCALE_ROWS>, Cfg8<128, SCALE_ROWS>::kSmem, rows_set, dev)))
        return FP4Q_ERR_CUDA;
    const Plan8 plan(a.rows, b.rows, p.blocks, both, p.boxed > 0, dev);
    if (plan.pairs == 2) return both ? launch_persistent<2, SCALE_BOTH>(a, b, p, stream) : launch_persistent<2, SCALE_ROWS>(a, b, p, stream);
    if (plan.pairs == 1) return both ? launch_persistent<1, SCALE_BOTH>(a, b, p, stream) : launch_persistent<1, SCALE_ROWS>(a, b, p, stream);
    return both ? launch_tiles<128, SCALE_BOTH>(a, b, p, plan.split, stream) : launch_tiles<128, SCALE_ROWS>(a, b, p, plan.split, stream);
}

// Row-major codes (transposed: of the transpose), which may be missing from a tensor that has none of these elements.
fp4q_status operand8(const fp4q_fp8_tensor &t, bool transposed, bool square, Operand8 &o)
{
    if (t.square != 0 && t.square != 1) return FP4Q_ERR_UNSUPPORTED;
    if ((t.square != 0) != square) return FP4Q_ERR_UNSUPPORTED;
    o.q = transposed ? t.q_t : t.q;
    o.rows = transposed ? t.cols : t.rows;
    o.cols = transposed ? t.rows : t.cols;
    o.ld = transposed ? t.ld_t : t.ld_q;
    if (o.rows > kMaxDim8 || o.cols > kMaxDim8) return FP4Q_ERR_UNSUPPORTED;
    const bool own = transposed && !square;   // scales of its own
    o.scales.p = own ? t.scale_t : t.scale;
    const int64_t ld = own ? t.ld_st : t.ld_s;
    o.scales.row = transposed && square ? 1 : ld;
    o.scales.block = transposed && square ? ld : 1;
    o.scales.shift = square ? 7 : 0;
    o.scales.fours = o.scales.block == 1 && o.scales.row % 4 == 0 && aligned(o.scales.p, 16);
    if (o.rows == 0 || o.cols == 0) return FP4Q_OK;
    if (!o.q || !o.scales.p) return FP4Q_ERR_NULL;
    if (o.ld < o.cols || ld < ceil_div(square ? t.cols : o.cols, kBlock8)) return FP4Q_ERR_SHAPE;
    return aligned(o.q, 16) && o.ld % 16 == 0 && aligned(o.scales.p, 4) ? FP4Q_OK : FP4Q_ERR_ALIGN;
}

fp4q_status call8(int which, const fp4q_fp8_tensor *x, const fp4q_fp8_tensor *y, void *c, int64_t ldc, fp4q_out dt, int accumulate, void *ws, size_t ws_bytes, void *stream)
{
    if (!x || !y) return FP4Q_ERR_NULL;
    if (x->rows < 0 || x->cols < 0 || y->rows < 0 || y->cols < 0) return FP4Q_ERR_SHAPE;
    const int type = (int)dt & ~(int)FP4Q_OUT_PADDED;
    if (type != FP4Q_OUT_BF16 && type != FP4Q_OUT_F32) return FP4Q_ERR_UNSUPPORTED;
    if (which == 0 ? x->cols != y->cols : which == 1 ? x->cols != y->rows : x->rows != y->rows) return FP4Q_ERR_SHAPE;
    Operand8 a, b;
    if (fp4q_status s = operand8(*x, which == 2, false, a)) return s;
    if (fp4q_status s = operand8(*y, which >= 1, which < 2, b)) return s;
    if (accumulate && type != FP4Q_OUT_F32) return FP4Q_ERR_UNSUPPORTED;
    if (a.rows == 0 || b.rows == 0) return FP4Q_OK;
    const int64_t bytes = type == FP4Q_OUT_F32 ? 4 : 2;
    if (!c) return FP4Q_ERR_NULL;
    if (ldc < b.rows) return FP4Q_ERR_SHAPE;
    if (!aligned(c, 16) || ldc * bytes % 16 != 0) return FP4Q_ERR_ALIGN;
    if (!ws || ws_bytes < sizeof(Workspace)) return FP4Q_ERR_WORKSPACE;
    if (!aligned(ws, 256)) return FP4Q_ERR_ALIGN;
    Gemm8Params p = {};
    p.c = c;
    p.ldc = ldc;
    p.f32 = type == FP4Q_OUT_F32;
    p.accumulate = accumulate != 0;
    p.wide = aligned(c, 32) && ldc * bytes % 32 == 0;
    p.status = static_cast<uint32_t *>(ws);
    const int64_t per16 = 16 / bytes;
    p.boxed = (int32_t)(((int)dt & (int)FP4Q_OUT_PADDED) ? round_up(b.rows, per16) : b.rows / per16 * per16);
    if (a.cols == 0) {   // an empty contraction: maps of something that exists, and no block of it
        a.q = b.q = static_cast<const uint8_t *>(c);
        a.ld = b.ld = 16;
        Operand8 one = a;
        one.rows = one.cols = 1;
        p.m = (int32_t)a.rows;
        p.n = (int32_t)b.rows;
        return launch_tiles<128, SCALE_ROWS>(one, one, p, 1, static_cast<cudaStream_t>(stream));
    }
    return product8(a, b, p, which == 2, static_cast<cudaStream_t>(stream));
}

}  // namespace

extern "C" fp4q_status fp4q_fp8_gemm_fwd(const fp4q_fp8_tensor *X, const fp4q_fp8_tensor *W, void *Y, int64_t ldy, fp4q_out dt, void *ws, size_t ws_bytes, void *stream)
{
    return call8(0, X, W, Y, ldy, dt, 0, ws, ws_bytes, stream);
}

extern "C" fp4q_status fp4q_fp8_gemm_dgrad(const fp4q_fp8_tensor *dY, const fp4q_fp8_tensor *W, void *dX, int64_t ldx, fp4q_out dt, void *ws, size_t ws_bytes, void *stream)
{
    return call8(1, dY, W, dX, ldx, dt, 0, ws, ws_bytes, stream);
}

extern "C" fp4q_status fp4q_fp8_gemm_wgrad(const fp4q_fp8_tensor *dY, const fp4q_fp8_tensor *X, void *dW, int64_t ldw, fp4q_out dt, int accumulate, void *ws, size_t ws_bytes,
                                           void *stream)
{
    return call8(2, dY, X, dW, ldw, dt, accumulate, ws, ws_bytes, stream);
}
