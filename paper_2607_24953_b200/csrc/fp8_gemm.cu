// Products of 8-bit tensors with a scale for every block of 128 contraction elements: C[M,N] = sum over blocks b of sA sB (A_b B_b^T), codes E4M3,
// scales FP32 (include/fp4q.h).
//
// A stage of the operand ring is one block: rows of 128 bytes.  Four tcgen05.mma (kind::f8f6f4, 32 elements each) make the block's product in an accumulator of its
// own in tensor memory; the epilogue's warps take it from there, times its scales, into sums in registers, while the next block's MMAs run into
// another accumulator.  The accumulator that the tensor cores cut off towards zero is thus never longer than 128 elements; the sums are rounded to nearest.
#include "gemm16.cuh"

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
    __device__ __forceinline__ float at(int r, int b) const { return load_global(p + (int64_t)(r >> shift) * row + b * block); }
};

struct Gemm8Params {
    int32_t m, n, blocks;            // rows of A and B, blocks of the contraction
    int32_t n_tiles, split;          // split: CTAs of a cluster, which share a tile's contraction
    Scales8 sa, sb;
    void *c;                         // row-major, [m, n] or, with SCALE_COLS, its transpose: [n, m]
    int64_t ldc;
    int32_t f32, accumulate, wide;
    uint32_t *status;
};
struct Maps8 {
    CUtensorMap a, b;
};

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

// Two FP32 in a register pair.
__device__ __forceinline__ uint64_t pair32(float a, float b)
{
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void unpair32(uint64_t v, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ uint64_t fma_pair(uint64_t a, uint64_t b, uint64_t c)
{
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t mul_pair(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

// 16 columns of an accumulator's row; the values are there after landed().
__device__ __forceinline__ void load_acc(uint32_t from, uint32_t (&v)[16]) { FP4Q_TMEM_LD_X16(from, v); }
__device__ __forceinline__ void landed(uint32_t (&v)[16])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]), "+r"(v[8]), "+r"(v[9]), "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]),
                   "+r"(v[14]), "+r"(v[15])
                 :: "memory");
}

// sum += a block's product times its scales, for COLS columns of a thread's row.  row_scale: of the row; cols: of the columns, in shared memory.
template <int MODE, int COLS>
__device__ __forceinline__ void add_block(uint64_t (&sum)[COLS / 2], uint32_t from, float row_scale, const float *cols)
{
    const uint64_t s = pair32(row_scale, row_scale);
    uint32_t v[2][16];
    load_acc(from, v[0]);
#pragma unroll
    for (int c = 0; c < COLS; c += 16) {
        uint32_t(&x)[16] = v[(c / 16) & 1];
        landed(x);
        if (c + 16 < COLS) load_acc(from + c + 16, v[(c / 16 + 1) & 1]);
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
            const uint64_t lo = pair32(__uint_as_float(x[e]), __uint_as_float(x[e + 1])), hi = pair32(__uint_as_float(x[e + 2]), __uint_as_float(x[e + 3]));
            uint64_t &a = sum[(c + e) / 2], &b = sum[(c + e) / 2 + 1];
            if (MODE == SCALE_ROWS) {
                a = fma_pair(lo, s, a);
                b = fma_pair(hi, s, b);
            } else {
                const float4 f = *reinterpret_cast<const float4 *>(cols + c + e);
                const uint64_t f0 = pair32(f.x, f.y), f1 = pair32(f.z, f.w);
                if (MODE == SCALE_COLS) {
                    a = fma_pair(lo, f0, a);
                    b = fma_pair(hi, f1, b);
                } else {
                    a = fma_pair(mul_pair(lo, f0), s, a);
                    b = fma_pair(mul_pair(hi, f1), s, b);
                }
            }
        }
    }
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
    static constexpr int kPitch = 129;                                     // of the CTA's sums where the cluster adds them up, in the operands' place
    static constexpr int kSmem = 1024 + kOperands + 2 * kScales * 4 + 256;
    static_assert(kPitch * BN * 4 <= kOperands && kSmem <= 227 * 1024, "shared memory budget");
};

template <int BN, int MODE>
__global__ void __launch_bounds__(Cfg8<BN, MODE>::kThreads, BN == 128 ? 1 : 2) gemm8_tile_kernel(const __grid_constant__ Maps8 maps, const Gemm8Params p)
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
    uint64_t sum[kSums / 2];

    if (warp == 0) {
        const bool issuer = elect_one();
        const uint32_t a0 = smem_u32(smem_a), bb0 = smem_u32(smem_b);
        Ring16<C::kStages> ring;
        uint32_t loads = 0;
        for (int b = b0; b < b1; b++, ring.next()) {
            if (!warp_wait(bar_empty + 8 * ring.slot, ring.phase ^ 1u, abort_flag, p.status, limit, 0x100u + ring.slot)) break;
            const uint32_t bar = bar_full + 8 * ring.slot;
            expect_tx_if(bar, C::kStageBytes, issuer);
            if (issuer && (withhold == 0u || ++loads != withhold)) tma_load_2d(a0 + ring.slot * C::kABytes, &maps.a, b * kBlock8, m0, bar);
            if (issuer) tma_load_2d(bb0 + ring.slot * C::kBBytes, &maps.b, b * kBlock8, n0, bar);
            __syncwarp();
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
#pragma unroll
            for (int i = 0; i < C::kAhead; i++) {
                const bool there = b + i < b1;
                const float other = !there || MODE == SCALE_BOTH ? 1.f : MODE == SCALE_ROWS ? p.sb.at(n0, b + i) : p.sa.at(m0, b + i);
#pragma unroll
                for (int j = lane; j < C::kRowScales; j += 32) to[i * C::kRowScales + j] = there && m0 + j < p.m ? p.sa.at(m0 + j, b + i) * other : 0.f;
#pragma unroll
                for (int j = lane; j < C::kColScales; j += 32) to[C::kAhead * C::kRowScales + i * C::kColScales + j] = there && n0 + j < p.n ? p.sb.at(n0 + j, b + i) * other : 0.f;
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(bar_sc_full + 8 * set.slot);
        }
    } else if (warp >= 4) {
        const int quarter = warp & 3, half = (warp - 4) >> 2;
#pragma unroll
        for (int i = 0; i < kSums / 2; i++) sum[i] = 0;
        Ring16<C::kAccs> acc;
        Ring16<2> set;
        for (int b = b0; b < b1; b++, acc.next()) {
            const int i = (b - b0) % C::kAhead;
            if (i == 0 && !warp_wait(bar_sc_full + 8 * set.slot, set.phase, abort_flag, p.status, limit, 0x500u)) break;
            if (!warp_wait(bar_acc_full + 8 * acc.slot, acc.phase, abort_flag, p.status, limit, 0x600u)) break;
            tcgen05_fence_after();
            const float *from = scales + set.slot * C::kScales;
            const float row = C::kRowScales ? from[i * C::kRowScales + 32 * quarter + lane] : 1.f;
            add_block<MODE, C::kCols>(sum, tmem + acc.slot * BN + half * C::kCols + ((uint32_t)(32 * quarter) << 16), row, from + C::kAhead * C::kRowScales + i * C::kColScales + half * C::kCols);
            tcgen05_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar_acc_empty + 8 * acc.slot);
            if (i == C::kAhead - 1 || b == b1 - 1) {
                if (lane == 0) mbar_arrive(bar_sc_empty + 8 * set.slot);
                set.next();
            }
        }
        const int in = 32 * quarter + lane;   // row of the tile
        if (p.split == 1) {
            if (m0 + in < p.m && *abort_flag == 0u) {
#pragma unroll
                for (int c = 0; c < C::kCols; c += 16) {
                    float v[16];
#pragma unroll
                    for (int e = 0; e < 16; e += 2) unpair32(sum[(c + e) / 2], v[e], v[e + 1]);
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
            float *mine = reinterpret_cast<float *>(smem) + in;
#pragma unroll
            for (int c = 0; c < C::kCols; c += 2) {
                float x, y;
                unpair32(sum[c / 2], x, y);
                mine[(half * C::kCols + c) * C::kPitch] = x;
                mine[(half * C::kCols + c + 1) * C::kPitch] = y;
            }
        }
    }
    __syncwarp();
    if (p.split > 1) {
        cluster_arrive();
        cluster_wait();
        // This CTA's share of the tile: the sums of all CTAs, in their order.
        if (*abort_flag == 0u) {
            const uint32_t base = smem_u32(smem);
            constexpr int kTile = 128 * BN;
            const int e0 = (int)((int64_t)kTile * rank / p.split), e1 = (int)((int64_t)kTile * (rank + 1) / p.split);
            for (int e = e0 + threadIdx.x; e < e1; e += C::kThreads) {
                const int row = MODE == SCALE_COLS ? e % 128 : e / BN, col = MODE == SCALE_COLS ? e / 128 : e % BN;
                if (m0 + row >= p.m || n0 + col >= p.n) continue;
                float v = 0.f;
                for (int r = 0; r < p.split; r++) {
                    float x;
                    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(x) : "r"(cluster_addr(base + (col * C::kPitch + row) * 4, r)) : "memory");
                    v += x;
                }
                if (MODE == SCALE_COLS) store_one(p, n0 + col, m0 + row, v);
                else store_one(p, m0 + row, n0 + col, v);
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
    const int64_t ctas = ceil_div(p.m, 128) * p.n_tiles * split;
    if (ctas > 0x7FFFFFFF) return FP4Q_ERR_UNSUPPORTED;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[2];
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
    return launched(cudaLaunchKernelEx(&cfg, gemm8_tile_kernel<BN, MODE>, maps, p));
}

// CTAs that share a tile's contraction: as many as fill the GPU's places, with two blocks each at least.
int split_of(int64_t tiles, int64_t places, int64_t blocks)
{
    return (int)std::max<int64_t>(1, std::min<int64_t>({8, places / tiles, blocks / 2}));
}

// mode: SCALE_ROWS: C[m, n] with A in 1D blocks and B in square ones; SCALE_BOTH: both in 1D blocks.
fp4q_status product8(const Operand8 &a, const Operand8 &b, Gemm8Params p, bool both, cudaStream_t stream)
{
    p.m = (int32_t)a.rows;
    p.n = (int32_t)b.rows;
    p.blocks = (int32_t)ceil_div(a.cols, kBlock8);
    p.sa = a.scales;
    p.sb = b.scales;
    if (!both && a.rows <= 64) {   // few tokens: B's rows become the tile's 128 rows
        std::swap(p.m, p.n);
        std::swap(p.sa, p.sb);
        const int bn = a.rows <= 16 ? 16 : a.rows <= 32 ? 32 : 64, split = split_of(ceil_div(b.rows, 128), 296, p.blocks);
        return bn == 16 ? launch_tiles<16, SCALE_COLS>(b, a, p, split, stream) : bn == 32 ? launch_tiles<32, SCALE_COLS>(b, a, p, split, stream) : launch_tiles<64, SCALE_COLS>(b, a, p, split, stream);
    }
    const int split = split_of(ceil_div(a.rows, 128) * ceil_div(b.rows, 128), 148, p.blocks);
    return both ? launch_tiles<128, SCALE_BOTH>(a, b, p, split, stream) : launch_tiles<128, SCALE_ROWS>(a, b, p, split, stream);
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
