// Products of 16-bit matrices (BF16 or FP16) on the tensor cores of sm_100a, FP32 accumulation: C[M,N] = A B with either operand
// stored along the contraction ("K-major") or across it ("MN-major"), for matrices cut into groups of rows that start anywhere, for
// contractions cut the same way, for stacks of matrices and for symmetric results.  The entry points are in ragged_gemm.cu and
// newton_schulz.cu.
//
// Persistent kernel, one CTA per SM, 12 warps.  A CTA has 128 rows of the accumulator; pairs (cta_group::2) share a tile of 256 rows and
// each loads half of B's columns, which is what lets 32 KB of operands feed 2 x 256 x 256 x 64 operations per stage (an SM gets 32 KB from L2
// in about 0.3 us, as long as the MMAs take at the clock that full load leaves); single CTAs have tiles of 128 x 128 for problems with few
// tiles, and of 32 x 64 for short groups (the MMAs have 128 rows all the same: those behind the first 32 are whatever lies in shared
// memory, and nobody looks at them), and of 64 x 64 for small stacks of matrices.  Long contractions of few tiles are cut into parts, whose
// accumulators meet in the caller's scratch memory.
//   warps 0, 3  TMA producers of A and B: a stage is 64 contraction elements (32 x 64 tiles: 256), boxes of 128 bytes with the 128-byte swizzle
//   warp 1      MMA issuer (in the leader of a pair): four tcgen05.mma of 16 contraction elements per box
//   warp 2      cut contractions: deals the tiles (in the leader of a pair), zeroes the rows of a group's last stage that lie behind the group
//   warps 4-11  epilogue: a thread has a row of the tile; the accumulator is double-buffered in tensor memory.  Outputs leave, and what an
//               epilogue reads comes, as boxes of 32 rows x 128 bytes through shared memory (TMA): with plain accesses a warp's 16 bytes
//               in each of 32 rows take the load/store unit 32 cycles, which made update products of 768 x 2048 epilogue-bound
// Every wait is bounded: when a limit is hit the CTA records FP4Q_ERR_TIMEOUT in the workspace, its roles stop and it leaves through the
// normal exit, after its copies in flight have landed.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "tcgen05.cuh"
#include "tensor_map.cuh"

namespace fp4q {

constexpr int kRows16 = 128;         // accumulator rows per CTA
constexpr int kBox16 = 64;           // contraction elements of a box: 128 bytes
constexpr int kThreads16 = 384;
constexpr int kRaster16 = 16;        // row tiles per rasterisation group: their A rows stay in L2 while the columns go by
constexpr int kMaxSorted16 = 256;    // cut contractions: so many groups are dealt longest first
constexpr int kDealt16 = 4;          // cut contractions: tiles that are dealt ahead
constexpr int kMaxGroups16 = 2047;   // boundaries and first tiles of this many groups lie in shared memory

// TILES_ROWS: groups of A rows (and of output rows), a matrix B per group.  TILES_CUT: a product per group, contracted over its rows.
// TILES_BATCH: a stack of products.  TILES_SYM: a stack of symmetric products; only tiles on and below the diagonal are computed.
enum { TILES_ROWS = 0, TILES_CUT = 1, TILES_BATCH = 2, TILES_SYM = 3 };
// EPI16_STORE: BF16 output.  EPI16_SUM: FP32 output.  The others are the three products of a Newton-Schulz step (newton_schulz.cu).
// The tensor cores cut the sum of an accumulator and 16 products off to FP32, towards zero: the error grows with the contraction, by 1e-9 of
// the result for every element (2e-5 at 16384; 8e-5 where all products are positive).  BF16 and FP16 outputs do not show it up to some 10^5
// elements, and longer contractions are cut into parts (newton_schulz.cu, CutPlan in ragged_gemm.cu); forward and input gradient, whose contraction is a
// layer's width, are not.  FP32 ones are sums, to nearest and in registers, of accumulators of 512 elements each.
enum { EPI16_STORE = 0, EPI16_GRAM = 1, EPI16_POLY = 2, EPI16_UPDATE = 3, EPI16_SUM = 4 };
constexpr int kSumElems = 512;

// TWO: an epilogue warp of a product that writes its output as it is has two boxes, at the price of a stage.  For contractions that are short
// beside their output (300 rows in 64 groups 30 -> 27 us, 24266 in 44 groups of 306 x 4270 183-199 -> 175); others lose (the expert layer's
// forward 363 -> 381).
// Tiles of 64 columns have 32 rows where rows come in short groups, and 64 in stacks of matrices (STACK), where they serve those so small
// that all their tiles run at once: the fewer bytes a CTA loads, the sooner it is done.
template <int CTAS, int BN, bool TWO = false, bool STACK = false>
struct Cfg16 {
    static_assert(CTAS == 1 || (CTAS == 2 && BN == 256), "tile shapes");
    static constexpr int kBRows = BN / CTAS;
    // 32 x 64 tiles take 128 cycles of MMAs per box, much less than a round of the issuer: their stages are four boxes deep, 64 x 64 ones' two.
    static constexpr int kBoxes = BN == 64 ? (STACK ? 2 : 4) : 1;
    static constexpr int kK = kBoxes * kBox16;                              // contraction elements per stage
    static constexpr int kRows = BN == 64 ? (STACK ? 64 : 32) : kRows16;    // rows of a CTA's part of a tile
    static constexpr int kABox = kRows * 128, kBBox = kBRows * 128;
    static constexpr int kABytes = kBoxes * kABox, kBBytes = kBoxes * kBBox;
    static constexpr int kStages = BN == 64 && !STACK ? 3 : TWO ? 4 : 5;
    // 64 x 64 tiles of operands in two numbers: a stage's two boxes are the upper and lower parts of one, and an MMA of 128 x 128 multiplies both of A,
    // above each other, with both of B.  The tile is the sum of the four quarters of what it makes.  (Three MMAs of 128 x 64, half of their rows for
    // nothing, instead: 384 x 384 122 us for 113, four of 128 x 1000 127 for 116, 256 x 256 99 for 101.)
    static constexpr bool kBoth = BN == 64 && STACK;
    static constexpr int kAccCols = kBoth ? 128 : BN;
    static constexpr int kTmemCols = 2 * kAccCols;
    static constexpr int kOperands = kStages * (kABytes + kBBytes);
    static constexpr int kTail = 512;                                       // barriers, tensor memory's address, abort flag
    static constexpr int kTables = 3 * (kMaxGroups16 + 1) * 4 + kMaxSorted16 * 2;   // row groups and cut contractions only
    // Of an epilogue warp: one box or two, or an upper and a lower one.
    __host__ __device__ static constexpr int staging(int epi) { return !TWO && (epi == EPI16_STORE || epi == EPI16_SUM) ? 4096 : 8192; }
    static constexpr int smem(int tiles, int epi) { return 1024 + kOperands + 8 * staging(epi) + kTail + (tiles <= TILES_CUT ? kTables : 0); }
    static constexpr int kTileRows = kRows * CTAS;
    static constexpr int64_t kPlaceBytes = (int64_t)CTAS * kRows16 * BN * 4;   // of a part's accumulator
    static_assert(1024 + kOperands + 8 * (TWO ? 8192 : 4096) + kTail + kTables <= 227 * 1024, "shared memory budget: groups");
    static_assert((BN == 64 && !STACK) || 1024 + kOperands + 8 * 8192 + kTail <= 227 * 1024, "shared memory budget: stacks");
};

// Division by a number that the host knows, of numbers below 2^31: with s = ceil(log2 d), n / d = n m >> (31 + s) for m = ceil(2^(31 + s) / d), since m d
// exceeds 2^(31 + s) by less than 2^s.
struct Divisor16 {
    uint32_t mul, shift;   // mul = 0: by one
    __host__ static Divisor16 of(int64_t d)
    {
        if (d <= 1) return Divisor16{0u, 0u};
        uint32_t s = 1;
        while ((1ll << s) < d) s++;
        return Divisor16{(uint32_t)(((1ull << (31 + s)) + (uint64_t)d - 1) / (uint64_t)d), s - 1};
    }
    __device__ __forceinline__ int operator()(int n) const { return mul == 0u ? n : (int)(__umulhi((uint32_t)n, mul) >> shift); }
};

struct Gemm16Params {
    int32_t m, n, k;                 // output rows and columns and contraction length of one product (TILES_ROWS: m = all rows, TILES_CUT: k = all rows)
    int32_t m_tiles, n_tiles;        // TILES_ROWS: m_tiles is found on the device
    Divisor16 by_matrix, by_band;    // tiles of a matrix or group (but TILES_ROWS), and of kRaster16 rows of tiles: set by launch_gemm16
    int32_t batch;                   // groups or matrices
    int32_t bf16;                    // operand type: 0 = FP16, 1 = BF16
    int32_t admit;                   // the next kernel may set up beside this one (it is one of the same call)
    uint32_t *deal;                  // TILES_CUT: tiles dealt, 0 when the kernel starts: they go to whoever is free; NULL: in turn
    int32_t a_box;                   // rows of one copy of a K-major A operand: 128, 64 in 64 x 64 tiles, 32 or 16 in tiles of 32 rows
    int32_t part_stages;             // stages of a part of a contraction in parts
    union {
        const int64_t *offsets;      // TILES_ROWS, TILES_CUT: batch + 1 boundaries; NULL: one group of all rows
        const int32_t *lift;         // GRAM, UPDATE: of each matrix: its first X is scaled by this power of two more than others
    };
    int64_t total_rows;              // rows that the boundaries are held to
    uint32_t *status;
    // Contractions in parts (TILES_CUT, EPI16_GRAM): a part's accumulator goes to `partial`, and who comes last to a tile, by its counter, adds up
    // the parts in their order.  NULL: no parts.
    float *partial;                  // [part][CTA of the tile][warp][column / 4][row][column % 4]
    uint32_t *counters;              // of a tile's warps; 0 between kernels
    // EPI16_STORE, EPI16_SUM
    void *c;
    int64_t ldc;
    int32_t accumulate, wide, zero_rest;   // zero_rest: rows that no group owns are written as zeros
    int32_t boxed;                   // columns that leave in boxes, whole 16 bytes; the rest of a row leaves by itself
    // EPI16_GRAM, _POLY, _UPDATE
    int32_t split;                   // 1: operands are sums of two numbers: the products upper x upper, upper x lower and lower x upper are added up
    float o_scale;                   // UPDATE, last step
    float fa, fb, fc;                // the step's coefficients, with the iterates' scales; POLY: fa on the diagonal
    int32_t grown, grown_next;       // powers of two by which X may have grown since, up to this step's product and behind it
    __nv_bfloat16 *o;                // UPDATE, last step: the result instead
    int64_t ld_o;
};

// Operands and their lower parts; what an epilogue reads (POLY: A, UPDATE: X's lower part, as in) and writes, upper and lower parts, in boxes of 32 rows x 128
// bytes; the mirrored tiles of symmetric results, in boxes of 64 rows x 64 bytes.
struct Maps16 {
    CUtensorMap a, b, a2, b2, in, in2, out, out2, mirror, mirror2;
};

// A tile as one CTA of it sees it.
struct Tile16 {
    int32_t batch, a_row, b_row, k0, k_len;    // where the operands start along M and N, where the contraction starts and how long it is
    int32_t row, col, rows, rows_peer;         // first output row and column of this CTA's half, its valid rows and the other CTA's
    int32_t s0, s1;                            // its stages (a part of all)
    int32_t parts, slot0, counter;             // parts of the contraction; where the first one's accumulator goes; the tile's counter
    bool mirror;                               // TILES_SYM: below the diagonal, so the transposed tile is written too; on it, A's boxes serve as B's
};

// By the lanes for which `issue` holds, without a branch (see tcgen05_mma_f16).  PAIR: the copy is counted on a barrier of the pair's leader.
template <bool PAIR = false>
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap *map, int32_t x, int32_t y, int32_t z, uint32_t bar, bool issue = true)
{
    if (PAIR)
        asm volatile("{\n .reg .pred q;\n setp.ne.b32 q, %6, 0;\n"
                     "@q cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];\n}"
                     ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar), "r"((uint32_t)issue) : "memory");
    else
        asm volatile("{\n .reg .pred q;\n setp.ne.b32 q, %6, 0;\n"
                     "@q cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];\n}"
                     ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar), "r"((uint32_t)issue) : "memory");
}
__device__ __forceinline__ void expect_tx_if(uint32_t bar, uint32_t bytes, bool issue)
{
    asm volatile("{\n .reg .pred q;\n .reg .b64 state;\n setp.ne.b32 q, %2, 0;\n @q mbarrier.arrive.expect_tx.shared::cta.b64 state, [%0], %1;\n}"
                 ::"r"(bar), "r"(bytes), "r"((uint32_t)issue) : "memory");
}
__device__ __forceinline__ void tma_store_3d(const CUtensorMap *map, int32_t x, int32_t y, int32_t z, uint32_t src)
{
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%1, %2, %3}], [%4];" ::"l"(map), "r"(x), "r"(y), "r"(z), "r"(src) : "memory");
}
__device__ __forceinline__ void tma_reduce_add_3d(const CUtensorMap *map, int32_t x, int32_t y, int32_t z, uint32_t src)
{
    asm volatile("cp.reduce.async.bulk.tensor.3d.global.shared::cta.add.tile.bulk_group [%0, {%1, %2, %3}], [%4];" ::"l"(map), "r"(x), "r"(y), "r"(z), "r"(src) : "memory");
}
__device__ __forceinline__ void st_shared_16(uint32_t at, uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(at), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ uint4 ld_shared_16(uint32_t at)
{
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
    return v;
}
// Arrival on a barrier of either CTA of a pair that orders this thread's writes, to shared memory or tensor memory, before what the waiter does.
__device__ __forceinline__ void mbar_arrive_release_cluster(uint32_t cluster_bar)
{
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_bar) : "memory");
}

// By the lanes for which `issue` holds.  The whole warp comes here, without a branch: what an instruction takes from uniform registers stays in them
// (a lane that branches off moves six words there for every MMA: 75 cycles each, now 37; and 8 rows in 8 groups
// of 768 x 2048 11.5 us, now 9.8, 11008 x 4096 updates 3160 and 3060).  Descriptors: their lower words, which hold the address, and the upper one.
template <int CTAS>
__device__ __forceinline__ void tcgen05_mma_f16(uint32_t d_tmem, uint32_t a_lo, uint32_t b_lo, uint32_t hi, uint32_t idesc, bool accumulate, bool issue)
{
    if (CTAS == 2)
        asm volatile("{\n .reg .pred p, q;\n .reg .b64 a, b;\n setp.ne.b32 p, %5, 0;\n setp.ne.b32 q, %6, 0;\n mov.b64 a, {%1, %3};\n mov.b64 b, {%2, %3};\n"
                     "@q tcgen05.mma.cta_group::2.kind::f16 [%0], a, b, %4, p;\n}"
                     ::"r"(d_tmem), "r"(a_lo), "r"(b_lo), "r"(hi), "r"(idesc), "r"((uint32_t)accumulate), "r"((uint32_t)issue) : "memory");
    else
        asm volatile("{\n .reg .pred p, q;\n .reg .b64 a, b;\n setp.ne.b32 p, %5, 0;\n setp.ne.b32 q, %6, 0;\n mov.b64 a, {%1, %3};\n mov.b64 b, {%2, %3};\n"
                     "@q tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %4, p;\n}"
                     ::"r"(d_tmem), "r"(a_lo), "r"(b_lo), "r"(hi), "r"(idesc), "r"((uint32_t)accumulate), "r"((uint32_t)issue) : "memory");
}
template <int CTAS>
__device__ __forceinline__ void tcgen05_commit_if(uint32_t bar, bool issue)
{
    if (CTAS == 1)
        asm volatile("{\n .reg .pred q;\n setp.ne.b32 q, %1, 0;\n @q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}" ::"r"(bar), "r"((uint32_t)issue) : "memory");
    else   // arrives on the barrier at this offset in both CTAs of the pair
        asm volatile("{\n .reg .pred q;\n setp.ne.b32 q, %2, 0;\n @q tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;\n}"
                     ::"r"(bar), "h"((uint16_t)3), "r"((uint32_t)issue) : "memory");
}
// MN-major operand tile: chunks of 64 elements x 64 contraction rows (8 KB each), a row of a chunk 128 bytes with the 128-byte swizzle;
// eight contraction rows make 1024 bytes.
__device__ __forceinline__ uint64_t smem_desc_mn_sw128(uint32_t addr)
{
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | ((uint64_t)(8192 >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
template <int CTAS>
__device__ __forceinline__ uint32_t instr_desc16(bool bf16, bool a_mn, bool b_mn, int cols)
{
    const uint32_t type = bf16 ? 1u : 0u;
    return (1u << 4) | (type << 7) | (type << 10) | ((uint32_t)a_mn << 15) | ((uint32_t)b_mn << 16) | ((uint32_t)(cols >> 3) << 17) |
           ((uint32_t)((kRows16 * CTAS) >> 4) << 24);
}
// A barrier's phase: CLUSTER if the other CTA of a pair arrives on it, whose writes this thread then sees.  (A fence behind the wait
// instead waits for all that the issuer has under way: 1.2 us whenever it went on to the next accumulator.)
template <bool CLUSTER>
__device__ __forceinline__ bool mbar_try(uint32_t bar, uint32_t parity)
{
    uint32_t done;
    if (CLUSTER)
        asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n selp.b32 %0, 1, 0, p;\n}" : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    else
        asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.b32 %0, 1, 0, p;\n}" : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    return done != 0u;
}
template <bool CLUSTER>
__device__ __forceinline__ bool mbar_look(uint32_t bar, uint32_t parity)   // without suspension
{
    uint32_t done;
    if (CLUSTER)
        asm volatile("{\n .reg .pred p;\n mbarrier.test_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n selp.b32 %0, 1, 0, p;\n}" : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    else
        asm volatile("{\n .reg .pred p;\n mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.b32 %0, 1, 0, p;\n}" : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    return done != 0u;
}
__device__ __forceinline__ uint64_t now_ns()
{
    uint64_t t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
    return t;
}
// A whole warp's bounded wait: all lanes go on or none does.  `limit` is in microseconds of the clock, the unit of the workspace's polls; a
// poll suspends the warp for as long as the hardware likes, which is finite.  (With suspensions of a microsecond at most, as the
// quantized products have them, the update product of 2048 x 5632 took 83 us instead of 67.)
template <bool CLUSTER = false>
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile uint32_t *abort_flag, uint32_t *status, uint64_t limit, uint32_t where)
{
    bool ok = true;
    uint64_t since = 0;
    while (!mbar_try<CLUSTER>(bar, parity)) {
        if (*abort_flag) { ok = false; break; }
        const uint64_t now = now_ns();
        if (since == 0) since = now;
        else if (now - since > limit * 1000) {
            *abort_flag = 1u;
            if (atomicCAS(status, 0u, (uint32_t)FP4Q_ERR_TIMEOUT) == 0u) status[1] = where;
            ok = false;
            break;
        }
    }
    return __all_sync(0xFFFFFFFFu, ok);
}
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(max(e, -126) + 127) << 23); }   // e <= 127
// A ring's next slot and its phase.
template <int N>
struct Ring16 {
    uint32_t slot = 0, phase = 0;
    __device__ __forceinline__ void next()
    {
        if (++slot == N) { slot = 0; phase ^= 1u; }
    }
};

// ---------------------------------------------------------------------------------------- tiles

// start[g], g = 0..n: the boundaries, held to [0, rows] and to rising order: whatever they are, no row outside the matrices is
// touched and none belongs to two groups.  first[g]: row tiles before group g (TILES_ROWS).
__device__ __forceinline__ int32_t group_rows(const int32_t *start, int g) { return start[g + 1] - start[g]; }

// The last g with first[g] <= tile, of n which do not fall, first[0] = 0: the whole warp looks, at one of every n / 32 and then at those between.  (With a search
// by halves and divisions by variables a tile was decoded in 1200 cycles, now in 600; all steps of an update 256 x 256 103 -> 100 us, 30 of 64 x 64 84 -> 82.)
__device__ __forceinline__ int find_group16(const int32_t *first, int n, int tile)
{
    const int lane = threadIdx.x & 31, run = (n + 31) / 32;
    const int at = (__popc(__ballot_sync(0xFFFFFFFFu, lane * run < n && first[lane * run] <= tile)) - 1) * run;
    if (run == 1) return at;
    int found = 0;
    for (int i = lane; i - lane < run; i += 32) found += __popc(__ballot_sync(0xFFFFFFFFu, i < run && at + i < n && first[at + i] <= tile));
    return at + found - 1;
}

// Parts that a contraction of `stages` stages is cut into.
__device__ __forceinline__ int parts16(const Gemm16Params &p, int stages) { return p.partial && stages > p.part_stages ? (stages + p.part_stages - 1) / p.part_stages : 1; }

// slots: TILES_CUT: places for accumulators that the groups before a group take, counted in tiles' parts.
template <int TILES, int CTAS, int BN>
__device__ __forceinline__ Tile16 decode16(const Gemm16Params &p, int tile, int m_tiles, int passes, const int32_t *start, const int32_t *first, const int32_t *slots,
                                           const uint16_t *order, int rank)
{
    using C = Cfg16<CTAS, BN, false, (TILES >= TILES_BATCH)>;
    constexpr int kRows = C::kRows, kBM = kRows * CTAS, kBRows = C::kBRows, kK = C::kK;
    Tile16 t;
    int mt, nt, part = 0;
    t.batch = 0;
    t.mirror = false;
    t.k0 = 0;
    t.k_len = p.k;
    t.parts = 1;
    t.slot0 = t.counter = 0;
    if (TILES == TILES_SYM) {
        // The first parts of all tiles, then the second ones: tiles that share rows read them at the same time.  (Updates of 4096 x 128256 in 4 parts 31.1 -> 29.7 ms.)
        t.parts = parts16(p, passes * ((p.k + kK - 1) / kK));
        const int per = m_tiles * (m_tiles + 1) / 2;
        part = t.parts == 1 ? 0 : tile / (p.batch * per);
        t.counter = tile - part * (p.batch * per);
        t.slot0 = t.counter * t.parts;
        t.batch = p.by_matrix(t.counter);
        const int r = t.counter - t.batch * per;
        mt = (int)((sqrtf(8.0f * (float)r + 1.0f) - 1.0f) * 0.5f);
        while (mt * (mt + 1) / 2 > r) mt--;
        while ((mt + 1) * (mt + 2) / 2 <= r) mt++;
        nt = r - mt * (mt + 1) / 2;
        t.mirror = mt != nt;
    } else {
        int r = tile;
        if (TILES == TILES_CUT) {
            const int per = m_tiles * p.n_tiles, at = p.partial ? find_group16(first, p.batch, tile) : p.by_matrix(tile);
            t.batch = order ? order[at] : at;
            t.k0 = start[t.batch];
            t.k_len = group_rows(start, t.batch);
            r = tile - (p.partial ? first[at] : at * per);
            if (p.partial) {
                t.parts = parts16(p, (t.k_len + kK - 1) / kK);
                // The first parts of all the group's tiles, then the second ones, as above, unless there are more parts than tiles.  (2^20 rows in 2 groups of 1024 x
                // 1024 2178 -> 1768 us, 32768 in 16 skewed ones of 2048 x 1024 220 -> 174; but 131072 in 100 of 256 x 256 87 -> 98.)
                int in_group;
                if (t.parts <= per) {
                    part = p.by_matrix(r);
                    in_group = r - part * per;
                } else {
                    in_group = r / t.parts;
                    part = r - in_group * t.parts;
                }
                t.slot0 = slots[at] + in_group * t.parts;
                t.counter = t.slot0;   // no two tiles start in one place
                r = in_group;
            }
        }
        if (TILES == TILES_BATCH) {
            const int per = m_tiles * p.n_tiles;
            t.batch = p.by_matrix(tile);
            r = tile - t.batch * per;
        }
        const int per_group = kRaster16 * p.n_tiles, g = p.by_band(r), m0 = g * kRaster16, h = min(kRaster16, m_tiles - m0), rem = r - g * per_group;
        nt = h == kRaster16 ? rem / kRaster16 : rem / h;
        mt = m0 + rem - nt * h;
    }
    t.col = nt * BN;
    t.b_row = t.col + rank * kBRows;
    int valid;   // rows of the whole tile
    if (TILES == TILES_ROWS) {
        t.batch = find_group16(first, p.batch, mt);
        const int in = (mt - first[t.batch]) * kBM;
        t.row = start[t.batch] + in;
        valid = group_rows(start, t.batch) - in;
    } else {
        t.row = mt * kBM;
        valid = p.m - t.row;
    }
    t.row += rank * kRows;
    t.a_row = t.row;
    t.rows = max(0, min(kRows, valid - rank * kRows));
    t.rows_peer = CTAS == 2 ? max(0, min(kRows, valid - (1 - rank) * kRows)) : 0;
    const int stages = C::kBoth && p.split ? (t.k_len + kBox16 - 1) / kBox16 : passes * ((t.k_len + kK - 1) / kK);
    t.s0 = part * p.part_stages;
    t.s1 = t.parts == 1 ? stages : min(t.s0 + p.part_stages, stages);
    return t;
}
// Operands in two numbers take two stages for a piece of the contraction, upper and lower parts: whether a stage is the second, and how much of
// the contraction (of k_len) is left where it starts.  (With three loads of each, one for every product, the
// updates of 14 of 7397 x 193 took 632 us instead of 563.)
template <bool SPLITS>
__device__ __forceinline__ bool lower16(const Gemm16Params &p, int s) { return SPLITS && (s & p.split) != 0; }   // not in 64 x 64 tiles
template <bool SPLITS, int K, bool BOTH>
__device__ __forceinline__ int left16(const Gemm16Params &p, const Tile16 &t, int s)
{
    return t.k_len - (BOTH ? s * (p.split ? kBox16 : K) : (SPLITS ? s >> p.split : s) * K);
}

// On the diagonal of a symmetric product both operands are the same rows: they are loaded once.  (128 of 768 x 2048, where half of the tiles lie
// there: P's stages 0.65 -> 0.57 us.)
template <int TILES>
__device__ __forceinline__ bool shares_a(const Tile16 &t) { return TILES == TILES_SYM && !t.mirror; }

// ---------------------------------------------------------------------------------------- epilogues: 32 columns of a thread's row

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    const __nv_bfloat162 b = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&b);
}
__device__ __forceinline__ uint32_t pack_half(float lo, float hi)
{
    const __half2 b = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&b);
}
__device__ __forceinline__ float2 unpack_half(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2 *>(&w)); }
__device__ __forceinline__ void store_32_bytes(void *p, const uint32_t *w)
{
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
}

// Row `row` (of all output rows), columns col .. col + 31, of which those below n exist.
__device__ __forceinline__ void store_bf16(const Gemm16Params &p, int64_t row, int col, const float *v)
{
    const int left = p.n - col;
    if (left <= 0) return;
    __nv_bfloat16 *c = static_cast<__nv_bfloat16 *>(p.c) + row * p.ldc + col;
    if (left >= 32) {
#pragma unroll
        for (int e = 0; e < 32; e += 16) {
            uint32_t w[8];
#pragma unroll
            for (int j = 0; j < 8; j++) w[j] = pack_bf16(v[e + 2 * j], v[e + 2 * j + 1]);
            if (p.wide) store_32_bytes(c + e, w);
            else {
                *reinterpret_cast<uint4 *>(c + e) = make_uint4(w[0], w[1], w[2], w[3]);
                *reinterpret_cast<uint4 *>(c + e + 8) = make_uint4(w[4], w[5], w[6], w[7]);
            }
        }
    } else {
#pragma unroll
        for (int e = 0; e < 32; e++)
            if (e < left) c[e] = __float2bfloat16_rn(v[e]);
    }
}
__device__ __forceinline__ void store_f32(const Gemm16Params &p, int64_t row, int col, const float *v)
{
    const int left = p.n - col;
    if (left <= 0) return;
    float *c = static_cast<float *>(p.c) + row * p.ldc + col;
    if (left >= 32) {
#pragma unroll
        for (int e = 0; e < 32; e += 8) {
            float w[8];
#pragma unroll
            for (int j = 0; j < 8; j++) w[j] = v[e + j];
            if (p.accumulate) {
                const float4 a = *reinterpret_cast<const float4 *>(c + e), b = *reinterpret_cast<const float4 *>(c + e + 4);
                w[0] += a.x; w[1] += a.y; w[2] += a.z; w[3] += a.w; w[4] += b.x; w[5] += b.y; w[6] += b.z; w[7] += b.w;
            }
            if (p.wide) store_32_bytes(c + e, reinterpret_cast<const uint32_t *>(w));
            else {
                *reinterpret_cast<float4 *>(c + e) = make_float4(w[0], w[1], w[2], w[3]);
                *reinterpret_cast<float4 *>(c + e + 4) = make_float4(w[4], w[5], w[6], w[7]);
            }
        }
    } else {
#pragma unroll
        for (int e = 0; e < 32; e++)
            if (e < left) c[e] = p.accumulate ? c[e] + v[e] : v[e];
    }
}

// An epilogue warp's box in shared memory: 32 rows of 128 bytes, 16-byte pieces swizzled as TMA does.  A lane writes and reads its own row.
struct Box16 {
    uint32_t row, swizzle;
    __device__ __forceinline__ Box16(uint32_t base, int lane) : row(base + lane * 128), swizzle((uint32_t)lane & 7u) {}
    __device__ __forceinline__ uint32_t piece(int i) const { return row + (((uint32_t)i ^ swizzle) << 4); }
    __device__ __forceinline__ void put(const uint32_t *w) const   // 32 words
    {
#pragma unroll
        for (int i = 0; i < 8; i++) st_shared_16(piece(i), w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
    }
};
__device__ __forceinline__ void load_blocks_transposed(uint32_t at, uint32_t *v)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void store_blocks(uint32_t at, const uint32_t *v)
{
    asm volatile("stmatrix.sync.aligned.m8n8.x4.shared.b16 [%0], {%1,%2,%3,%4};" ::"r"(at), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]) : "memory");
}
__device__ __forceinline__ void fence_async_shared() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
// The warp's stores have read its boxes.
__device__ __forceinline__ void boxes_free(int lane)
{
    if (lane == 0) bulk_wait_read_all();
    __syncwarp();
}

// ---------------------------------------------------------------------------------------- kernel

template <int CTAS, int BN, bool A_MN, bool B_MN, int EPI, int TILES, bool TWO = false>
__global__ void __launch_bounds__(kThreads16, 1) gemm16_kernel(const __grid_constant__ Maps16 maps, const Gemm16Params p)
{
    using C = Cfg16<CTAS, BN, TWO, (TILES >= TILES_BATCH)>;
    constexpr int kStages = C::kStages, kStaging = C::staging(EPI);
    constexpr bool kSplits = EPI == EPI16_GRAM || EPI == EPI16_POLY || EPI == EPI16_UPDATE, kTwoStages = kSplits && !C::kBoth;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint8_t *smem_a = smem, *smem_b = smem + kStages * C::kABytes;
    uint8_t *smem_boxes = smem + C::kOperands;
    uint64_t *bars = reinterpret_cast<uint64_t *>(smem_boxes + 8 * kStaging);
    // bars[0..7] full, [8..15] empty, [16..17] accumulator full, [18..19] accumulator empty, [20..27] a group's last stage has landed here,
    // [28..35] (leader of a pair) it is ready in the other CTA, [36..43] an epilogue warp's boxes have come ([40..43]
    // in 64 x 64 tiles: lower halves of a tile's sums have been sent, and read), [44..47] a tile is dealt,
    // [48..51] (leader) it has been taken
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(bars + 52);
    volatile uint32_t *abort_flag = tmem_slot + 1;
    int32_t *shared_tiles = reinterpret_cast<int32_t *>(tmem_slot + 2);
    int32_t *start = reinterpret_cast<int32_t *>(reinterpret_cast<uint8_t *>(bars) + C::kTail), *first = start + kMaxGroups16 + 1, *slots = first + kMaxGroups16 + 1;
    uint16_t *order = reinterpret_cast<uint16_t *>(slots + kMaxGroups16 + 1);
    int32_t *dealt = shared_tiles + 1;   // kDealt16 tiles
    static_assert(kStages <= 8 && 52 * 8 + 16 + 4 * kDealt16 <= C::kTail, "barriers");

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t bar_full = smem_u32(bars), bar_empty = smem_u32(bars + 8), bar_acc_full = smem_u32(bars + 16), bar_acc_empty = smem_u32(bars + 18),
                   bar_cut = smem_u32(bars + 20), bar_peer = smem_u32(bars + 28);
    const int rank = CTAS == 2 ? (int)cluster_ctarank() : 0;

    if (warp == 4) {
        mbar_init(smem_u32(bars + lane), lane >= 18 && lane < 20 ? 8 * CTAS : 1);
        // A dealt tile is taken by both producers, the epilogue's warps, the leader's issuer and the other CTA's warp 2.
        if (lane < 20) mbar_init(smem_u32(bars + 32 + lane), lane >= 16 ? (CTAS == 2 ? 22 : 11) : 1);
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
    } else if (warp == 0 && lane == 0) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.a) : "memory");
        if (kSplits && p.split) asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.a2) : "memory");
    } else if (warp == 3 && lane == 0) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.b) : "memory");
        if (kSplits && p.split) asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.b2) : "memory");
    } else if (warp == 5 && lane == 0) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.out) : "memory");
        if (EPI == EPI16_POLY) asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.in) : "memory");
    }
    __syncthreads();
    if (CTAS == 2) { cluster_arrive(); cluster_wait(); }
    tcgen05_fence_after();
    const uint32_t tmem = *tmem_slot;
    // The workspace's settings.  The products of a Newton-Schulz step run behind other kernels of the same call, which is behind whatever
    // wrote them: those are read ahead of the wait.
    uint32_t limit_word = 0u, withhold = 0u;
    auto settings = [&]() {
        limit_word = load_global(p.status + 2);
        if (blockIdx.x == 0) withhold = load_global(p.status + 3);
    };
    if (kSplits) settings();
    wait_for_predecessor();   // from here on global memory is read and written
    if (!kSplits) settings();

    const uint64_t limit = limit_word != 0u ? limit_word : kWaitLimit;
    int m_tiles = p.m_tiles;
    const bool deals = TILES == TILES_CUT && p.deal;
    if (TILES <= TILES_CUT) {
        // A lane of warp 4 has a run of boundaries, up to eight in registers.  Boundaries that fall are lifted; then the row tiles of all groups
        // before a group's are counted (TILES_ROWS).
        if (warp == 4) {
            constexpr int kBM = C::kRows * CTAS, kRun = 8;
            const int run = (p.batch + 32) / 32, g0 = min(lane * run, p.batch + 1), g1 = min(g0 + run, p.batch + 1);
            auto boundary = [&](int g) { return !p.offsets ? (g == 0 ? 0 : (int32_t)p.total_rows) : (int32_t)max((int64_t)0, min(p.total_rows, load_global(p.offsets + g))); };
            int b[kRun], top = 0;
            if (run <= kRun) {
#pragma unroll
                for (int i = 0; i < kRun; i++) b[i] = g0 + i < g1 ? boundary(g0 + i) : 0;
#pragma unroll
                for (int i = 0; i < kRun; i++) top = b[i] = max(top, b[i]);
            } else {
                for (int g = g0; g < g1; g++) start[g] = top = max(top, boundary(g));
            }
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int other = __shfl_up_sync(0xFFFFFFFFu, top, d);
                if (lane >= d) top = max(top, other);
            }
            int before = __shfl_up_sync(0xFFFFFFFFu, top, 1);
            if (lane == 0) before = 0;
            if (run <= kRun) {
#pragma unroll
                for (int i = 0; i < kRun; i++)
                    if (g0 + i < g1) start[g0 + i] = b[i] = max(before, b[i]);
            } else {
                for (int g = g0; g < g1; g++) start[g] = max(before, start[g]);
            }
            if (TILES == TILES_ROWS) {
                __syncwarp();
                const int last = min(g1, p.batch), after = g1 <= p.batch ? start[g1] : 0;   // the boundary behind the run
                int sum = 0;
                if (run <= kRun) {
#pragma unroll
                    for (int i = 0; i < kRun; i++) {
                        const int next = i + 1 < kRun && g0 + i + 1 < g1 ? b[i + 1 < kRun ? i + 1 : 0] : after;
                        b[i] = g0 + i < last ? (next - b[i] + kBM - 1) / kBM : 0;
                        sum += b[i];
                    }
                } else {
                    for (int g = g0; g < last; g++) sum += (group_rows(start, g) + kBM - 1) / kBM;
                }
                before = sum;
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) {
                    const int other = __shfl_up_sync(0xFFFFFFFFu, before, d);
                    if (lane >= d) before += other;
                }
                if (lane == 31) *shared_tiles = before;
                before -= sum;
                if (run <= kRun) {
#pragma unroll
                    for (int i = 0; i < kRun; i++) {
                        if (g0 + i < last) first[g0 + i] = before;
                        before += b[i];
                    }
                } else {
                    for (int g = g0; g < last; g++) {
                        first[g] = before;
                        before += (group_rows(start, g) + kBM - 1) / kBM;
                    }
                }
            }
        }
        __syncthreads();
        if (TILES == TILES_ROWS) m_tiles = *shared_tiles;
        // The groups longest first, then the parts of tiles before each.
        if (!deals || p.batch > kMaxSorted16) order = nullptr;
        if (TILES == TILES_CUT && order) {
            for (int g = threadIdx.x; g < p.batch; g += kThreads16) {
                const int len = group_rows(start, g);
                int place = 0, from = start[0];
#pragma unroll 8
                for (int h = 0; h < p.batch; h++) {
                    const int to = start[h + 1], other = to - from;
                    from = to;
                    place += other > len || (other == len && h < g);
                }
                order[place] = (uint16_t)g;
            }
            __syncthreads();
        }
        if (TILES == TILES_CUT && p.partial) {
            if (warp == 4) {
                const int run = (p.batch + 31) / 32, g0 = min(lane * run, p.batch), last = min(g0 + run, p.batch), each = m_tiles * p.n_tiles;
                int units = 0, places = 0;
                for (int i = g0; i < last; i++) {
                    const int parts = parts16(p, (group_rows(start, order ? order[i] : i) + C::kK - 1) / C::kK);
                    first[i] = units;
                    slots[i] = places;
                    units += parts * each;
                    if (parts > 1) places += parts * each;
                }
                int units_before = units, places_before = places;
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) {
                    const int u = __shfl_up_sync(0xFFFFFFFFu, units_before, d), v = __shfl_up_sync(0xFFFFFFFFu, places_before, d);
                    if (lane >= d) { units_before += u; places_before += v; }
                }
                if (lane == 31) *shared_tiles = units_before;
                units_before -= units;
                places_before -= places;
                for (int i = g0; i < last; i++) { first[i] += units_before; slots[i] += places_before; }
            }
            __syncthreads();
        }
    }
    const int passes = kSplits && p.split ? 2 : 1;   // stages for a piece of the contraction
    const bool both = C::kBoth && p.split;
    const int tiles = TILES == TILES_ROWS ? m_tiles * p.n_tiles : TILES == TILES_CUT && p.partial ? *shared_tiles : TILES <= TILES_BATCH ? p.batch * m_tiles * p.n_tiles
                      : p.batch * (m_tiles * (m_tiles + 1) / 2) * parts16(p, passes * ((p.k + C::kK - 1) / C::kK));   // or parts of tiles
    const int tile0 = blockIdx.x / CTAS, step = gridDim.x / CTAS;
    // Cut contractions differ in length: the tiles may be dealt to the CTAs or pairs as these fall free (128 groups with loads of 302 to 15157 rows:
    // dealt round in turn, the last pair would have 1.4 times the average of stages).  Which CTA has a tile changes nothing in its result.
    Ring16<kDealt16> deal;
    const uint32_t bar_dealt = smem_u32(bars + 44), bar_taken = smem_u32(bars + 48);
    auto next_tile = [&](int tile) {   // the tile after `tile` of this CTA or pair (a warp's first: tile = -1); tiles or more: no more
        if (!deals) return tile < 0 ? tile0 : tile + step;
        if (!warp_wait<CTAS == 2>(bar_dealt + 8 * deal.slot, deal.phase, abort_flag, p.status, limit * 16, 0x900u)) return tiles;
        const int t = dealt[deal.slot];
        __syncwarp();
        if (lane == 0) {
            if (CTAS == 2) mbar_arrive_release_cluster(cluster_addr(bar_taken + 8 * deal.slot, 0));
            else mbar_arrive(bar_taken + 8 * deal.slot);
        }
        deal.next();
        return t;
    };
    if (p.admit) admit_successor();

    if (warp == 0 || warp == 3) {
        // ------------------------------------------------------------------ TMA producers: warp 0 loads A and announces the bytes, warp 3 loads B
        // One thread that issued up to four copies a stage needed 0.55 us for it, longer than the stage's MMAs take.  (What comes out of memory
        // fetched into L2 some stages ahead by the same threads was 2 to 25 % slower: the copies' unit takes 65 bytes a cycle, a stage's 32 KB in
        // as long as its MMAs take, and the fetches pass through it too.)
        const bool a_side = warp == 0;
        uint32_t loads = 0, issued = 0;
        Ring16<kStages> ring;
        bool ok = true;
        const bool issuer = elect_one();
        const uint32_t a0 = smem_u32(smem_a), b0 = smem_u32(smem_b), lead = CTAS == 2 ? cluster_addr(bar_full, 0) : bar_full;
        // The boxes of a stage of this side.  TILES_ROWS and TILES_CUT: the token matrices are one matrix, the weights a stack.
        auto load_stage = [&](const Tile16 &t, int st, int copies, uint32_t to, uint32_t bar, bool in_pair, bool issue) {
            const int left = left16<kSplits, C::kK, C::kBoth>(p, t, st), at0 = t.k0 + t.k_len - left;
            auto load = [&](uint32_t offset, const CUtensorMap *map, int x, int y, int z, bool there) {
                if (CTAS == 2 && in_pair) tma_load_3d<true>(to + offset, map, x, y, z, bar, there);
                else tma_load_3d(to + offset, map, x, y, z, bar, there);
            };
            if (a_side) {
                const CUtensorMap *map = lower16<kTwoStages>(p, st) ? &maps.a2 : &maps.a;
                const int z = TILES <= TILES_CUT ? 0 : t.batch;
                constexpr int kCopies = A_MN ? C::kRows / 64 : C::kRows == 32 ? 2 : 1;
                const uint32_t copy_bytes = A_MN ? 8192u : (uint32_t)p.a_box * 128u;
#pragma unroll
                for (int i = 0; i < C::kBoxes; i++)
#pragma unroll
                    for (int j = 0; j < kCopies; j++) {
                        const bool there = issue && j < copies && (both || i * kBox16 < left);
                        const CUtensorMap *of = both && i == 1 ? &maps.a2 : map;
                        const int at = at0 + (both ? 0 : i * kBox16);
                        if (A_MN) load(i * C::kABox + j * copy_bytes, of, t.a_row + 64 * j, at, z, there);
                        else load(i * C::kABox + j * copy_bytes, of, at, t.a_row + j * p.a_box, z, there);
                    }
            } else {
                const CUtensorMap *map = lower16<kTwoStages>(p, st) ? &maps.b2 : &maps.b;
                const int z = TILES == TILES_CUT ? 0 : t.batch;
#pragma unroll
                for (int i = 0; i < C::kBoxes; i++) {
                    const bool there = issue && (both || i * kBox16 < left);
                    const CUtensorMap *of = both && i == 1 ? &maps.b2 : map;
                    const int at = at0 + (both ? 0 : i * kBox16);
                    if (B_MN) {
#pragma unroll
                        for (int j = 0; j < C::kBRows / 64; j++) load(i * C::kBBox + j * 8192, of, t.b_row + 64 * j, at, z, there);
                    } else {
                        load(i * C::kBBox, of, at, t.b_row, z, there);
                    }
                }
            }
        };
        static_assert(TILES != TILES_SYM || (A_MN == B_MN && C::kABytes == C::kBBytes), "a symmetric product's operands lie alike");
        for (int tile = next_tile(-1); tile < tiles; tile = next_tile(tile)) {
            const Tile16 t = decode16<TILES, CTAS, BN>(p, tile, m_tiles, passes, start, first, slots, order, rank);
            const int a_copies = A_MN ? C::kRows / 64 : (t.rows + p.a_box - 1) / p.a_box;
            const uint32_t a_copy_bytes = A_MN ? 8192u : (uint32_t)p.a_box * 128u;
            const uint32_t a_bytes = (uint32_t)a_copies * a_copy_bytes;   // of this CTA, and of the other
            const uint32_t a_peer = CTAS == 2 ? (uint32_t)(A_MN ? C::kRows / 64 : (t.rows_peer + p.a_box - 1) / p.a_box) * a_copy_bytes : 0u;
            for (int s = t.s0; s < t.s1; s++, ring.next()) {
                if (!warp_wait(bar_empty + 8 * ring.slot, ring.phase ^ 1u, abort_flag, p.status, limit, 0x100u + ring.slot)) { ok = false; break; }
                issued++;
                // A stage with rows behind its group's end lands on a barrier of its own in each CTA, where warp 2 waits for it.
                const int left = left16<kSplits, C::kK, C::kBoth>(p, t, s);
                const bool cut = TILES == TILES_CUT && left < C::kK, own_b = !shares_a<TILES>(t);
                const uint32_t b_bytes = own_b ? (uint32_t)C::kBBox : 0u;
                const int boxes = C::kBoxes == 1 ? 1 : both ? 2 : min(C::kBoxes, (left + kBox16 - 1) / kBox16);
                const uint32_t own_bar = (cut ? bar_cut : bar_full) + 8 * ring.slot, bar = CTAS == 2 && !cut ? lead + 8 * ring.slot : own_bar;
                expect_tx_if(own_bar, (uint32_t)boxes * (a_bytes + b_bytes + (CTAS == 1 || cut ? 0u : a_peer + b_bytes)), issuer && a_side && (rank == 0 || cut));
                if ((a_side || own_b) && (withhold == 0u || !a_side || ++loads != withhold))
                    load_stage(t, s, a_copies, a_side ? a0 + ring.slot * C::kABytes : b0 + ring.slot * C::kBBytes, bar, !cut, issuer);
                __syncwarp();
            }
            if (!ok) break;
        }
        // The MMAs' last reports reach this CTA's barriers while it is still there.
        for (uint32_t i = 0; ok && i < kStages; i++, ring.next())
            if (issued >= kStages - i) ok = warp_wait(bar_empty + 8 * ring.slot, ring.phase ^ 1u, abort_flag, p.status, limit, 0x700u + ring.slot);
    } else if (warp == 1 && rank == 0) {
        // ------------------------------------------------------------------ MMA issuer
        const uint32_t idesc = instr_desc16<CTAS>(p.bf16 != 0, A_MN, B_MN, both ? C::kAccCols : BN);
        Ring16<kStages> ring;
        Ring16<2> acc;      // accumulators
        constexpr bool kPeerFills = TILES == TILES_CUT && CTAS == 2;   // the other CTA's warp 2 has part in "full"
        bool ok = true, ready = false, acc_ready = false;   // the next stage has been seen full, the next accumulator empty
        const bool issuer = elect_one();
        const uint32_t a_desc0 = (uint32_t)(A_MN ? smem_desc_mn_sw128(smem_u32(smem_a)) : smem_desc_sw128(smem_u32(smem_a)));
        const uint32_t b_desc0 = (uint32_t)(B_MN ? smem_desc_mn_sw128(smem_u32(smem_b)) : smem_desc_sw128(smem_u32(smem_b)));
        constexpr uint32_t desc_hi = (1024 >> 4) | (1u << 14) | (2u << 29);   // of either order
        for (int tile = next_tile(-1); tile < tiles; tile = next_tile(tile)) {
            const Tile16 t = decode16<TILES, CTAS, BN>(p, tile, m_tiles, passes, start, first, slots, order, rank);
            const uint32_t b_desc = shares_a<TILES>(t) ? a_desc0 : b_desc0;
            uint32_t d = 0, upper = 0;
            for (int s = t.s0; s < t.s1; s++) {
                const int left = left16<kSplits, C::kK, C::kBoth>(p, t, s), n = s - t.s0;
                constexpr int kChunk = kSumElems / C::kK;
                const bool opens = EPI == EPI16_SUM ? n % kChunk == 0 : n == 0;
                const bool closes = s == t.s1 - 1 || (EPI == EPI16_SUM && n % kChunk == kChunk - 1);
                if (opens) {
                    if (!acc_ready && !warp_wait<CTAS == 2>(bar_acc_empty + 8 * acc.slot, acc.phase ^ 1u, abort_flag, p.status, limit, 0x200u)) { ok = false; break; }
                    d = tmem + acc.slot * C::kAccCols;
                }
                if (!ready && !warp_wait<kPeerFills>(bar_full + 8 * ring.slot, ring.phase, abort_flag, p.status, limit, 0x300u + ring.slot)) { ok = false; break; }
                const uint32_t slot = ring.slot;
                ring.next();
                // Looked at before this stage is issued: afterwards the look would wait for the MMAs.  What it saw is asked for after them.
                const bool full = mbar_look<kPeerFills>(bar_full + 8 * ring.slot, ring.phase);
                bool empty = false;
                const uint32_t acc_bar = 8 * acc.slot;
                if (closes) {
                    acc.next();
                    empty = mbar_look<CTAS == 2>(bar_acc_empty + 8 * acc.slot, acc.phase ^ 1u);
                }
                tcgen05_fence_after();
                auto product = [&](uint32_t a_slot, uint32_t b_slot, bool adds) {
#pragma unroll
                    for (int j = 0; j < 4 * C::kBoxes; j++) {
                        constexpr int kAStep = A_MN ? 2048 : 32, kBStep = B_MN ? 2048 : 32;
                        const uint32_t ad = a_desc0 + ((a_slot * C::kABytes + (j / 4) * C::kABox + (j % 4) * kAStep) >> 4);
                        const uint32_t bd = b_desc + ((b_slot * C::kBBytes + (j / 4) * C::kBBox + (j % 4) * kBStep) >> 4);
                        tcgen05_mma_f16<CTAS>(d, ad, bd, desc_hi, idesc, adds || j > 0, issuer && 16 * j < left && (!both || j < 4));
                    }
                };
                if (lower16<kTwoStages>(p, s)) {   // with the upper parts, which lie in the stage before
                    product(upper, slot, true);
                    product(slot, upper, true);
                    tcgen05_commit_if<CTAS>(bar_empty + 8 * upper, issuer);
                    tcgen05_commit_if<CTAS>(bar_empty + 8 * slot, issuer);
                } else {
                    product(slot, slot, !opens);
                    if (!kTwoStages || !p.split) tcgen05_commit_if<CTAS>(bar_empty + 8 * slot, issuer);
                }
                if (closes) tcgen05_commit_if<CTAS>(bar_acc_full + acc_bar, issuer);
                upper = slot;
                ready = __all_sync(0xFFFFFFFFu, full);
                if (closes) acc_ready = __all_sync(0xFFFFFFFFu, empty);
            }
            if (!ok) break;
        }
    } else if (warp == 2 && TILES == TILES_CUT) {
        // ------------------------------------------------------------------ rows behind a group's end
        // The last stage of a group holds rows of the next one, or whatever lies behind it.  Up to 15 of them meet an MMA: they are zeroed in
        // both operands (in one, an infinity in the other would make NaN).  Then, and in a pair when the other CTA has done the same, the
        // stage is full.  A slot is filled again only when the MMAs have read it, so its barriers are never a phase ahead.
        uint32_t slot = 0, phases = 0;
        // The leader's warp 2 deals: a number from the call's counter is the next tile, for both CTAs, as far ahead as there are places.
        Ring16<kDealt16> dealing;
        int ahead = 0, mine = 0, more = 1, hand[kDealt16];
        auto deal_ahead = [&]() {
            while (rank == 0 && more && ahead < kDealt16) {
                if (!warp_wait<CTAS == 2>(bar_taken + 8 * dealing.slot, dealing.phase ^ 1u, abort_flag, p.status, limit * 16, 0xA00u)) return false;
                int n = 0;
                if (lane == 0) {
                    n = (int)min(atomicAdd(p.deal, 1u), (uint32_t)tiles);
                    dealt[dealing.slot] = n;
                    if (CTAS == 2) {
                        asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(cluster_addr(smem_u32(dealt + dealing.slot), 1)), "r"(n) : "memory");
                        mbar_arrive_release_cluster(cluster_addr(bar_dealt + 8 * dealing.slot, 0));
                        mbar_arrive_release_cluster(cluster_addr(bar_dealt + 8 * dealing.slot, 1));
                    } else {
                        mbar_arrive(bar_dealt + 8 * dealing.slot);
                    }
                }
                n = __shfl_sync(0xFFFFFFFFu, n, 0);
#pragma unroll
                for (int i = 0; i < kDealt16; i++)
                    if (i == (int)dealing.slot) hand[i] = n;
                more = n < tiles;
                ahead++;
                dealing.next();
            }
            return true;
        };
        auto my_tile = [&](int tile) {
            if (!deals || rank != 0) return next_tile(tile);
            if (!deal_ahead()) return tiles;
            int t = tiles;
#pragma unroll
            for (int i = 0; i < kDealt16; i++)
                if (i == mine) t = hand[i];
            mine = mine + 1 == kDealt16 ? 0 : mine + 1;
            ahead--;
            return t;
        };
        for (int tile = my_tile(-1); tile < tiles; tile = my_tile(tile)) {
            const Tile16 t = decode16<TILES, CTAS, BN>(p, tile, m_tiles, passes, start, first, slots, order, rank);
            const int left = t.k_len - (t.s1 - 1) * C::kK;   // rows of the last stage
            if (t.s1 == t.s0 || left >= C::kK) {
                slot = (slot + t.s1 - t.s0) % kStages;
                continue;
            }
            slot = (slot + t.s1 - t.s0 - 1) % kStages;
            const uint32_t parity = (phases >> slot) & 1u;
            phases ^= 1u << slot;
            if (!warp_wait(bar_cut + 8 * slot, parity, abort_flag, p.status, limit, 0x500u + slot)) break;
            const int in_box = left % kBox16, pieces = (((in_box + 15) & ~15) - in_box) * 8;
            const uint32_t box = left / kBox16;   // in_box is 0, and nothing is zeroed, where this box is not there
            for (int c = 0; c < 2 + C::kBRows / 64; c++) {
                uint8_t *chunk = c < 2 ? smem_a + slot * C::kABytes + box * C::kABox + c * 8192 : smem_b + slot * C::kBBytes + box * C::kBBox + (c - 2) * 8192;
                for (int i = lane; i < pieces; i += 32) *reinterpret_cast<uint4 *>(chunk + in_box * 128 + i * 16) = make_uint4(0u, 0u, 0u, 0u);
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (CTAS == 2 && rank == 0) {
                if (!warp_wait<true>(bar_peer + 8 * slot, parity, abort_flag, p.status, limit, 0x400u + slot)) break;
            }
            if (lane == 0) {
                if (rank == 0 && CTAS == 2) mbar_arrive_release_cluster(cluster_addr(bar_full + 8 * slot, 0));
                else if (rank == 0) mbar_arrive(bar_full + 8 * slot);
                else mbar_arrive_release_cluster(cluster_addr(bar_peer + 8 * slot, 0));
            }
            __syncwarp();
            slot = (slot + 1) % kStages;
        }
    } else if (warp >= 4) {
        // ------------------------------------------------------------------ epilogue
        constexpr bool kNarrow = BN == 64 && TILES >= TILES_BATCH;   // four warps have all the columns, the others none
        const int quarter = warp & 3, half = kNarrow ? 0 : (warp - 4) >> 2;
        const uint32_t boxes = smem_u32(smem_boxes) + (warp - 4) * kStaging, bar_box = smem_u32(bars + 36 + warp - 4);
        const Box16 up(boxes, lane), lo(boxes + 4096, lane);
        constexpr int kCols = kNarrow ? BN : BN / 2, kChunk = EPI == EPI16_SUM || kCols < 64 ? 32 : 64;   // a warp's columns, and those of a box
        Ring16<2> acc;
        uint32_t box_phase = 0, second = 0, half_phase = 0;
        for (int tile = next_tile(-1); tile < tiles; tile = next_tile(tile)) {
            const Tile16 t = decode16<TILES, CTAS, BN>(p, tile, m_tiles, passes, start, first, slots, order, rank);
            const int in = 32 * quarter + lane;
            const int elems = (t.s1 - t.s0) * C::kK, chunks = EPI == EPI16_SUM ? (elems + kSumElems - 1) / kSumElems : elems > 0;   // accumulators of the tile
            const uint64_t acc_limit = limit * (uint64_t)(1 + (t.k_len >> 8));
            const uint32_t from = tmem + half * kCols + ((uint32_t)(32 * quarter) << 16);
            const int col0 = t.col + half * kCols, row0 = t.row + 32 * quarter, rows = kNarrow && warp >= 8 ? 0 : t.rows - 32 * quarter;   // this warp's first column and row, its rows
            const int batch = TILES == TILES_ROWS ? 0 : t.batch;
            const int64_t row = (TILES == TILES_CUT ? (int64_t)t.batch * p.m : 0) + t.row + in;
            // The accumulator may be overwritten as soon as all warps have it in registers: reads of tensor memory, which the fence orders, and
            // nothing else.  (Release at cluster scope, here and in the leader's own CTA too, held the warp up for 0.7 us.)
            auto release = [&]() {
                tcgen05_fence_before();
                __syncwarp();
                if (lane == 0) {
                    const uint32_t bar = bar_acc_empty + 8 * acc.slot;
                    if (rank != 0) mbar_arrive_cluster(cluster_addr(bar, 0));
                    else mbar_arrive(bar);
                }
                __syncwarp();
            };
            // Parts: this one's accumulator, columns c and up, goes to its place; the sum of all parts comes from there.
            constexpr bool kParts = TILES == TILES_CUT || (TILES == TILES_SYM && EPI == EPI16_GRAM);
            const int64_t place = kParts ? ((int64_t)(t.slot0 * CTAS + rank) * 8 + (warp - 4)) * (32 * kCols) + 4 * lane : 0;
            constexpr int64_t kPlace = (int64_t)CTAS * 8 * 32 * kCols;
            auto put_part = [&](const float *v, int c, int n) {
                float4 *to = reinterpret_cast<float4 *>(p.partial + place + (t.s0 / p.part_stages) * kPlace + 32 * c);
#pragma unroll
                for (int e = 0; e < n; e += 4) to[8 * e] = make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]);
            };
            // Several parts are on their way at a time; they are added in their order all the same.
            auto add_parts = [&](float *v, int c, int n) {
                constexpr bool kFull = EPI == EPI16_SUM && kCols > 64;               // the sums take most of the registers
                constexpr int kBatch = kFull ? 16 : 32, kWay = kFull ? 2 : 3;   // columns, and parts of them
#pragma unroll
                for (int e0 = 0; e0 < n; e0 += kBatch) {
                    const float4 *from = reinterpret_cast<const float4 *>(p.partial + place + 32 * (c + e0));
#pragma unroll
                    for (int e = 0; e < kBatch; e++) v[e0 + e] = 0.f;
                    for (int i = 0; i < t.parts; i += kWay) {
                        float4 x[kWay][kBatch / 4];
#pragma unroll
                        for (int w = 0; w < kWay; w++)
#pragma unroll
                            for (int e = 0; e < kBatch / 4; e++) x[w][e] = i + w < t.parts ? __ldcg(from + (i + w) * (kPlace / 4) + 32 * e) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                        for (int w = 0; w < kWay; w++)
#pragma unroll
                            for (int e = 0; e < kBatch / 4; e++) {
                                v[e0 + 4 * e] += x[w][e].x; v[e0 + 4 * e + 1] += x[w][e].y; v[e0 + 4 * e + 2] += x[w][e].z; v[e0 + 4 * e + 3] += x[w][e].w;
                            }
                    }
                }
            };
            auto last_part = [&]() {   // whether all the others have been put
                __threadfence();
                __syncwarp();
                uint32_t before = 0;
                if (lane == 0) {
                    uint32_t *counter = p.counters + (t.counter * CTAS + rank) * 8 + warp - 4;
                    before = atomicAdd(counter, 1u);
                    if (before == (uint32_t)t.parts - 1u) *counter = 0u;
                }
                before = __shfl_sync(0xFFFFFFFFu, before, 0);
                __threadfence();
                return before == (uint32_t)t.parts - 1u;
            };
            // A box leaves.  Rows of a group's last box, which shares its rows with the next group, and a row's last bytes leave by themselves.
            auto send = [&](const uint32_t *w, const float *v, int col) {
                if (col < p.boxed && rows >= (TILES == TILES_ROWS ? 32 : 1)) {
                    if (TWO) {   // the store before the last has read the box that is next
                        if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
                        __syncwarp();
                        if (second) lo.put(w);
                        else up.put(w);
                    } else {
                        boxes_free(lane);
                        up.put(w);
                    }
                    fence_async_shared();
                    __syncwarp();
                    if (lane == 0) {
                        if (EPI == EPI16_SUM && p.accumulate) tma_reduce_add_3d(&maps.out, col, row0, batch, boxes + second);
                        else tma_store_3d(&maps.out, col, row0, batch, boxes + second);
                        bulk_commit();
                    }
                    if (TWO) second ^= 4096u;
                    if (col + kChunk > p.boxed && lane < rows) {
#pragma unroll
                        for (int e = 0; e < kChunk; e++) {
                            if (col + e < p.boxed || col + e >= p.n) continue;
                            if (EPI == EPI16_SUM) {
                                float *c = static_cast<float *>(p.c) + row * p.ldc + col + e;
                                *c = p.accumulate ? *c + v[e] : v[e];
                            } else static_cast<__nv_bfloat16 *>(p.c)[row * p.ldc + col + e] = __float2bfloat16_rn(v[e]);
                        }
                    }
                } else if (lane < rows) {
#pragma unroll
                    for (int e = 0; e < kChunk; e += 32) {
                        if (EPI == EPI16_SUM) store_f32(p, row, col + e, v + e);
                        else store_bf16(p, row, col + e, v + e);
                    }
                }
                __syncwarp();
            };
            if (EPI == EPI16_SUM) {
                float sum[kCols];
#pragma unroll
                for (int e = 0; e < kCols; e++) sum[e] = 0.f;
                bool ok = true;
                for (int k = 0; k < chunks; k++, acc.next()) {
                    if (!warp_wait(bar_acc_full + 8 * acc.slot, acc.phase, abort_flag, p.status, acc_limit, 0x600u)) { ok = false; break; }
                    tcgen05_fence_after();
#pragma unroll
                    for (int c = 0; c < kCols; c += 16) {
                        uint32_t v[16];
                        FP4Q_TMEM_LD_X16(from + acc.slot * C::kAccCols + c, v);
                        asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
                        for (int e = 0; e < 16; e++) sum[c + e] += __uint_as_float(v[e]);
                    }
                    release();
                }
                if (!ok) break;
                if (kParts && t.parts > 1) {
                    if (rows <= 0 || col0 >= p.n) continue;
                    put_part(sum, 0, kCols);
                    if (!last_part()) continue;
                    add_parts(sum, 0, kCols);
                }
                if (chunks > 0 || !p.accumulate) {
#pragma unroll
                    for (int c = 0; c < kCols; c += kChunk) send(reinterpret_cast<const uint32_t *>(sum) + c, sum + c, col0 + c);
                }
                continue;
            }
            // What a step's epilogue reads is fetched before it waits for the accumulator, and for a later chunk when the one before has left.
            // P has a I in it, so that the product brings a X as well; a times X's lower part is left to add, or nothing where that is an operand too.
            const bool two = EPI == EPI16_UPDATE || p.split != 0;      // upper and lower parts
            const bool reads_up = EPI == EPI16_POLY, reads_lo = EPI == EPI16_UPDATE ? p.split == 0 : EPI == EPI16_POLY && p.split != 0;
            const bool reads = reads_up || reads_lo;
            // The scale that a small X has beside the usual one, now and in the next step.
            float fa = p.fa, fb = p.fb, fc = p.fc;
            if (EPI == EPI16_GRAM || EPI == EPI16_UPDATE) {
                const int lift = load_global(p.lift + t.batch), now = max(0, lift - p.grown), next = p.o ? 0 : max(0, lift - p.grown_next);
                const float by = power_of_two(EPI == EPI16_GRAM ? -2 * now : next - now);
                fa *= by; fb *= by; fc *= by;
            }
            auto fetch = [&](int col) {
                if (!reads || rows <= 0 || col >= p.n) return;
                boxes_free(lane);
                if (lane == 0) {
                    mbar_arrive_expect_tx(bar_box, reads_up && reads_lo ? 8192u : 4096u);
                    if (reads_up) tma_load_3d(boxes, &maps.in, col, row0, batch, bar_box);
                    if (reads_lo) tma_load_3d(boxes + 4096, &maps.in2, col, row0, batch, bar_box);
                }
            };
            fetch(col0);
            if (chunks > 0) {
                if (!warp_wait(bar_acc_full + 8 * acc.slot, acc.phase, abort_flag, p.status, acc_limit, 0x600u)) break;
                tcgen05_fence_after();
            }
            bool ok = true;
            if (kParts && t.parts > 1) {
#pragma unroll 1
                for (int c = 0; c < kCols; c += 32) {
                    uint32_t v[32];
                    FP4Q_TMEM_LD_X32(from + acc.slot * C::kAccCols + c, v);
                    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
                    if (c == kCols - 32) release();
                    if (rows > 0 && col0 + c < p.n) put_part(reinterpret_cast<const float *>(v), c, 32);
                }
                acc.next();
                if (rows <= 0 || col0 >= p.n || !last_part()) continue;
            }
#pragma unroll 1
            for (int c = 0; c < kCols; c += kChunk) {
                uint32_t v[kChunk];
                const int col = col0 + c;
                if (kParts && t.parts > 1) {
                    if (col < p.n) add_parts(reinterpret_cast<float *>(v), c, kChunk);
                } else if (chunks > 0) {
#pragma unroll
                    for (int e = 0; e < kChunk; e += 32) FP4Q_TMEM_LD_X32(from + acc.slot * C::kAccCols + c + e, (v + e));
                    if (C::kBoth && both) {
                        float *sum = reinterpret_cast<float *>(v);
#pragma unroll
                        for (int e = 0; e < kChunk; e += 32) {
                            uint32_t u[32];
                            FP4Q_TMEM_LD_X32(from + acc.slot * C::kAccCols + BN + e, u);
                            asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
                            for (int i = 0; i < 32; i++) sum[e + i] += __uint_as_float(u[i]);
                        }
                        release();
                        // The lower halves, of warps 6 and 7, are added to the upper ones, of warps 4 and 5, by way of their boxes.
                        const uint32_t half_box = smem_u32(smem_boxes) + (quarter | 2) * kStaging + lane * 256;
                        const uint32_t sent = smem_u32(bars + 40 + (quarter & 1)), read = smem_u32(bars + 42 + (quarter & 1));   // warps 8 to 11 have no boxes
                        if (warp >= 6 && warp < 8) {
                            if (!warp_wait(read, half_phase ^ 1u, abort_flag, p.status, limit, 0xB00u)) { ok = false; break; }
#pragma unroll
                            for (int i = 0; i < kChunk / 4; i++) st_shared_16(half_box + ((i ^ (lane & 7)) << 4), v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
                            __syncwarp();
                            if (lane == 0) mbar_arrive(sent);
                        } else if (warp < 6) {
                            if (!warp_wait(sent, half_phase, abort_flag, p.status, limit, 0xC00u)) { ok = false; break; }
#pragma unroll
                            for (int i = 0; i < kChunk / 4; i++) {
                                const uint4 w = ld_shared_16(half_box + ((i ^ (lane & 7)) << 4));
                                sum[4 * i] += __uint_as_float(w.x); sum[4 * i + 1] += __uint_as_float(w.y); sum[4 * i + 2] += __uint_as_float(w.z); sum[4 * i + 3] += __uint_as_float(w.w);
                            }
                            __syncwarp();
                            if (lane == 0) mbar_arrive(read);
                        }
                        half_phase ^= 1u;
                    } else {
                        asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
                        if (c == kCols - kChunk) release();
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < kChunk; e++) v[e] = 0u;
                }
                const float *x = reinterpret_cast<const float *>(v);
                if (EPI == EPI16_STORE) {
                    uint32_t w[32];
#pragma unroll
                    for (int e = 0; e < kChunk / 2; e++) w[e] = pack_bf16(x[2 * e], x[2 * e + 1]);
                    if (kChunk == 64) send(w, x, col);
                    else if (lane < rows) store_bf16(p, row, col, x);   // half a box
                    __syncwarp();
                    continue;
                }
                if (rows <= 0 || col >= p.n) continue;
                if (reads) {
                    if (!warp_wait(bar_box, box_phase, abort_flag, p.status, limit, 0x800u)) { ok = false; break; }
                    box_phase ^= 1u;
                }
                // The new values, upper and lower parts, replace those that were read, a piece of eight columns at a time.
                const bool out = EPI == EPI16_UPDATE && p.o;
                if (!reads) boxes_free(lane);
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    float w[8];
                    const uint4 a = reads_up ? ld_shared_16(up.piece(i)) : make_uint4(0u, 0u, 0u, 0u), b = reads_lo ? ld_shared_16(lo.piece(i)) : make_uint4(0u, 0u, 0u, 0u);
                    const uint32_t au[4] = {a.x, a.y, a.z, a.w}, bu[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
                    for (int j = 0; j < 4; j++) {
                        const float2 y = unpack_half(au[j]), z = unpack_half(bu[j]);
                        const float v0 = x[8 * i + 2 * j], v1 = x[8 * i + 2 * j + 1];
                        w[2 * j] = EPI == EPI16_GRAM ? v0 * fa : fmaf(fb, y.x + z.x, fc * v0);
                        w[2 * j + 1] = EPI == EPI16_GRAM ? v1 * fa : fmaf(fb, y.y + z.y, fc * v1);
                    }
                    uint32_t h[4], l[4];
                    if (out) {
#pragma unroll
                        for (int j = 0; j < 4; j++) h[j] = pack_bf16(w[2 * j] * p.o_scale, w[2 * j + 1] * p.o_scale);
                    } else {
#pragma unroll
                        for (int j = 0; j < 4; j++) {
                            h[j] = pack_half(w[2 * j], w[2 * j + 1]);
                            const float2 y = unpack_half(h[j]);
                            l[j] = pack_half(w[2 * j] - y.x, w[2 * j + 1] - y.y);
                        }
                        if (two || EPI == EPI16_POLY) st_shared_16(lo.piece(i), l[0], l[1], l[2], l[3]);
                    }
                    st_shared_16(up.piece(i), h[0], h[1], h[2], h[3]);
                }
                if (EPI == EPI16_POLY) {   // a I: this row's element in the box, if it has one
                    // From both parts, whether the lower one leaves or not: b A + c A A may nearly cancel a, which would magnify its rounding.  (Added to the FP32
                    // values instead, the code of 64 columns, fetched anew by every kernel, cost 0.8 us a step.)
                    const uint32_t e = (uint32_t)(row0 + lane - col);
                    if (e < 64u) {
                        const uint32_t at = (e & 7u) * 2u;
                        uint16_t h, l;
                        asm volatile("ld.shared.u16 %0, [%1];" : "=h"(h) : "r"(up.piece(e >> 3) + at) : "memory");
                        asm volatile("ld.shared.u16 %0, [%1];" : "=h"(l) : "r"(lo.piece(e >> 3) + at) : "memory");
                        const float w = unpack_half(h).x + unpack_half(l).x + p.fa;
                        const uint32_t v_up = pack_half(w, 0.f), v_lo = pack_half(w - unpack_half(v_up).x, 0.f);
                        asm volatile("st.shared.u16 [%0], %1;" ::"r"(up.piece(e >> 3) + at), "h"((uint16_t)v_up) : "memory");
                        if (two) asm volatile("st.shared.u16 [%0], %1;" ::"r"(lo.piece(e >> 3) + at), "h"((uint16_t)v_lo) : "memory");
                    }
                }
                fence_async_shared();
                __syncwarp();
                if (out && col + kChunk > p.boxed) {
                    // Columns that do not leave in boxes: row by row, two columns of a row a lane.
                    __nv_bfloat16 *o = p.o + ((int64_t)t.batch * p.m + row0) * p.ld_o + col;
                    const int left = p.n - col, c0 = 2 * lane;
#pragma unroll 4
                    for (int r = 0; r < 32; r++) {
                        if (r >= rows) break;
                        uint32_t w;
                        asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w) : "r"(boxes + r * 128 + ((((uint32_t)lane >> 2) ^ (r & 7)) << 4) + (lane & 3) * 4) : "memory");
                        const __nv_bfloat162 pair = *reinterpret_cast<const __nv_bfloat162 *>(&w);
                        if (c0 < left && col + c0 >= p.boxed) o[r * p.ld_o + c0] = pair.x;
                        if (c0 + 1 < left && col + c0 >= p.boxed) o[r * p.ld_o + c0 + 1] = pair.y;
                    }
                    __syncwarp();
                }
                if (lane == 0 && !(out && col >= p.boxed)) {
                    tma_store_3d(&maps.out, col, row0, batch, boxes);
                    if (two && !out) tma_store_3d(&maps.out2, col, row0, batch, boxes + 4096);
                    bulk_commit();
                }
                if (EPI != EPI16_UPDATE && t.mirror) {
                    // The transposed box, 64 rows of 64 bytes, in place of the box itself once that has left.  A lane gives the addresses of its
                    // row's pieces: four blocks of 8 x 8 at a time are read transposed, and written where they then belong.
                    uint32_t block_up[32], block_lo[32];
#pragma unroll
                    for (int i = 0; i < 8; i++) {
                        load_blocks_transposed(up.piece(i), block_up + 4 * i);
                        if (two) load_blocks_transposed(lo.piece(i), block_lo + 4 * i);
                    }
                    boxes_free(lane);
                    const uint32_t there = boxes + (lane & 7) * 64 + (lane >> 3) * 16;
#pragma unroll
                    for (int i = 0; i < 8; i++) {
                        store_blocks(there + i * 512, block_up + 4 * i);
                        if (two) store_blocks(there + 4096 + i * 512, block_lo + 4 * i);
                    }
                    fence_async_shared();
                    __syncwarp();
                    if (lane == 0) {
                        tma_store_3d(&maps.mirror, row0, col, batch, boxes);
                        if (two) tma_store_3d(&maps.mirror2, row0, col, batch, boxes + 4096);
                        bulk_commit();
                    }
                }
                if (c + kChunk < kCols) fetch(col + kChunk);
            }
            if (!ok) break;
            if (chunks > 0 && !(kParts && t.parts > 1)) acc.next();
        }
        // The stores have read shared memory; what they write is there when the grid has completed.
        boxes_free(lane);
    }

    if (TILES == TILES_ROWS && p.zero_rest && warp >= 4) {
        constexpr int kElem = EPI == EPI16_SUM ? 4 : 2;
        const int64_t head = start[0], rest = head + p.total_rows - start[p.batch];
        const int64_t halves = (int64_t)p.n * kElem / 2, pieces = halves / 8;
        for (int64_t i = blockIdx.x * 8 + warp - 4; i < rest; i += gridDim.x * 8) {
            uint8_t *row = static_cast<uint8_t *>(p.c) + (i < head ? i : start[p.batch] + i - head) * p.ldc * kElem;
            for (int64_t e = lane; e < pieces; e += 32) reinterpret_cast<uint4 *>(row)[e] = make_uint4(0u, 0u, 0u, 0u);
            for (int64_t e = pieces * 8 + lane; e < halves; e += 32) reinterpret_cast<uint16_t *>(row)[e] = 0;
        }
    }

    // Shared memory and tensor memory stay until all roles, of both CTAs of a pair, have done with them.  Where a wait has run out, copies and
    // MMAs may still be under way: they take microseconds, a millisecond is left to them.
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

// A stack of `batch` matrices [rows, cols], `pitch` elements from row to row and `stride` from matrix to matrix.
struct Operand16 {
    const void *base;
    int64_t cols, rows, batch, pitch, stride;
};
inline bool make_map16(CUtensorMap *map, const Operand16 &o, int box_cols, int box_rows, CUtensorMapSwizzle swizzle = CU_TENSOR_MAP_SWIZZLE_128B, bool f32 = false)
{
    const cuuint64_t dims[3] = {(cuuint64_t)o.cols, (cuuint64_t)o.rows, (cuuint64_t)o.batch};
    const cuuint64_t strides[2] = {(cuuint64_t)o.pitch * (f32 ? 4 : 2), (cuuint64_t)o.stride * (f32 ? 4 : 2)};
    const cuuint32_t box[3] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows, 1u};
    return encode_tiled(map, f32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_UINT16, 3, const_cast<void *>(o.base), dims, strides, box, swizzle,
                        CU_TENSOR_MAP_L2_PROMOTION_L2_256B);
}

// maps: what lies beside the operands is the caller's.  a2, b2: the operands' lower parts (p.split).  most_tiles: no fewer than the tiles
// there can be.
template <int CTAS, int BN, bool A_MN, bool B_MN, int EPI, int TILES, bool TWO = false>
fp4q_status launch_gemm16(const Operand16 &a, const Operand16 &b, const Operand16 &a2, const Operand16 &b2, Maps16 &maps, Gemm16Params p, int64_t most_tiles,
                          cudaStream_t stream)
{
    p.by_matrix = Divisor16::of(TILES == TILES_SYM ? (int64_t)p.m_tiles * (p.m_tiles + 1) / 2 : (int64_t)p.m_tiles * p.n_tiles);
    p.by_band = Divisor16::of((int64_t)kRaster16 * p.n_tiles);
    using C = Cfg16<CTAS, BN, TWO, (TILES >= TILES_BATCH)>;
    const int a_rows = A_MN ? kBox16 : p.a_box, b_rows = B_MN ? kBox16 : C::kBRows;
    if (!make_map16(&maps.a, a, kBox16, a_rows) || !make_map16(&maps.b, b, kBox16, b_rows)) return FP4Q_ERR_CUDA;
    if (p.split && (!make_map16(&maps.a2, a2, kBox16, a_rows) || !make_map16(&maps.b2, b2, kBox16, b_rows))) return FP4Q_ERR_CUDA;
    const int dev = current_device();
    if (dev < 0) return FP4Q_ERR_CUDA;
    constexpr int kSmem = C::smem(TILES, EPI);
    static std::atomic<bool> attr_set[kMaxDevices];   // the attribute is a property of (kernel, device)
    if (!attr_set[dev].load(std::memory_order_relaxed)) {
        if (cudaFuncSetAttribute(gemm16_kernel<CTAS, BN, A_MN, B_MN, EPI, TILES, TWO>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem) != cudaSuccess) {
            cudaGetLastError();
            return FP4Q_ERR_CUDA;
        }
        attr_set[dev].store(true, std::memory_order_relaxed);
    }
    const int64_t slots = sm_count(dev) / CTAS;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[2];
    cfg.gridDim = dim3((unsigned)(CTAS * (most_tiles < slots ? most_tiles : slots)));
    cfg.blockDim = dim3(kThreads16);
    cfg.dynamicSmemBytes = kSmem;
    cfg.stream = stream;
    cfg.attrs = attr;
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.numAttrs = 1;
    if (CTAS == 2) {
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = CTAS;
        attr[1].val.clusterDim.y = 1;
        attr[1].val.clusterDim.z = 1;
        cfg.numAttrs = 2;
    }
    return launched(cudaLaunchKernelEx(&cfg, gemm16_kernel<CTAS, BN, A_MN, B_MN, EPI, TILES, TWO>, maps, p));
}

}  // namespace fp4q
