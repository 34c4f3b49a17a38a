// BF16 products of groups of rows that start anywhere: forward, input gradient, weight gradient (include/fp4q.h).  The kernel and its
// variants are in gemm16.cuh; here are the arguments' checks and the choice of a variant.
#include "gemm16.cuh"

#include <algorithm>
#include <cmath>

using namespace fp4q;

namespace {

const int kOutFlags = (int)FP4Q_OUT_PADDED | (int)FP4Q_OUT_ZERO_REST;
const int64_t kMaxDim16 = 0x7FFFFFFF - 4096;

struct Matrix16 {
    const void *p;
    int64_t rows, cols, ld;
};

fp4q_status check_groups16(const fp4q_groups *g)
{
    if (!g) return FP4Q_OK;
    if (g->n_groups <= 0) return FP4Q_ERR_SHAPE;
    if (g->row_alignment != 0 && g->row_alignment != 1 && g->row_alignment != 128 && g->row_alignment != 256) return FP4Q_ERR_UNSUPPORTED;
    if (g->n_groups > kMaxGroups16) return FP4Q_ERR_UNSUPPORTED;
    if (!g->row_offsets) return FP4Q_ERR_NULL;
    return FP4Q_OK;
}
fp4q_status check_shape16(const Matrix16 &m)
{
    if (m.rows < 0 || m.cols < 0 || m.ld < m.cols) return FP4Q_ERR_SHAPE;
    return m.rows > kMaxDim16 || m.cols > kMaxDim16 ? FP4Q_ERR_UNSUPPORTED : FP4Q_OK;
}
fp4q_status check_operand16(const Matrix16 &m)
{
    if (m.rows == 0 || m.cols == 0) return FP4Q_OK;
    if (!m.p) return FP4Q_ERR_NULL;
    return aligned(m.p, 16) && m.ld % 8 == 0 ? FP4Q_OK : FP4Q_ERR_ALIGN;
}
bool type_ok(fp4q_out dt)
{
    const int type = (int)dt & ~kOutFlags;
    return type == FP4Q_OUT_BF16 || type == FP4Q_OUT_F32;
}
bool out_f32(fp4q_out dt) { return ((int)dt & ~kOutFlags) == FP4Q_OUT_F32; }
fp4q_status check_output16(void *c, int64_t ldc, int64_t cols, fp4q_out dt, Gemm16Params &p)
{
    if (!c) return FP4Q_ERR_NULL;
    if (ldc < cols) return FP4Q_ERR_SHAPE;
    const int64_t bytes = out_f32(dt) ? 4 : 2;
    if (!aligned(c, 16) || ldc * bytes % 16 != 0) return FP4Q_ERR_ALIGN;
    p.c = c;
    p.ldc = ldc;
    p.zero_rest = ((int)dt & (int)FP4Q_OUT_ZERO_REST) != 0;
    p.wide = aligned(c, 32) && ldc * bytes % 32 == 0;
    return FP4Q_OK;
}
fp4q_status check_workspace(const void *ws, size_t ws_bytes)
{
    if (!ws || ws_bytes < sizeof(Workspace)) return FP4Q_ERR_WORKSPACE;
    return aligned(ws, 256) ? FP4Q_OK : FP4Q_ERR_ALIGN;
}
Operand16 operand16(const Matrix16 &m, int64_t rows, int64_t batch) { return Operand16{m.p, m.cols, rows, batch, m.ld, rows * m.ld}; }

template <int CTAS, int BN, bool A_MN, bool B_MN, int TILES, bool TWO = false>
fp4q_status launch_store16(const Operand16 &a, const Operand16 &b, Gemm16Params &p, fp4q_out dt, int64_t most_tiles, cudaStream_t stream)
{
    Maps16 maps = {};
    const bool f32 = out_f32(dt);
    p.boxed = p.n / (f32 ? 4 : 8) * (f32 ? 4 : 8);   // a store of a box fills the 16 bytes in which a row ends
    const int64_t groups = TILES == TILES_CUT ? p.batch : 1;
    if (p.boxed > 0 && !make_map16(&maps.out, Operand16{p.c, p.boxed, p.m, groups, p.ldc, p.m * p.ldc}, f32 ? 32 : 64, 32, CU_TENSOR_MAP_SWIZZLE_128B, f32)) return FP4Q_ERR_CUDA;
    return f32 ? launch_gemm16<CTAS, BN, A_MN, B_MN, EPI16_SUM, TILES, TWO>(a, b, a, b, maps, p, most_tiles, stream)
               : launch_gemm16<CTAS, BN, A_MN, B_MN, EPI16_STORE, TILES, TWO>(a, b, a, b, maps, p, most_tiles, stream);
}

// What a product of rows in tiles of rows x cols takes, in us, where `groups` groups may have rows and each fills its last tile by half: rounds of tiles
// over the GPU's slots, per tile `each` us beside its boxes, of which an SM gets 115 GB/s from L2 and all of them together 15 TB/s.  (Where the rule decides,
// the variant it takes and the next: 64 rows in one group, 4096 x 4096, 32 x 64 tiles 13.6 us and pairs 24.2; 600 in 4, 2048 x 1024, 128 x 128 tiles 9.5
// and pairs 11.9; 1531 in 8, 1003 x 2731, 17.2 and 20.6; 1999 in 13 pairs 22.0 and 30.6; 3000 in 100, 2048 x 768, 32 x 64 60.5 and 69.)
double rows_cost(int64_t T, int64_t groups, int64_t n, int64_t k, int rows, int cols, int slots, double box_bytes, int ctas, double each)
{
    const double row_tiles = groups == 1 ? (double)ceil_div(T, rows) : std::max<double>((double)groups, (double)T / rows + 0.5 * groups), tiles = row_tiles * ceil_div(n, cols);
    const double rate = std::min(115e3, 15e6 / (ctas * std::min<double>(tiles, slots)));   // bytes a us
    return std::ceil(tiles / slots) * (each + (double)ceil_div(k, 64) * box_bytes / rate);
}

// Rows of groups, T in all.  Pairs for groups of many rows, tiles of 32 rows for groups of few, 128 x 128 between them.
template <bool B_MN>
fp4q_status rows_product(const Operand16 &a, const Operand16 &b, Gemm16Params &p, fp4q_out dt, int64_t T, int64_t groups, cudaStream_t stream)
{
    const int64_t few = T < groups ? T : groups;   // groups that have rows, at most
    const int box = T <= 16 * few ? 16 : 32;
    const double pairs = rows_cost(T, few, p.n, p.k, 256, 256, 74, 32768.0, 2, 3.6), singles = rows_cost(T, few, p.n, p.k, 128, 128, 148, 32768.0, 1, 3.0),
                 small = rows_cost(T, few, p.n, p.k, 32, 64, 148, 8192.0 + 128.0 * box, 1, 0.6);
    const double least = std::min(pairs, std::min(singles, small));
    p.a_box = 128;
    if (least == pairs) {
        p.n_tiles = (int32_t)ceil_div(p.n, 256);
        return launch_store16<2, 256, false, B_MN, TILES_ROWS>(a, b, p, dt, (T / 256 + few) * p.n_tiles, stream);
    }
    if (least == singles) {
        p.n_tiles = (int32_t)ceil_div(p.n, 128);
        return launch_store16<1, 128, false, B_MN, TILES_ROWS>(a, b, p, dt, (T / 128 + few) * p.n_tiles, stream);
    }
    p.a_box = box;
    p.n_tiles = (int32_t)ceil_div(p.n, 64);
    return launch_store16<1, 64, false, B_MN, TILES_ROWS>(a, b, p, dt, (T / 32 + few) * p.n_tiles, stream);
}

// which: 0 = Y = X W^T, 1 = dX = dY W.
fp4q_status rows_call(int which, const Matrix16 &x, const Matrix16 &w, void *c, int64_t ldc, fp4q_out dt, const fp4q_groups *g, void *ws, size_t ws_bytes, void *stream)
{
    if (fp4q_status s = check_groups16(g)) return s;
    if (!type_ok(dt)) return FP4Q_ERR_UNSUPPORTED;
    if (fp4q_status s = check_shape16(x)) return s;
    if (fp4q_status s = check_shape16(w)) return s;
    const int64_t groups = g ? g->n_groups : 1;
    if (w.rows % groups) return FP4Q_ERR_SHAPE;
    const int64_t out_features = w.rows / groups, contraction = which ? out_features : w.cols, cols = which ? w.cols : out_features;
    if (x.cols != contraction) return FP4Q_ERR_SHAPE;
    if (x.rows == 0 || cols == 0) return FP4Q_OK;
    Gemm16Params p = {};
    if (fp4q_status s = check_output16(c, ldc, cols, dt, p)) return s;
    if (fp4q_status s = check_operand16(x)) return s;
    if (fp4q_status s = check_operand16(w)) return s;
    if (fp4q_status s = check_workspace(ws, ws_bytes)) return s;
    if ((x.rows / 32 + groups) * ceil_div(cols, 64) > kMaxDim16) return FP4Q_ERR_UNSUPPORTED;   // tiles are counted in 32 bits
    p.m = (int32_t)x.rows;
    p.n = (int32_t)cols;
    p.k = (int32_t)contraction;
    p.batch = (int32_t)groups;
    p.bf16 = 1;
    p.offsets = g ? g->row_offsets : nullptr;
    p.total_rows = x.rows;
    p.status = static_cast<uint32_t *>(ws);
    // Without a contraction nothing is read: the maps describe some memory, the output's.
    const Operand16 a = contraction ? operand16(x, x.rows, 1) : Operand16{c, 8, 1, 1, 8, 8};
    const Operand16 b = contraction ? operand16(w, out_features, groups) : a;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    return which ? rows_product<true>(a, b, p, dt, x.rows, groups, s) : rows_product<false>(a, b, p, dt, x.rows, groups, s);
}

}  // namespace

extern "C" fp4q_status fp4q_ragged_gemm_fwd(const void *x, int64_t T, int64_t K, int64_t ldx, const void *w, int64_t w_rows, int64_t ldw, void *Y, int64_t ldy,
                                            fp4q_out dt, const fp4q_groups *g, void *ws, size_t ws_bytes, void *stream)
{
    return rows_call(0, Matrix16{x, T, K, ldx}, Matrix16{w, w_rows, K, ldw}, Y, ldy, dt, g, ws, ws_bytes, stream);
}

extern "C" fp4q_status fp4q_ragged_gemm_dgrad(const void *dY, int64_t T, int64_t N, int64_t ld_dy, const void *w, int64_t w_rows, int64_t K, int64_t ldw, void *dX,
                                              int64_t ldx, fp4q_out dt, const fp4q_groups *g, void *ws, size_t ws_bytes, void *stream)
{
    return rows_call(1, Matrix16{dY, T, N, ld_dy}, Matrix16{w, w_rows, K, ldw}, dX, ldx, dt, g, ws, ws_bytes, stream);
}

namespace {

// How a weight gradient is computed: in pairs' tiles or single CTAs', and the parts that long contractions are cut into: a group of most of the rows
// has few tiles, which would otherwise leave most of the GPU idle.  Estimated for groups of the same length: rounds of tiles or of their parts, a box
// 0.38 us in a pair and 0.285 in a single CTA (0.32 with all of them at work), 3.3 and 1.7 us a tile, and where there are parts 3 us and 1.4 or 0.7 us
// for each, which whoever comes last reads.  Groups longer than the others are cut at half of what a CTA or pair would have to do if all had the same.
// (131072 rows in 4 groups, 256 x 256: 9 parts in single CTAs 39 us, 32 parts in pairs 198; 131072 in one, 768 x 2048: 3 parts in pairs 300, 14 of them
// 411, single CTAs 544; 8192 in 2, 2048 x 2048: uncut in pairs 55, in parts of 56 stages 111, single CTAs 82.)  Where the output is BF16 no part is longer
// than kMostStages: its accumulators are cut off towards zero, by 5e-9 of a sum of one sign for every row, which adds up (2^20 rows, 768 x 2048, in 3 parts:
// 2.5e-3 too small in the mean, half a step of BF16 being 2 to 4e-3; in parts of this length 0.3e-3).
//
// Where there are parts, groups of several lengths are dealt to whoever is free, by a counter, but not where every tile has a CTA or pair to itself
// (65536 rows in 64 skewed groups, 1024 x 1024: 190 us dealt, 224 in turn; 32768 in 16, 2048 x 1024: 152 and 169).  Without parts a group
// alone fills the GPU, or all are short, and tiles go in turn (8192 rows in 32, 4096 x 2048: 348 us dealt, 276 in turn; 1024 in 4, 768 x 2048: 14.6 and 12.3).  The counters of a
// call lie in its own scratch memory, so that calls which share a workspace do not meddle with one another's tiles.
struct CutPlan {
    static constexpr int64_t kDealBytes = 256, kMostStages = 2048;
    bool pairs = false, cut = false, deals = false;   // without scratch memory neither parts nor dealing
    int64_t m_tiles, n_tiles, part_stages = 0, places = 0, most_tiles, counter_bytes = 0;   // counters: the tiles dealt, then those of the parts
    size_t bytes = 0;
    CutPlan(int64_t T, int64_t N, int64_t K, int64_t groups, bool scratch, bool f32)
    {
        const int64_t stages = ceil_div(T, kBox16);
        const double mean = std::max(1.0, (double)stages / groups + (groups > 1 ? 0.5 : 0.0));   // stages of a group
        double least = 1e30;
        for (int two = 0; two < (N > 128 && K > 128 ? 2 : 1); two++) {
            const int64_t edge = two ? 256 : 128, slots = two ? 74 : 148, tiles = groups * ceil_div(N, edge) * ceil_div(K, edge);
            const int64_t fewest = scratch && !f32 ? (int64_t)std::ceil(mean / kMostStages) : 1, most = scratch ? std::max(fewest > 1 ? fewest + 2 : 1, std::min<int64_t>(64, (int64_t)mean / 16)) : 1;
            for (int64_t n = fewest; n <= most; n++) {
                const double box = two ? 0.38 : tiles * n >= slots ? 0.32 : 0.285;
                const double us = (double)ceil_div(tiles * n, slots) * (std::ceil(mean / n) * box + (two ? 3.3 : 1.7)) + (n > 1 ? 3.0 + (two ? 1.4 : 0.7) * (double)n : 0.0);
                if (us >= least) continue;
                least = us;
                pairs = two != 0;
                const double half = (double)tiles * mean / (2.0 * slots);
                part_stages = round_up(std::max<int64_t>(16, (int64_t)std::ceil(n > 1 ? mean / n : std::max(half, 1.25 * mean))), 8);
            }
        }
        if (!f32) part_stages = std::min(part_stages, kMostStages);
        m_tiles = ceil_div(N, pairs ? 256 : 128);
        n_tiles = ceil_div(K, pairs ? 256 : 128);
        const int64_t each = m_tiles * n_tiles;
        most_tiles = groups * each;
        cut = scratch && stages > part_stages;
        if (!cut) return;
        // Groups with more stages than a part: no more than this, and with so many parts.
        const int64_t longer = std::min(groups, stages / part_stages + 1);
        places = each * (ceil_div(stages + longer, part_stages) + longer);
        most_tiles += places;
        deals = groups > 1 && T >= 256 * groups && most_tiles > (pairs ? 74 : 148);
        counter_bytes = kDealBytes + round_up(places * (pairs ? 2 : 1) * 8 * 4, 256);
        bytes = (size_t)(counter_bytes + places * (pairs ? Cfg16<2, 256>::kPlaceBytes : Cfg16<1, 128>::kPlaceBytes));
    }
};

// Tiles, and parts of them, are counted in 32 bits.
bool tiles_fit(int64_t T, int64_t N, int64_t K, int64_t groups)
{
    const int64_t each = ceil_div(N, 128) * ceil_div(K, 128);
    return groups * each <= kMaxDim16 / 2 && each * ceil_div(T, 1024) <= kMaxDim16 / 4;
}

}  // namespace

extern "C" size_t fp4q_ragged_gemm_wgrad_scratch_bytes(int64_t T, int64_t N, int64_t K, int32_t n_groups)
{
    if (T <= 0 || N <= 0 || K <= 0 || n_groups <= 0 || n_groups > kMaxGroups16 || T > kMaxDim16 || N > kMaxDim16 || K > kMaxDim16) return 0;
    return tiles_fit(T, N, K, n_groups) ? std::max(CutPlan(T, N, K, n_groups, true, false).bytes, CutPlan(T, N, K, n_groups, true, true).bytes) : 0;   // of either type
}

extern "C" fp4q_status fp4q_ragged_gemm_wgrad(const void *dY, int64_t T, int64_t N, int64_t ld_dy, const void *x, int64_t K, int64_t ldx, void *dW, int64_t ldw,
                                              fp4q_out dt, int accumulate, const fp4q_groups *g, void *scratch, size_t scratch_bytes, void *ws, size_t ws_bytes, void *stream)
{
    const Matrix16 d = {dY, T, N, ld_dy}, m = {x, T, K, ldx};
    if (fp4q_status s = check_groups16(g)) return s;
    if (!type_ok(dt)) return FP4Q_ERR_UNSUPPORTED;
    if (fp4q_status s = check_shape16(d)) return s;
    if (fp4q_status s = check_shape16(m)) return s;
    const int64_t groups = g ? g->n_groups : 1;
    if (N == 0 || K == 0) return FP4Q_OK;
    Gemm16Params p = {};
    if (fp4q_status s = check_output16(dW, ldw, K, dt, p)) return s;
    if (accumulate && !out_f32(dt)) return FP4Q_ERR_UNSUPPORTED;
    if (fp4q_status s = check_operand16(d)) return s;
    if (fp4q_status s = check_operand16(m)) return s;
    if (fp4q_status s = check_workspace(ws, ws_bytes)) return s;
    if (!tiles_fit(T, N, K, groups)) return FP4Q_ERR_UNSUPPORTED;
    const CutPlan plan(T, N, K, groups, scratch != nullptr, out_f32(dt));
    if (scratch && scratch_bytes < plan.bytes) return FP4Q_ERR_WORKSPACE;
    if (scratch && !aligned(scratch, 256)) return FP4Q_ERR_ALIGN;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    p.m = (int32_t)N;
    p.n = (int32_t)K;
    p.k = (int32_t)T;
    p.m_tiles = (int32_t)plan.m_tiles;
    p.n_tiles = (int32_t)plan.n_tiles;
    p.batch = (int32_t)groups;
    p.bf16 = 1;
    p.a_box = 128;
    p.offsets = g ? g->row_offsets : nullptr;
    p.total_rows = T;
    p.accumulate = accumulate != 0;
    p.status = static_cast<uint32_t *>(ws);
    if (plan.bytes) {
        uint8_t *counters = static_cast<uint8_t *>(scratch);
        if (plan.deals) p.deal = reinterpret_cast<uint32_t *>(counters);
        p.part_stages = (int32_t)plan.part_stages;
        p.counters = reinterpret_cast<uint32_t *>(counters + CutPlan::kDealBytes);
        p.partial = reinterpret_cast<float *>(counters + plan.counter_bytes);
        if (fp4q_status st = launched(cudaMemsetAsync(scratch, 0, (size_t)plan.counter_bytes, s))) return st;
    }
    const Operand16 a = T ? operand16(d, T, 1) : Operand16{dW, 8, 1, 1, 8, 8}, b = T ? operand16(m, T, 1) : a;
    if (T < 256 * groups)   // short contractions
        return plan.pairs ? launch_store16<2, 256, true, true, TILES_CUT, true>(a, b, p, dt, plan.most_tiles, s) : launch_store16<1, 128, true, true, TILES_CUT, true>(a, b, p, dt, plan.most_tiles, s);
    return plan.pairs ? launch_store16<2, 256, true, true, TILES_CUT>(a, b, p, dt, plan.most_tiles, s) : launch_store16<1, 128, true, true, TILES_CUT>(a, b, p, dt, plan.most_tiles, s);
}
