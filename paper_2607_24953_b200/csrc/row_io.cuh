// Rows of BF16 or FP32 that start on any element: 8 or 16 consecutive elements of a row per lane, read and written in aligned 16-byte pieces.
#pragma once

#include <cuda_bf16.h>

#include "common.cuh"

namespace fp4q {

// A matrix of T.
template <typename T>
struct RowsOf {
    T *p;
    int64_t ld;
};
template <typename T>
inline RowsOf<T> rows_of(const void *p, int64_t ld) { return RowsOf<T>{static_cast<T *>(const_cast<void *>(p)), ld}; }

// Whether rows of `size` bytes an element begin on 16 bytes.
inline bool on_grid(const void *p, int64_t ld, int64_t rows, size_t size) { return !p || (aligned(p, 16) && (rows <= 1 || ld * (int64_t)size % 16 == 0)); }

__device__ __forceinline__ uint32_t pack_pair(float lo, float hi)
{
    const __nv_bfloat162 b = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&b);
}
__device__ __forceinline__ void store_element(float *p, float v) { *p = v; }
__device__ __forceinline__ void store_element(__nv_bfloat16 *p, float v) { *p = __float2bfloat16_rn(v); }
__device__ __forceinline__ float rounded(float v, const float *) { return v; }
__device__ __forceinline__ float rounded(float v, const __nv_bfloat16 *) { return __bfloat162float(__float2bfloat16_rn(v)); }

// E (8 or 16) elements as they lie in memory: pairs of BF16 or FP32 in words.
template <typename T, int E = 16>
struct Raw {
    static constexpr int kWords = (int)sizeof(T) * E / 4;
    uint32_t w[kWords];
    __device__ __forceinline__ float operator[](int e) const
    {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[e]);
        else return __uint_as_float((e & 1) ? w[e >> 1] & 0xFFFF0000u : w[e >> 1] << 16);
    }
    __device__ __forceinline__ void set(const float (&v)[E])
    {
#pragma unroll
        for (int i = 0; i < kWords; i++) {
            if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(v[i]);
            else w[i] = pack_pair(v[2 * i], v[2 * i + 1]);
        }
    }
};

// The words of a run of bytes that begins `off` bytes (0 to 15, whole elements) behind the first one: in place of w.
template <int N, int KEEP>
__device__ __forceinline__ void drop_bytes(uint32_t (&w)[N], uint32_t off)
{
    if (off & 8u)
#pragma unroll
        for (int i = 0; i + 2 < N; i++) w[i] = w[i + 2];
    if (off & 4u)
#pragma unroll
        for (int i = 0; i + 1 < N; i++) w[i] = w[i + 1];
    if (off & 2u)
#pragma unroll
        for (int i = 0; i < KEEP; i++) w[i] = __funnelshift_r(w[i], w[i + 1 < N ? i + 1 : i], 16);
}

// How many of the columns c0 .. c0 + E - 1 exist.
template <int E = 16>
__device__ __forceinline__ int columns_at(int64_t c0, int64_t cols) { return c0 >= cols ? 0 : cols - c0 < E ? (int)(cols - c0) : E; }

// Columns c0 .. c0 + E - 1 of row i, of which the first n exist, on their way: the 16-byte pieces that hold them, read whole (an allocation begins and ends on 16 bytes).  Nothing here waits for what
// is read.  GRID: rows begin on 16 bytes.
template <typename T, bool GRID, int E = 16>
struct Pieces {
    static constexpr int kWords = Raw<T, E>::kWords + (GRID ? 0 : 4);
    uint32_t w[kWords];
    __device__ __forceinline__ void fetch(const RowsOf<T> &m, int64_t i, int64_t c0, int n)
    {
        const uintptr_t at = reinterpret_cast<uintptr_t>(m.p + i * m.ld + c0);
        const uint32_t off = GRID ? 0u : (uint32_t)at & 15u;
        const int pieces = n > 0 ? (int)(off + n * (uint32_t)sizeof(T) + 15u) >> 4 : 0;
        const uint4 *src = reinterpret_cast<const uint4 *>(at - off);
#pragma unroll
        for (int k = 0; k < kWords / 4; k++) {
            uint4 v = make_uint4(0u, 0u, 0u, 0u);
            if (k < pieces) v = load_global(src + k);
            w[4 * k] = v.x; w[4 * k + 1] = v.y; w[4 * k + 2] = v.z; w[4 * k + 3] = v.w;
        }
    }
    // The elements, zeros behind the first n.
    __device__ __forceinline__ Raw<T, E> land(const RowsOf<T> &m, int64_t i, int64_t c0, int n)
    {
        constexpr int W = Raw<T, E>::kWords;
        if constexpr (!GRID) drop_bytes<kWords, W>(w, (uint32_t)reinterpret_cast<uintptr_t>(m.p + i * m.ld + c0) & 15u);
        Raw<T, E> r;
#pragma unroll
        for (int k = 0; k < W; k++) r.w[k] = w[k];
        if (n < E) {
#pragma unroll
            for (int k = 0; k < W; k++) {
                if constexpr (sizeof(T) == 4) r.w[k] = k < n ? r.w[k] : 0u;
                else r.w[k] = 2 * k + 1 < n ? r.w[k] : 2 * k < n ? r.w[k] & 0xFFFFu : 0u;
            }
        }
        return r;
    }
};
template <typename T, bool GRID = false, int E = 16>
__device__ __forceinline__ Raw<T, E> load_row(const RowsOf<T> &m, int64_t i, int64_t c0, int n)
{
    Pieces<T, GRID, E> p;
    p.fetch(m, i, c0, n);
    return p.land(m, i, c0, n);
}

// The same columns written, the first n.  All lanes of the warp come here; lanes next to one another in a run of `team` (a power of two up to 32) have neighbouring
// columns of one row.  Rows off the 16-byte grid: a lane writes the pieces that begin in it and, with its neighbour's last elements, the one before; where the
// neighbour has none, or not all, of its elements, each writes its own one by one.
template <typename T, bool GRID = false, int E = 16>
__device__ __forceinline__ void store_row(const RowsOf<T> &m, int64_t i, int64_t c0, int n, const Raw<T, E> &r, int team)
{
    constexpr int W = Raw<T, E>::kWords, P = W / 4, S = (int)sizeof(T);
    T *dst = m.p + i * m.ld + c0;
    if constexpr (GRID) {
        if (n == E) {
#pragma unroll
            for (int k = 0; k < P; k++) reinterpret_cast<uint4 *>(dst)[k] = make_uint4(r.w[4 * k], r.w[4 * k + 1], r.w[4 * k + 2], r.w[4 * k + 3]);
        } else if (n > 0) {
#pragma unroll
            for (int e = 0; e < E; e++)
                if (e < n) {
                    if constexpr (S == 4) reinterpret_cast<uint32_t *>(dst)[e] = r.w[e];
                    else reinterpret_cast<uint16_t *>(dst)[e] = (uint16_t)(r.w[e >> 1] >> (16 * (e & 1)));
                }
        }
        return;
    }
    const uint32_t off = (uint32_t)reinterpret_cast<uintptr_t>(dst) & 15u;
    const bool full = n == E;
    if (__all_sync(0xFFFFFFFFu, n == 0 || (full && off == 0u))) {
        if (full)
#pragma unroll
            for (int k = 0; k < P; k++) reinterpret_cast<uint4 *>(dst)[k] = make_uint4(r.w[4 * k], r.w[4 * k + 1], r.w[4 * k + 2], r.w[4 * k + 3]);
        return;
    }
    const int lane = threadIdx.x & 31, in = lane & (team - 1);
    uint32_t w[W + 4];
#pragma unroll
    for (int k = 0; k < 4; k++) w[k] = __shfl_up_sync(0xFFFFFFFFu, r.w[W - 4 + k], 1);
#pragma unroll
    for (int k = 0; k < W; k++) w[4 + k] = r.w[k];
    const uint32_t fulls = __ballot_sync(0xFFFFFFFFu, full);
    const bool before = in > 0 && (fulls >> ((lane - 1) & 31) & 1u), behind = in < team - 1 && (fulls >> ((lane + 1) & 31) & 1u);
    int lo = 0, hi = n;   // elements written one by one: below lo, and from hi on
    if (full) {
        drop_bytes<W + 4, W>(w, off ? 16u - off : 0u);
        if (off == 0u) {
#pragma unroll
            for (int k = 0; k < W; k++) w[k] = r.w[k];
        }
        uint4 *to = reinterpret_cast<uint4 *>(reinterpret_cast<uintptr_t>(dst) - off);
#pragma unroll
        for (int k = 0; k < P; k++)
            if (k > 0 || before || off == 0u) to[k] = make_uint4(w[4 * k], w[4 * k + 1], w[4 * k + 2], w[4 * k + 3]);
        lo = before || off == 0u ? 0 : (int)(16u - off) / S;
        hi = behind ? E : E - (int)off / S;
    } else {
        lo = n;
    }
    if (lo > 0 || hi < n) {
#pragma unroll
        for (int e = 0; e < E; e++)
            if (e < n && (e < lo || e >= hi)) {
                if constexpr (S == 4) reinterpret_cast<uint32_t *>(dst)[e] = r.w[e];
                else reinterpret_cast<uint16_t *>(dst)[e] = (uint16_t)(r.w[e >> 1] >> (16 * (e & 1)));
            }
    }
}

}  // namespace fp4q
