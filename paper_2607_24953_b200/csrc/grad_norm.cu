// fp4q_global_norm and fp4q_clip_by_norm (include/fp4q.h): the norm of all gradients of a step, and their clipping.
//
// Every tensor is cut into units of 8 elements, those of a row on the 16-byte grid of its memory, and chunks of 1024 units, which the CTAs take in turn; the
// tensors' descriptions travel as kernel parameters, up to 450 a launch.  Bound by memory: the norm reads everything, the clipping reads it again, last
// chunks first, since those are still in L2, and writes it.  202 M FP32 elements into BF16 312 us: 124 for the norm (6.5 TB/s), 181 for the scaling (6.7).
#include <cuda_bf16.h>

#include "common.cuh"
#include "row_io.cuh"

#include <algorithm>

using namespace fp4q;

namespace {

constexpr int kUnit = 8, kChunkUnits = 1024;   // four units a thread
constexpr int kNormCtas = 148 * 6;
constexpr int kFew = 56, kMany = 450;          // tensors of a launch: parameters of up to 4 and 32 KB

struct Span {
    void *data, *out;
    int64_t units_row, units, cols, ld, ld_out;   // units of a row and of the tensor; a tensor without gaps is one row
    int64_t chunk0;                               // chunks of the tensors before it
    int32_t f32, out_f32;
};
template <int N>
struct SpanParams {
    int64_t chunks;
    int32_t n, in_place;
    double *partial;
    int64_t parts;          // scaling: sums that the norm is the root of, and where it goes; 0: the norm is there
    float *norm;
    float max_norm, eps;
    Span span[N];
};
static_assert(sizeof(SpanParams<kFew>) <= 4096 && sizeof(SpanParams<kMany>) <= 32764, "a kernel's parameters");

// The tensor that a chunk belongs to: the last one that begins at or before it.
template <int N>
__device__ __forceinline__ int span_of(const SpanParams<N> &p, int64_t chunk)
{
    int lo = 0, hi = p.n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (p.span[mid].chunk0 <= chunk) lo = mid;
        else hi = mid;
    }
    return lo;
}

// A unit: element e of its row's columns k .. k + 7 (k may begin before the row).
struct Unit {
    int64_t row, col;
    bool whole;   // all eight exist; they lie on 16 bytes
};
__device__ __forceinline__ Unit unit_of(const Span &s, int64_t u)
{
    Unit r;
    r.row = 0;
    if (s.units != s.units_row) {
        r.row = s.units <= 0xFFFFFFFFll ? (uint32_t)u / (uint32_t)s.units_row : u / s.units_row;
        u -= r.row * s.units_row;
    }
    const uintptr_t at = reinterpret_cast<uintptr_t>(s.data) + (uintptr_t)(r.row * s.ld) * (s.f32 ? 4 : 2);
    r.col = u * kUnit - (int64_t)((at & 15u) >> (s.f32 ? 2 : 1));
    r.whole = r.col >= 0 && r.col + kUnit <= s.cols;
    return r;
}
__device__ __forceinline__ void load_unit(const Span &s, const Unit &u, bool exists, uint32_t (&w)[8])
{
#pragma unroll
    for (int i = 0; i < 8; i++) w[i] = 0u;
    if (!exists) return;
    const int64_t at = u.row * s.ld + u.col;
    if (u.whole) {
        const uint4 *src = s.f32 ? reinterpret_cast<const uint4 *>(static_cast<const float *>(s.data) + at) : reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(s.data) + at);
        const uint4 a = load_global(src);
        w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w;
        if (s.f32) {
            const uint4 b = load_global(src + 1);
            w[4] = b.x; w[5] = b.y; w[6] = b.z; w[7] = b.w;
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < kUnit; e++) {
        if (u.col + e < 0 || u.col + e >= s.cols) continue;
        if (s.f32) w[e] = load_global(static_cast<const uint32_t *>(s.data) + at + e);
        else w[e >> 1] |= (uint32_t)load_global(static_cast<const uint16_t *>(s.data) + at + e) << (16 * (e & 1));
    }
}
__device__ __forceinline__ float element(const Span &s, const uint32_t (&w)[8], int e)
{
    return s.f32 ? __uint_as_float(w[e]) : __uint_as_float((e & 1) ? w[e >> 1] & 0xFFFF0000u : w[e >> 1] << 16);
}

// A chunk all of whose units are whole and lie behind one another: its first element, else NULL.
__device__ __forceinline__ const void *solid_chunk(const Span &s, int64_t u0)
{
    const uintptr_t skip = (reinterpret_cast<uintptr_t>(s.data) & 15u) >> (s.f32 ? 2 : 1);
    const int64_t col = u0 * kUnit - (int64_t)skip;
    if (s.units != s.units_row || col < 0 || col + kChunkUnits * kUnit > s.cols) return nullptr;
    return static_cast<const uint8_t *>(s.data) + col * (s.f32 ? 4 : 2);
}
__device__ __forceinline__ float low(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// A run of 32 squares.  One that is normal has lost no square that counts; another one, with squares out of FP32's range, is added up in 64 bits.
template <typename F>
__device__ __forceinline__ double sum_run(F value)
{
    float run = 0.f;
#pragma unroll
    for (int e = 0; e < 32; e++) run = fmaf(value(e), value(e), run);
    double total = (double)run;
    if (!(run > 1e-30f && run < 1e38f)) {
        total = 0.0;
#pragma unroll
        for (int e = 0; e < 32; e++) {
            const double v = (double)value(e);
            total = fma(v, v, total);
        }
    }
    return total;
}

template <int N>
__global__ void __launch_bounds__(256) sum_squares_kernel(const __grid_constant__ SpanParams<N> p)
{
    wait_for_predecessor();
    admit_successor();
    __shared__ double sums[8];
    double total = 0.0;
    for (int64_t chunk = blockIdx.x; chunk < p.chunks; chunk += gridDim.x) {
        const Span &s = p.span[span_of(p, chunk)];
        const int64_t u0 = (chunk - s.chunk0) * kChunkUnits + threadIdx.x;
        const uint4 *solid = static_cast<const uint4 *>(solid_chunk(s, u0 - threadIdx.x));
        if (solid) {
            uint4 v[8];
            const int n = s.f32 ? 8 : 4;
#pragma unroll
            for (int k = 0; k < 8; k++)
                if (k < n) v[k] = load_global(solid + 256 * k + threadIdx.x);
            if (s.f32) total += sum_run([&](int e) { return __uint_as_float(e % 4 == 0 ? v[e / 4].x : e % 4 == 1 ? v[e / 4].y : e % 4 == 2 ? v[e / 4].z : v[e / 4].w); });
            else
                total += sum_run([&](int e) {
                    const uint32_t w = e / 2 % 4 == 0 ? v[e / 8].x : e / 2 % 4 == 1 ? v[e / 8].y : e / 2 % 4 == 2 ? v[e / 8].z : v[e / 8].w;
                    return e % 2 ? high(w) : low(w);
                });
            continue;
        }
        uint32_t w[4][8];
#pragma unroll
        for (int k = 0; k < 4; k++) {
            const int64_t u = u0 + 256 * k;
            load_unit(s, unit_of(s, u), u < s.units, w[k]);
        }
        total += sum_run([&](int e) { return element(s, w[e / 8], e % 8); });
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) total += __shfl_xor_sync(0xFFFFFFFFu, total, d);
    if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = total;
    __syncthreads();
    if (threadIdx.x != 0) return;
    total = 0.0;
#pragma unroll
    for (int k = 0; k < 8; k++) total += sums[k];
    p.partial[blockIdx.x] = total;
}

// The root of the sum of the CTAs' sums, the same in every CTA of 256 threads that comes here.
__device__ __forceinline__ float root_of(const double *partial, int64_t n, double *shared)
{
    double total = 0.0;
    for (int64_t i = threadIdx.x; i < n; i += 256) total += load_global(partial + i);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) total += __shfl_xor_sync(0xFFFFFFFFu, total, d);
    if ((threadIdx.x & 31) == 0) shared[threadIdx.x >> 5] = total;
    __syncthreads();
    total = 0.0;
#pragma unroll
    for (int k = 0; k < 8; k++) total += shared[k];
    return (float)sqrt(total);
}

struct RootParams {
    const double *partial;
    int64_t n;
    float *norm;
};
__global__ void __launch_bounds__(256) root_kernel(const __grid_constant__ RootParams p)
{
    wait_for_predecessor();
    admit_successor();
    __shared__ double sums[8];
    const float norm = root_of(p.partial, p.n, sums);
    if (threadIdx.x == 0) *p.norm = norm;
}

template <int N>
__global__ void __launch_bounds__(256) scale_kernel(const __grid_constant__ SpanParams<N> p)
{
    wait_for_predecessor();
    admit_successor();
    __shared__ double sums[8];
    const float norm = p.parts ? root_of(p.partial, p.parts, sums) : load_global(p.norm);
    if (p.parts && blockIdx.x == 0 && threadIdx.x == 0) *p.norm = norm;
    const float bound = norm + p.eps, ratio = __fdiv_rn(p.max_norm, bound), factor = ratio > 1.f || bound == 0.f ? 1.f : ratio;   // zeros stay zeros
    if (p.in_place && factor == 1.f) return;
    for (int64_t back = blockIdx.x; back < p.chunks; back += gridDim.x) {
        const int64_t chunk = p.chunks - 1 - back;
        const Span &s = p.span[span_of(p, chunk)];
        const int64_t u0 = (chunk - s.chunk0) * kChunkUnits + threadIdx.x;
        const uint4 *solid = static_cast<const uint4 *>(solid_chunk(s, u0 - threadIdx.x));
        const int64_t start = solid ? (reinterpret_cast<uintptr_t>(solid) - reinterpret_cast<uintptr_t>(s.data)) >> (s.f32 ? 2 : 1) : 0;
        uint8_t *to = static_cast<uint8_t *>(s.out) + start * (s.out_f32 ? 4 : 2);
        if (solid && (reinterpret_cast<uintptr_t>(to) & 15u) == 0u) {
            uint4 v[8];
            const int n = s.f32 ? 8 : 4;
#pragma unroll
            for (int k = 0; k < 8; k++)
                if (k < n) v[k] = load_global(solid + 256 * k + threadIdx.x);
#pragma unroll
            for (int k = 0; k < 8; k++) {
                if (k >= n) break;
                const int at = 256 * k + threadIdx.x;
                const uint32_t *w = reinterpret_cast<const uint32_t *>(&v[k]);
                if (s.f32) {
                    const float a = __uint_as_float(w[0]) * factor, b = __uint_as_float(w[1]) * factor, c = __uint_as_float(w[2]) * factor, d = __uint_as_float(w[3]) * factor;
                    if (s.out_f32) reinterpret_cast<float4 *>(to)[at] = make_float4(a, b, c, d);
                    else reinterpret_cast<uint2 *>(to)[at] = make_uint2(pack_pair(a, b), pack_pair(c, d));
                } else if (s.out_f32) {
                    reinterpret_cast<float4 *>(to)[2 * at] = make_float4(low(w[0]) * factor, high(w[0]) * factor, low(w[1]) * factor, high(w[1]) * factor);
                    reinterpret_cast<float4 *>(to)[2 * at + 1] = make_float4(low(w[2]) * factor, high(w[2]) * factor, low(w[3]) * factor, high(w[3]) * factor);
                } else {
                    reinterpret_cast<uint4 *>(to)[at] = make_uint4(pack_pair(low(w[0]) * factor, high(w[0]) * factor), pack_pair(low(w[1]) * factor, high(w[1]) * factor),
                                                                   pack_pair(low(w[2]) * factor, high(w[2]) * factor), pack_pair(low(w[3]) * factor, high(w[3]) * factor));
                }
            }
            continue;
        }
        uint32_t w[4][8];
#pragma unroll
        for (int k = 0; k < 4; k++) {
            const int64_t u = u0 + 256 * k;
            load_unit(s, unit_of(s, u), u < s.units, w[k]);
        }
#pragma unroll
        for (int k = 0; k < 4; k++) {
            const int64_t u = u0 + 256 * k;
            if (u >= s.units) continue;
            const Unit at = unit_of(s, u);
            float v[kUnit];
#pragma unroll
            for (int e = 0; e < kUnit; e++) v[e] = element(s, w[k], e) * factor;
            const int64_t where = at.row * s.ld_out + at.col;
            if (s.out_f32) {
                float *o = static_cast<float *>(s.out) + where;
                if (at.whole && (reinterpret_cast<uintptr_t>(o) & 15u) == 0u) {
                    reinterpret_cast<float4 *>(o)[0] = make_float4(v[0], v[1], v[2], v[3]);
                    reinterpret_cast<float4 *>(o)[1] = make_float4(v[4], v[5], v[6], v[7]);
                } else {
#pragma unroll
                    for (int e = 0; e < kUnit; e++)
                        if (at.col + e >= 0 && at.col + e < s.cols) o[e] = v[e];
                }
            } else {
                __nv_bfloat16 *o = static_cast<__nv_bfloat16 *>(s.out) + where;
                if (at.whole && (reinterpret_cast<uintptr_t>(o) & 15u) == 0u) {
                    uint32_t b[4];
#pragma unroll
                    for (int e = 0; e < 4; e++) b[e] = pack_pair(v[2 * e], v[2 * e + 1]);
                    *reinterpret_cast<uint4 *>(o) = make_uint4(b[0], b[1], b[2], b[3]);
                } else {
#pragma unroll
                    for (int e = 0; e < kUnit; e++)
                        if (at.col + e >= 0 && at.col + e < s.cols) o[e] = __float2bfloat16_rn(v[e]);
                }
            }
        }
    }
}

fp4q_status check_span(const fp4q_span &t)
{
    if (t.rows < 0 || t.cols < 0) return FP4Q_ERR_SHAPE;
    if (t.type != FP4Q_OUT_BF16 && t.type != FP4Q_OUT_F32) return FP4Q_ERR_UNSUPPORTED;
    if (t.rows == 0 || t.cols == 0) return FP4Q_OK;
    if (!t.data) return FP4Q_ERR_NULL;
    if (t.rows > 1 && t.ld < t.cols) return FP4Q_ERR_SHAPE;
    return aligned(t.data, t.type == FP4Q_OUT_F32 ? 4 : 2) ? FP4Q_OK : FP4Q_ERR_ALIGN;
}
fp4q_status check_spans(const fp4q_span *t, int32_t n)
{
    if (n < 0) return FP4Q_ERR_SHAPE;
    if (n > 0 && !t) return FP4Q_ERR_NULL;
    for (int32_t i = 0; i < n; i++)
        if (fp4q_status s = check_span(t[i])) return s;
    return FP4Q_OK;
}

// As the kernels take it.  o: the tensor that the result goes to.
Span span_for(const fp4q_span &t, const fp4q_span &o)
{
    Span s = {};
    s.data = t.data;
    s.out = o.data;
    s.f32 = t.type == FP4Q_OUT_F32;
    s.out_f32 = o.type == FP4Q_OUT_F32;
    const bool gaps = t.rows > 1 && (t.ld != t.cols || o.ld != o.cols);
    const int64_t rows = gaps ? t.rows : 1, size = s.f32 ? 4 : 2;
    s.cols = gaps ? t.cols : t.rows * t.cols;
    s.ld = t.ld;
    s.ld_out = o.ld;
    // A row off the grid has one unit more.
    const bool off = !aligned(t.data, 16) || (rows > 1 && t.ld * size % 16 != 0);
    s.units_row = (s.cols + kUnit - 1 + (off ? 16 / size - 1 : 0)) / kUnit;
    s.units = rows * s.units_row;
    return s;
}

// The tensors from `at` on that are not empty, as many as there is room for; at: the first that is left.
template <int N>
int64_t take_spans(const fp4q_span *t, const fp4q_span *o, int32_t n, int32_t &at, SpanParams<N> &p)
{
    for (; at < n && p.n < N; at++) {
        if (t[at].rows == 0 || t[at].cols == 0) continue;
        Span &s = p.span[p.n++] = span_for(t[at], o[at]);
        s.chunk0 = p.chunks;
        p.chunks += ceil_div(s.units, kChunkUnits);
    }
    return std::min<int64_t>(kNormCtas, p.chunks);
}

// The tensors' sums of squares, one for every CTA; parts: how many.
fp4q_status launch_sums(const fp4q_span *tensors, int32_t n, double *partial, int64_t &parts, cudaStream_t s)
{
    fp4q_status st = FP4Q_OK;
    parts = 0;
    auto launch = [&](auto &p, auto kernel, int32_t &at) {
        p.partial = partial + parts;
        const int64_t ctas = take_spans(tensors, tensors, n, at, p);
        parts += ctas;
        if (ctas) st = launched(launch_dependent(kernel, dim3((unsigned)ctas), 256, s, p));
    };
    for (int32_t at = 0; at < n && !st;) {
        if (n - at <= kFew) {
            SpanParams<kFew> p = {};
            launch(p, sum_squares_kernel<kFew>, at);
        } else {
            SpanParams<kMany> p = {};
            launch(p, sum_squares_kernel<kMany>, at);
        }
    }
    return st;
}
// parts: the norm is still to be taken from so many sums (and nothing may have overwritten them when the last launch has begun); 0: it is there.
fp4q_status launch_scaling(const fp4q_span *tensors, const fp4q_span *outs, int32_t n, float *norm, double *partial, int64_t parts, float max_norm, float eps, cudaStream_t s)
{
    fp4q_status st = FP4Q_OK;
    auto launch = [&](auto &p, auto kernel, int32_t &at) {
        p.norm = norm;
        p.partial = partial;
        p.parts = parts;
        p.max_norm = max_norm;
        p.eps = eps;
        p.in_place = !outs;
        const int64_t ctas = take_spans(tensors, outs ? outs : tensors, n, at, p);
        if (ctas) st = launched(launch_dependent(kernel, dim3((unsigned)ctas), 256, s, p));
    };
    for (int32_t at = 0; at < n && !st;) {
        if (n - at <= kFew) {
            SpanParams<kFew> p = {};
            launch(p, scale_kernel<kFew>, at);
        } else {
            SpanParams<kMany> p = {};
            launch(p, scale_kernel<kMany>, at);
        }
    }
    return st;
}
fp4q_status check_norm(const float *norm, const fp4q_span *tensors, int32_t n, void *scratch, size_t scratch_bytes)
{
    if (!norm) return FP4Q_ERR_NULL;
    if (!aligned(norm, 4)) return FP4Q_ERR_ALIGN;
    if (!scratch || scratch_bytes < fp4q_global_norm_scratch_bytes(tensors, n)) return FP4Q_ERR_WORKSPACE;
    return aligned(scratch, 256) ? FP4Q_OK : FP4Q_ERR_ALIGN;
}
fp4q_status check_clip(const fp4q_span *tensors, const fp4q_span *outs, int32_t n, float max_norm, float eps)
{
    if (fp4q_status s = check_spans(tensors, n)) return s;
    if (outs) {
        if (fp4q_status s = check_spans(outs, n)) return s;
        for (int32_t i = 0; i < n; i++)
            if (outs[i].rows != tensors[i].rows || outs[i].cols != tensors[i].cols) return FP4Q_ERR_SHAPE;
    }
    return max_norm >= 0.f && eps >= 0.f ? FP4Q_OK : FP4Q_ERR_UNSUPPORTED;
}

}  // namespace

extern "C" size_t fp4q_global_norm_scratch_bytes(const fp4q_span *tensors, int32_t n_tensors)
{
    if (n_tensors <= 0 || !tensors) return 256;
    return (size_t)round_up(ceil_div(n_tensors, kMany) * kNormCtas * 8, 256);
}

extern "C" fp4q_status fp4q_global_norm(const fp4q_span *tensors, int32_t n_tensors, float *norm, void *scratch, size_t scratch_bytes, void *stream)
{
    if (fp4q_status s = check_spans(tensors, n_tensors)) return s;
    if (fp4q_status s = check_norm(norm, tensors, n_tensors, scratch, scratch_bytes)) return s;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    double *partial = static_cast<double *>(scratch);
    int64_t parts;
    if (fp4q_status st = launch_sums(tensors, n_tensors, partial, parts, s)) return st;
    const RootParams r = {partial, parts, norm};
    return launched(launch_dependent(root_kernel, dim3(1), 256, s, r));
}

extern "C" fp4q_status fp4q_clip_by_norm(const fp4q_span *tensors, const fp4q_span *outs, int32_t n_tensors, const float *norm, float max_norm, float eps, void *stream)
{
    if (fp4q_status s = check_clip(tensors, outs, n_tensors, max_norm, eps)) return s;
    if (!norm) return FP4Q_ERR_NULL;
    if (!aligned(norm, 4)) return FP4Q_ERR_ALIGN;
    return launch_scaling(tensors, outs, n_tensors, const_cast<float *>(norm), nullptr, 0, max_norm, eps, static_cast<cudaStream_t>(stream));   // which only reads it
}

extern "C" fp4q_status fp4q_clip_grad_norm(const fp4q_span *tensors, const fp4q_span *outs, int32_t n_tensors, float max_norm, float eps, float *norm, void *scratch, size_t scratch_bytes,
                                           void *stream)
{
    if (fp4q_status s = check_clip(tensors, outs, n_tensors, max_norm, eps)) return s;
    if (fp4q_status s = check_norm(norm, tensors, n_tensors, scratch, scratch_bytes)) return s;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    double *partial = static_cast<double *>(scratch);
    int64_t parts;
    if (fp4q_status st = launch_sums(tensors, n_tensors, partial, parts, s)) return st;
    if (parts == 0) {   // no elements
        const RootParams r = {partial, 0, norm};
        return launched(launch_dependent(root_kernel, dim3(1), 256, s, r));
    }
    return launch_scaling(tensors, outs, n_tensors, norm, partial, parts, max_norm, eps, s);
}
