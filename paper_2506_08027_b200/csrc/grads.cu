// Norm of all gradients of a step, and clipping by it (mxfp8_grad_sumsq, mxfp8_grad_scale, mxfp8_grad_clip).
//
//   S = sum g^2;  norm = sqrt(S);  factor = min(1, max_norm / (norm + 1e-6));  dst = factor * src
//
// Bound by memory: every gradient is read once for S, then read and written once.  The items go to the kernels by value, as
// a table in the launch's parameters (nothing to copy or to keep alive, and a captured launch holds its own).  Items are cut into
// pieces of PIECE elements, counted from the 16-byte boundary at or before the item's first element, so that all
// vectors of a piece are aligned whatever the item's alignment.
#include <cuda_bf16.h>

#include "mxfp8_device.cuh"
#include "mxfp8_host.h"

namespace mxfp8 {
namespace {

constexpr int GRAD_THREADS = 256, GRAD_WARPS = GRAD_THREADS / 32;
constexpr int PIECE = 16384;                    // elements
constexpr int GRAD_CTAS = 4 * 148;              // at most, of one launch: one partial sum each
constexpr int MANY_ITEMS = 1024, FEW_ITEMS = 96;

template <int N>
struct GradTable {
    const void* src[N];
    void* dst[N];
    int64_t numel[N];
    uint32_t first[N + 1];       // first piece of every item; [count] is the number of pieces
    uint8_t bf16[N];
    int count;
};

// Where a piece lies: its item and the elements first .. last - 1 of it; vectors start at `base`, which is first or, at the item's
// begin, up to seven (three) elements before it.
struct Piece {
    int item;
    int64_t base, first, last;
};
template <int N>
__device__ __forceinline__ Piece find_piece(const GradTable<N>& t, uint32_t piece)
{
    int lo = 0, hi = t.count;                    // the last item whose first piece is not behind this one
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (t.first[mid] <= piece) lo = mid;
        else hi = mid;
    }
    const int bytes = t.bf16[lo] ? 2 : 4;
    const int64_t before = (int64_t)(reinterpret_cast<uintptr_t>(t.src[lo]) & 15u) / bytes;
    Piece p;
    p.item = lo;
    p.base = (int64_t)(piece - t.first[lo]) * PIECE - before;
    p.first = p.base < 0 ? 0 : p.base;
    p.last = min(p.base + PIECE, t.numel[lo]);
    return p;
}

__device__ __forceinline__ float bf16_low(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_high(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// Sum of the squares of V values.  In FP32 where the largest lies between 2^-40 and 2^60 (eight squares stay in range, and what
// falls below FP32's is less than 2^-46 of the sum), in FP64 elsewhere.
template <int V>
__device__ __forceinline__ double squares(const float (&v)[V])
{
    float peak = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) peak = fmaxf(peak, fabsf(v[i]));
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) s = fmaf(v[i], v[i], s);
    if (peak < 0x1p60f && peak > 0x1p-40f) return (double)s;
    double d = 0.0;
#pragma unroll
    for (int i = 0; i < V; ++i) d = fma((double)v[i], (double)v[i], d);
    return d;
}

__device__ __forceinline__ double cta_sum(double v, double* area)
{
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, off);
    if ((threadIdx.x & 31) == 0) area[threadIdx.x >> 5] = v;
    __syncthreads();
    v = 0.0;
    for (int w = 0; w < GRAD_WARPS; ++w) v += area[w];
    return v;
}

template <int N>
__global__ void __launch_bounds__(GRAD_THREADS) grad_squares_kernel(const __grid_constant__ GradTable<N> t, double* partial)
{
    __shared__ double area[GRAD_WARPS];
    double sum = 0.0;
    for (uint32_t piece = blockIdx.x; piece < t.first[t.count]; piece += gridDim.x) {
        const Piece p = find_piece(t, piece);
        if (t.bf16[p.item]) {
            const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(t.src[p.item]);
            for (int64_t i = p.base + threadIdx.x * 8; i < p.last; i += GRAD_THREADS * 8) {
                float v[8];
                if (i >= p.first && i + 8 <= p.last) {
                    const uint4 w = *reinterpret_cast<const uint4*>(src + i);
                    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                    for (int k = 0; k < 4; ++k) { v[2 * k] = bf16_low(u[k]); v[2 * k + 1] = bf16_high(u[k]); }
                } else {
#pragma unroll
                    for (int k = 0; k < 8; ++k) v[k] = (i + k >= p.first && i + k < p.last) ? __bfloat162float(src[i + k]) : 0.f;
                }
                sum += squares(v);
            }
        } else {
            const float* src = static_cast<const float*>(t.src[p.item]);
            for (int64_t i = p.base + threadIdx.x * 4; i < p.last; i += GRAD_THREADS * 4) {
                float v[4];
                if (i >= p.first && i + 4 <= p.last) {
                    const float4 w = *reinterpret_cast<const float4*>(src + i);
                    v[0] = w.x; v[1] = w.y; v[2] = w.z; v[3] = w.w;
                } else {
#pragma unroll
                    for (int k = 0; k < 4; ++k) v[k] = (i + k >= p.first && i + k < p.last) ? src[i + k] : 0.f;
                }
                sum += squares(v);
            }
        }
    }
    sum = cta_sum(sum, area);
    if (threadIdx.x == 0) partial[blockIdx.x] = sum;
}

// Sum of `count` FP64 values by one CTA, in a fixed order.
__device__ __forceinline__ double sum_of(const double* partial, int count, double* area)
{
    double s = 0.0;
    for (int i = threadIdx.x; i < count; i += GRAD_THREADS) s += partial[i];
    return cta_sum(s, area);
}

__global__ void __launch_bounds__(GRAD_THREADS) grad_sum_kernel(const double* partial, int count, double* sumsq)
{
    __shared__ double area[GRAD_WARPS];
    const double s = sum_of(partial, count, area);
    if (threadIdx.x == 0) *sumsq = s;
}

template <int N>
__global__ void __launch_bounds__(GRAD_THREADS) grad_scale_kernel(const __grid_constant__ GradTable<N> t, const double* partial, int count, float max_norm,
                                                                  float* result)
{
    __shared__ double area[GRAD_WARPS];
    const float norm = (float)sqrt(sum_of(partial, count, area));
    float factor = fminf(1.0f, max_norm / (norm + 1e-6f));
    if (!(norm <= 3.402823466e38f)) factor = 1.0f;               // infinite or not a number
    if (result && blockIdx.x == 0 && threadIdx.x == 0) {
        result[0] = norm;
        result[1] = factor;
    }
    for (uint32_t piece = blockIdx.x; piece < t.first[t.count]; piece += gridDim.x) {
        const Piece p = find_piece(t, piece);
        if (factor == 1.0f && t.src[p.item] == t.dst[p.item]) continue;
        const bool together = ((reinterpret_cast<uintptr_t>(t.src[p.item]) ^ reinterpret_cast<uintptr_t>(t.dst[p.item])) & 15u) == 0;
        if (t.bf16[p.item]) {
            const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(t.src[p.item]);
            __nv_bfloat16* dst = static_cast<__nv_bfloat16*>(t.dst[p.item]);
            for (int64_t i = p.base + threadIdx.x * 8; i < p.last; i += GRAD_THREADS * 8) {
                if (together && i >= p.first && i + 8 <= p.last) {
                    uint4 w = *reinterpret_cast<const uint4*>(src + i);
                    uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const __nv_bfloat162 v = __floats2bfloat162_rn(bf16_low(u[k]) * factor, bf16_high(u[k]) * factor);
                        u[k] = *reinterpret_cast<const uint32_t*>(&v);
                    }
                    *reinterpret_cast<uint4*>(dst + i) = make_uint4(u[0], u[1], u[2], u[3]);
                } else {
                    for (int k = 0; k < 8; ++k)
                        if (i + k >= p.first && i + k < p.last) dst[i + k] = __float2bfloat16_rn(__bfloat162float(src[i + k]) * factor);
                }
            }
        } else {
            const float* src = static_cast<const float*>(t.src[p.item]);
            float* dst = static_cast<float*>(t.dst[p.item]);
            for (int64_t i = p.base + threadIdx.x * 4; i < p.last; i += GRAD_THREADS * 4) {
                if (together && i >= p.first && i + 4 <= p.last) {
                    float4 w = *reinterpret_cast<const float4*>(src + i);
                    w.x *= factor; w.y *= factor; w.z *= factor; w.w *= factor;
                    *reinterpret_cast<float4*>(dst + i) = w;
                } else {
                    for (int k = 0; k < 4; ++k)
                        if (i + k >= p.first && i + k < p.last) dst[i + k] = src[i + k] * factor;
                }
            }
        }
    }
}

// Calls f(table, CTAs) for the items, as many at a time as a table holds.  Returns the first error.
template <typename F>
cudaError_t by_tables(const mxfp8_grad_item* items, int count, F f)
{
    auto fill = [](auto& t, const mxfp8_grad_item* from, int n) {
        t.count = 0;
        uint32_t pieces = 0;
        for (int i = 0; i < n; ++i) {
            if (from[i].numel == 0) continue;
            const int bytes = from[i].dtype == MXFP8_BF16 ? 2 : 4, k = t.count++;
            t.src[k] = from[i].src; t.dst[k] = from[i].dst; t.numel[k] = from[i].numel; t.bf16[k] = bytes == 2;
            t.first[k] = pieces;
            pieces += (uint32_t)((from[i].numel + (int64_t)(reinterpret_cast<uintptr_t>(from[i].src) & 15u) / bytes + PIECE - 1) / PIECE);
        }
        t.first[t.count] = pieces;
        return pieces < (uint32_t)GRAD_CTAS ? (pieces ? pieces : 1u) : (uint32_t)GRAD_CTAS;
    };
    if (count <= FEW_ITEMS) {
        GradTable<FEW_ITEMS> t;
        const unsigned ctas = fill(t, items, count);
        return f(t, ctas);
    }
    for (int at = 0; at < count; at += MANY_ITEMS) {
        GradTable<MANY_ITEMS> t;
        const unsigned ctas = fill(t, items + at, count - at < MANY_ITEMS ? count - at : MANY_ITEMS);
        const cudaError_t err = f(t, ctas);
        if (err != cudaSuccess) return err;
    }
    return cudaSuccess;
}

int tables_of(int count) { return count <= FEW_ITEMS ? 1 : (count + MANY_ITEMS - 1) / MANY_ITEMS; }

int items_check(const mxfp8_grad_item* items, int count, bool scaled)
{
    if (count < 0) return MXFP8_ERR_SHAPE;
    if (count > 0 && !items) return MXFP8_ERR_NULL;
    for (int i = 0; i < count; ++i) {
        if (items[i].dtype != MXFP8_FP32 && items[i].dtype != MXFP8_BF16) return MXFP8_ERR_ENUM;
        if (items[i].numel < 0) return MXFP8_ERR_SHAPE;
        if (items[i].numel == 0) continue;
        if (!items[i].src || (scaled && !items[i].dst)) return MXFP8_ERR_NULL;
        const uintptr_t mask = items[i].dtype == MXFP8_BF16 ? 1u : 3u;
        if ((reinterpret_cast<uintptr_t>(items[i].src) & mask) || (scaled && (reinterpret_cast<uintptr_t>(items[i].dst) & mask))) return MXFP8_ERR_ALIGN;
        if (items[i].numel > (1LL << 34)) return MXFP8_ERR_UNSUPPORTED;      // pieces of a table are counted in 32 bits
    }
    return MXFP8_OK;
}

// Partial sums of all items, GRAD_CTAS to a table at most; returns their number through `parts`.
cudaError_t launch_squares(const mxfp8_grad_item* items, int count, double* ws, int& parts, cudaStream_t st)
{
    parts = 0;
    return by_tables(items, count, [&](auto& t, unsigned ctas) {
        constexpr int N = sizeof(t.bf16);
        grad_squares_kernel<N><<<ctas, GRAD_THREADS, 0, st>>>(t, ws + parts);
        parts += (int)ctas;
        count_launch(1);
        return cudaGetLastError();
    });
}

cudaError_t launch_scale(const mxfp8_grad_item* items, int count, const double* partial, int parts, float max_norm, float* norm, cudaStream_t st)
{
    return by_tables(items, count, [&](auto& t, unsigned ctas) {
        constexpr int N = sizeof(t.bf16);
        grad_scale_kernel<N><<<ctas, GRAD_THREADS, 0, st>>>(t, partial, parts, max_norm, norm);
        norm = nullptr;                                     // the first launch writes it
        count_launch(1);
        return cudaGetLastError();
    });
}

int workspace_check(const mxfp8_grad_item* items, int count, const void* ws, size_t ws_bytes)
{
    if (!ws || ws_bytes < mxfp8_grad_ws_bytes(items, count)) return MXFP8_ERR_WORKSPACE;
    return (reinterpret_cast<uintptr_t>(ws) & 7u) ? MXFP8_ERR_ALIGN : MXFP8_OK;
}

}  // namespace
}  // namespace mxfp8

using namespace mxfp8;

extern "C" size_t mxfp8_grad_ws_bytes(const mxfp8_grad_item* items, int count)
{
    (void)items;
    return count < 0 ? 0 : (size_t)tables_of(count) * GRAD_CTAS * sizeof(double);
}

extern "C" int mxfp8_grad_sumsq(const mxfp8_grad_item* items, int count, double* sumsq, void* ws, size_t ws_bytes, void* stream)
{
    int rc = items_check(items, count, false);
    if (rc != MXFP8_OK) return rc;
    if (!sumsq) return MXFP8_ERR_NULL;
    if (reinterpret_cast<uintptr_t>(sumsq) & 7u) return MXFP8_ERR_ALIGN;
    if ((rc = workspace_check(items, count, ws, ws_bytes)) != MXFP8_OK) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    int parts = 0;
    if (launch_squares(items, count, static_cast<double*>(ws), parts, st) != cudaSuccess) return MXFP8_ERR_CUDA;
    grad_sum_kernel<<<1, GRAD_THREADS, 0, st>>>(static_cast<const double*>(ws), parts, sumsq);
    count_launch(1);
    return cudaGetLastError() == cudaSuccess ? MXFP8_OK : MXFP8_ERR_CUDA;
}

extern "C" int mxfp8_grad_scale(const mxfp8_grad_item* items, int count, const double* sumsq, float max_norm, float* norm, void* stream)
{
    const int rc = items_check(items, count, true);
    if (rc != MXFP8_OK) return rc;
    if (!sumsq || !norm) return MXFP8_ERR_NULL;
    if (!(max_norm >= 0.f)) return MXFP8_ERR_SHAPE;
    if ((reinterpret_cast<uintptr_t>(sumsq) & 7u) || (reinterpret_cast<uintptr_t>(norm) & 3u)) return MXFP8_ERR_ALIGN;
    return launch_scale(items, count, sumsq, 1, max_norm, norm, static_cast<cudaStream_t>(stream)) == cudaSuccess ? MXFP8_OK : MXFP8_ERR_CUDA;
}

extern "C" int mxfp8_grad_clip(const mxfp8_grad_item* items, int count, float max_norm, float* norm, void* ws, size_t ws_bytes, void* stream)
{
    int rc = items_check(items, count, true);
    if (rc != MXFP8_OK) return rc;
    if (!norm) return MXFP8_ERR_NULL;
    if (!(max_norm >= 0.f)) return MXFP8_ERR_SHAPE;
    if (reinterpret_cast<uintptr_t>(norm) & 3u) return MXFP8_ERR_ALIGN;
    if ((rc = workspace_check(items, count, ws, ws_bytes)) != MXFP8_OK) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    int parts = 0;
    if (launch_squares(items, count, static_cast<double*>(ws), parts, st) != cudaSuccess) return MXFP8_ERR_CUDA;
    return launch_scale(items, count, static_cast<const double*>(ws), parts, max_norm, norm, st) == cudaSuccess ? MXFP8_OK : MXFP8_ERR_CUDA;
}
