// Norm of all gradients of a step, and clipping by it (mxfp8_grad_sumsq, mxfp8_grad_scale, mxfp8_grad_clip).
//
//   S = sum g^2;  norm = sqrt(S);  factor = min(1, max_norm / (norm + 1e-6));  dst = factor * src
//
// Bound by memory: every gradient is read once for S, then read and written once (218 M FP32 elements 433 us, 93 % of the measured copy
// rate; where nothing is clipped in place the second pass writes nothing: 1.3 G elements of both types 434 us).  The items go to the kernels by value, as
// a table in the launch's parameters (nothing to copy or to keep alive, and a captured launch holds its own).  Items are cut into
// pieces of a few thousand elements, counted from the 16-byte boundary at or before the item's first element, so that all
// vectors of a piece are aligned whatever the item's alignment.
#include <cuda_bf16.h>

#include "mxfp8_device.cuh"
#include "mxfp8_host.h"

namespace mxfp8 {
namespace {

constexpr int GRAD_THREADS = 256, GRAD_WARPS = GRAD_THREADS / 32;
constexpr int GRAD_CTAS = 4 * 148;              // at most, of one launch: one partial sum each
constexpr int UNROLL = 4;                       // vectors of 16 bytes in flight per thread; four CTAs per multiprocessor
constexpr int MANY_ITEMS = 1024, FEW_ITEMS = 96;

template <int N>
struct GradTable {
    const void* src[N];
    void* dst[N];
    int64_t numel[N];
    uint32_t first[N + 1];       // first piece of every item; [count] is the number of pieces
    uint8_t bf16[N];
    int count;
    int piece_log;               // elements of a piece
    bool in_place;               // all items
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
    p.base = ((int64_t)(piece - t.first[lo]) << t.piece_log) - before;
    p.first = p.base < 0 ? 0 : p.base;
    p.last = min(p.base + (1 << t.piece_log), t.numel[lo]);
    return p;
}

__device__ __forceinline__ float bf16_low(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_high(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// Sum of the squares of eight values.  In FP32 where the largest lies between 2^-40 and 2^60 (eight squares stay in range, and what
// falls below FP32's is less than 2^-46 of the sum), in FP64 elsewhere.
__device__ __forceinline__ double squares(const float (&v)[8])
{
    float peak = 0.f, s = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        peak = fmaxf(peak, fabsf(v[i]));
        s = fmaf(v[i], v[i], s);
    }
    if (peak < 0x1p60f && peak > 0x1p-40f) return (double)s;
    double d = 0.0;
#pragma unroll
    for (int i = 0; i < 8; ++i) d = fma((double)v[i], (double)v[i], d);
    return d;
}

// The elements of a 16-byte vector: eight of BF16, four of FP32
template <typename T> constexpr int PER = 16 / sizeof(T);
template <typename T>
__device__ __forceinline__ void unpack(const uint4& w, float* v)
{
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if (sizeof(T) == 2) { v[2 * k] = bf16_low(u[k]); v[2 * k + 1] = bf16_high(u[k]); }
        else v[k] = __uint_as_float(u[k]);
    }
}
__device__ __forceinline__ float element(const float* p) { return *p; }
__device__ __forceinline__ float element(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

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

// The whole vectors of a piece, begin .. end - 1 in elements; a few elements at the item's first and last vector lie outside.
template <typename T>
__device__ __forceinline__ void whole_vectors(const Piece& p, int64_t& begin, int64_t& end)
{
    begin = p.base < p.first ? p.base + PER<T> : p.base;
    end = max(begin, p.base + (p.last - p.base) / PER<T> * PER<T>);
}
// Calls f for those elements, a thread for each.
template <typename T, typename F>
__device__ __forceinline__ void other_elements(const Piece& p, int64_t begin, int64_t end, F f)
{
    const int64_t head = p.first + threadIdx.x, tail = end + threadIdx.x - PER<T>;
    if (threadIdx.x < PER<T> && head < min(begin, p.last)) f(head);
    if (threadIdx.x >= PER<T> && threadIdx.x < 2 * PER<T> && tail < p.last) f(tail);
}

template <typename T>
__device__ __forceinline__ double piece_squares(const T* src, const Piece& p)
{
    constexpr int V = PER<T>, STEP = GRAD_THREADS * V;
    int64_t begin, end;
    whole_vectors<T>(p, begin, end);
    double sum = 0.0;
    for (int64_t i = begin + threadIdx.x * V; i < end; i += UNROLL * STEP) {
        uint4 w[UNROLL];
#pragma unroll
        for (int k = 0; k < UNROLL; ++k) w[k] = i + k * STEP < end ? *reinterpret_cast<const uint4*>(src + i + k * STEP) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
        for (int k = 0; k < UNROLL; k += 8 / V) {
            float v[8];
            unpack<T>(w[k], v);
            if constexpr (V == 4) unpack<T>(w[k + 1], v + 4);
            sum += squares(v);
        }
    }
    other_elements<T>(p, begin, end, [&](int64_t at) {
        const double d = element(src + at);
        sum = fma(d, d, sum);
    });
    return sum;
}

template <int N>
__global__ void __launch_bounds__(GRAD_THREADS, 4) grad_squares_kernel(const __grid_constant__ GradTable<N> t, double* partial)
{
    __shared__ double area[GRAD_WARPS];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    double sum = 0.0;
    for (uint32_t piece = blockIdx.x; piece < t.first[t.count]; piece += gridDim.x) {
        const Piece p = find_piece(t, piece);
        sum += t.bf16[p.item] ? piece_squares(static_cast<const __nv_bfloat16*>(t.src[p.item]), p) : piece_squares(static_cast<const float*>(t.src[p.item]), p);
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
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const double s = sum_of(partial, count, area);
    if (threadIdx.x == 0) *sumsq = s;
}

template <typename T>
__device__ __forceinline__ void piece_scale(const T* src, T* dst, const Piece& p, float factor)
{
    constexpr int V = PER<T>, STEP = GRAD_THREADS * V;
    // vectors of both need the same place within 16 bytes
    const bool together = ((reinterpret_cast<uintptr_t>(src) ^ reinterpret_cast<uintptr_t>(dst)) & 15u) == 0;
    auto scaled = [&](uint4 w) {
        float v[V];
        unpack<T>(w, v);
        uint32_t u[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if constexpr (V == 8) {
                const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * k] * factor, v[2 * k + 1] * factor);
                u[k] = *reinterpret_cast<const uint32_t*>(&b);
            } else u[k] = __float_as_uint(v[k] * factor);
        }
        return make_uint4(u[0], u[1], u[2], u[3]);
    };
    if (!together) {
        for (int64_t i = p.first + threadIdx.x; i < p.last; i += GRAD_THREADS) put(dst + i, element(src + i) * factor);
        return;
    }
    int64_t begin, end;
    whole_vectors<T>(p, begin, end);
    for (int64_t i = begin + threadIdx.x * V; i < end; i += UNROLL * STEP) {
        uint4 w[UNROLL];
#pragma unroll
        for (int k = 0; k < UNROLL; ++k)
            if (i + k * STEP < end) w[k] = __ldcs(reinterpret_cast<const uint4*>(src + i + k * STEP));
#pragma unroll
        for (int k = 0; k < UNROLL; ++k)
            if (i + k * STEP < end) __stcs(reinterpret_cast<uint4*>(dst + i + k * STEP), scaled(w[k]));
    }
    other_elements<T>(p, begin, end, [&](int64_t at) { put(dst + at, element(src + at) * factor); });
}

// Pieces in the opposite order to the sums': what those read last is in L2 (126 MB) and is read again first, and leaves it at once.
template <int N>
__global__ void __launch_bounds__(GRAD_THREADS, 4) grad_scale_kernel(const __grid_constant__ GradTable<N> t, const double* partial, int count, float max_norm,
                                                                     float* result)
{
    __shared__ double area[GRAD_WARPS];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const float norm = (float)sqrt(sum_of(partial, count, area));
    float factor = fminf(1.0f, max_norm / (norm + 1e-6f));
    if (!(norm <= 3.402823466e38f)) factor = 1.0f;               // infinite or not a number
    if (result && blockIdx.x == 0 && threadIdx.x == 0) {
        result[0] = norm;
        result[1] = factor;
    }
    if (factor == 1.0f && t.in_place) return;
    const uint32_t pieces = t.first[t.count];
    for (uint32_t i = blockIdx.x; i < pieces; i += gridDim.x) {
        const Piece p = find_piece(t, pieces - 1 - i);
        if (factor == 1.0f && t.src[p.item] == t.dst[p.item]) continue;
        if (t.bf16[p.item]) piece_scale(static_cast<const __nv_bfloat16*>(t.src[p.item]), static_cast<__nv_bfloat16*>(t.dst[p.item]), p, factor);
        else piece_scale(static_cast<const float*>(t.src[p.item]), static_cast<float*>(t.dst[p.item]), p, factor);
    }
}

// Calls f(table, CTAs) for the items, as many at a time as a table holds.  Returns the first error.
template <typename F>
cudaError_t by_tables(const mxfp8_grad_item* items, int count, F f)
{
    auto fill = [](auto& t, const mxfp8_grad_item* from, int n) {
        int64_t elements = 0;
        for (int i = 0; i < n; ++i) elements += from[i].numel;
        // a piece is a round of all threads' BF16 vectors (UNROLL each), or two of them while that leaves every CTA eight pieces
        t.piece_log = (elements >> 14) >= 8 * GRAD_CTAS ? 14 : 13;
        t.count = 0;
        t.in_place = true;
        uint32_t pieces = 0;
        for (int i = 0; i < n; ++i) {
            if (from[i].numel == 0) continue;
            const int bytes = from[i].dtype == MXFP8_BF16 ? 2 : 4, k = t.count++;
            t.src[k] = from[i].src; t.dst[k] = from[i].dst; t.numel[k] = from[i].numel; t.bf16[k] = bytes == 2;
            t.in_place = t.in_place && from[i].src == from[i].dst;
            t.first[k] = pieces;
            pieces += (uint32_t)((from[i].numel + (int64_t)(reinterpret_cast<uintptr_t>(from[i].src) & 15u) / bytes + (1 << t.piece_log) - 1) >> t.piece_log);
        }
        t.first[t.count] = pieces;
        const uint32_t rounds = pieces / GRAD_CTAS + (pieces % GRAD_CTAS != 0);             // as few CTAs as take no more rounds
        return rounds ? (pieces + rounds - 1) / rounds : 1u;
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

// A launch that may begin before the one ahead of it has ended; its kernel waits for that one itself.
template <typename Kernel, typename... Args>
cudaError_t launch_early(Kernel kernel, unsigned ctas, cudaStream_t st, const Args&... args)
{
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(ctas);
    cfg.blockDim = dim3(GRAD_THREADS);
    cfg.stream = st;
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    const cudaError_t rc = cudaLaunchKernelEx(&cfg, kernel, args...);
    if (rc == cudaSuccess) count_launch(1);
    return rc;
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
        const cudaError_t rc = launch_early(grad_scale_kernel<N>, ctas, st, t, partial, parts, max_norm, norm);
        norm = nullptr;                                     // the first launch writes it
        return rc;
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
    return launch_early(grad_sum_kernel, 1, st, static_cast<const double*>(ws), parts, sumsq) == cudaSuccess ? MXFP8_OK : MXFP8_ERR_CUDA;
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
