// The seam between two blocks of a residual stream, forward and backward (mxfp8_residual_rmsnorm and relatives).
//
//   rstd_post = 1 / sqrt(mean y^2 + eps);  n = (y rstd_post) gamma_post;  h = residual_scale h_in + (branch_scale gate) n
//   rstd_pre  = 1 / sqrt(mean h^2 + eps);  x = (h rstd_pre) gamma_pre
//
// Bound by memory: forward y, h_in -> h, x; backward dx, dh, y, h -> dy, dh_in, each element once.  8192 x 4096 in BF16: forward
// 49.5 us, backward 76 to 81 us, 83 and 76 to 81 % of the measured copy rate.  Further from it: FP32 streams (forward 91 us, 68 %; backward 142 us,
// 65 %), backward rows above 4096 columns (65 % in BF16, 44 % in FP32) and rows off 16-byte boundaries (8192 x 4095 BF16: 147 and 463 us).
#include <cuda_bf16.h>

#include <initializer_list>
#include <type_traits>

#include "mxfp8_device.cuh"
#include "mxfp8_host.h"

namespace mxfp8 {
namespace {

constexpr int SEAM_MAX_COLS = 16384;
constexpr int SEAM_THREADS = 256;                // of the kernels for any alignment
constexpr int SEAM_MAX_WARPS = 32;

struct SeamArgs {
    int64_t rows;
    int cols;
    const void *gamma_post, *gate, *gamma_pre;
    bool bf16_params;
    int64_t rows_per_gate;
    float branch_scale, residual_scale, eps;
    const void *y, *h_in;                        // forward inputs; the backward pass reads y and h
    void *h, *x;
    float *rstd_post, *rstd_pre;
    const void *dx, *dh;                         // backward
    void *dy, *dh_in;
    float *d_gamma_pre, *d_gamma_post, *d_gate;
    float* ws;
    int64_t chunk;                               // rows of a CTA
    int64_t gates;
    uint32_t gate_magic;                         // of rows_per_gate, where rows fit 31 bits
    uint8_t *q_row, *s_row;                      // forward: x converted with row blocks instead of stored
    int elem, rule, layout;
};

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

__device__ __forceinline__ float param(const void* p, int64_t at, bool bf16)
{
    return bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(p)[at]) : static_cast<const float*>(p)[at];
}

__device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, off);
    return v;
}

// Sums over the CTA, the same in every thread and in a fixed order.  `turn` alternates between two areas, so that one barrier per call is
// enough.  Every warp adds the warps' sums the same way.
__device__ __forceinline__ float cta_sum(float v, float (*area)[SEAM_MAX_WARPS], int& turn)
{
    v = warp_sum(v);
    float* here = area[turn];
    turn ^= 1;
    if ((threadIdx.x & 31) == 0) here[threadIdx.x >> 5] = v;
    __syncthreads();
    const int warps = blockDim.x >> 5;
    if (warps <= 4) {
        v = here[0];
        for (int w = 1; w < warps; ++w) v += here[w];
        return v;
    }
    v = (threadIdx.x & 31) < warps ? here[threadIdx.x & 31] : 0.f;
    if (warps > 8) {
        v += __shfl_xor_sync(0xFFFFFFFFu, v, 16);
        v += __shfl_xor_sync(0xFFFFFFFFu, v, 8);
    }
#pragma unroll
    for (int off = 4; off > 0; off >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, off);
    return __shfl_sync(0xFFFFFFFFu, v, 0);
}

// Three sums at once.  The first two steps of the tree hand half of the values to the other half of the lanes, so that a warp needs six
// shuffles instead of fifteen; lanes 0, 8 and 16 end with the sums.
__device__ __forceinline__ float three_sums(float v0, float v1, float v2)
{
    const int lane = threadIdx.x & 31;
    const bool high = lane & 16, odd = lane & 8;
    float a = high ? v2 : v0, b = high ? 0.f : v1;
    a += __shfl_xor_sync(0xFFFFFFFFu, high ? v0 : v2, 16);
    b += __shfl_xor_sync(0xFFFFFFFFu, high ? v1 : 0.f, 16);
    float s = odd ? b : a;
    s += __shfl_xor_sync(0xFFFFFFFFu, odd ? a : b, 8);
#pragma unroll
    for (int off = 4; off > 0; off >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, off);
    return s;
}
__device__ __forceinline__ void cta_sums(float (&v)[3], float4 (*area)[SEAM_MAX_WARPS], int& turn)
{
    const int lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    float s = three_sums(v[0], v[1], v[2]);
    float4* here = area[turn];
    turn ^= 1;
    if ((lane & 7) == 0) reinterpret_cast<float*>(here + (threadIdx.x >> 5))[lane >> 3] = s;          // sums 0, 1, 2 and nothing
    __syncthreads();
    if (warps > 8) {
        const float4 one = lane < warps ? here[lane] : make_float4(0.f, 0.f, 0.f, 0.f);
        s = three_sums(one.x, one.y, one.z);
        v[0] = __shfl_sync(0xFFFFFFFFu, s, 0);
        v[1] = __shfl_sync(0xFFFFFFFFu, s, 8);
        v[2] = __shfl_sync(0xFFFFFFFFu, s, 16);
        return;
    }
    float4 all = here[0];
#pragma unroll 4
    for (int w = 1; w < warps; ++w) {
        const float4 more = here[w];
        all.x += more.x; all.y += more.y; all.z += more.z;
    }
    v[0] = all.x; v[1] = all.y; v[2] = all.z;
}

// 1 / sqrt(mean + eps), within two units of the last place
__device__ __forceinline__ float rstd_of(float sum, float cols, float eps) { return rsqrtf(sum / cols + eps); }

// The row of the gate for row r
__device__ __forceinline__ int64_t gate_row(const SeamArgs& a, int64_t r)
{
    if (a.rows > 0x7FFFFFFFLL) return r / a.rows_per_gate;
    int g, rest;
    divmod((uint32_t)r, (uint32_t)a.rows_per_gate, a.gate_magic, g, rest);
    return g;
}

// What a kernel may know of a seam when it is compiled: nothing (0), or that all tensors and both norms are there, the parameters have
// the stream's type and there is no gate (1) or one whose gradient is wanted (2).
template <int MODE, typename H>
struct Known {
    const SeamArgs& a;
    __device__ __forceinline__ bool post() const { return MODE != 0 || a.gamma_post != nullptr; }
    __device__ __forceinline__ bool gate() const { return MODE == 2 || (MODE == 0 && a.gate != nullptr); }
    __device__ __forceinline__ bool d_gate() const { return MODE == 2 || (MODE == 0 && a.d_gate != nullptr); }
    __device__ __forceinline__ bool dx() const { return MODE != 0 || a.dx != nullptr; }
    __device__ __forceinline__ bool dh() const { return MODE != 0 || a.dh != nullptr; }
    __device__ __forceinline__ bool dy() const { return MODE != 0 || a.dy != nullptr; }
    __device__ __forceinline__ bool dh_in() const { return MODE != 0 || a.dh_in != nullptr; }
    __device__ __forceinline__ bool bf16() const { return MODE != 0 ? sizeof(H) == 2 : a.bf16_params; }
};

// ---------------------------------------------------------------------------------------------------------------------
// Any width and alignment: a CTA per row, NE elements of it in every thread's registers, V neighbours at a time (two where rows have an even
// number of elements).  All loads of a row are asked for at once; other CTAs cover their latency.
template <typename T, int V>
__device__ __forceinline__ void load_few(const T* p, float (&v)[V])
{
    if constexpr (V == 1) v[0] = to_float(*p);
    else if constexpr (sizeof(T) == 2) {
        const uint32_t w = *reinterpret_cast<const uint32_t*>(p);
        v[0] = __uint_as_float(w << 16);
        v[1] = __uint_as_float(w & 0xFFFF0000u);
    } else {
        const float2 w = *reinterpret_cast<const float2*>(p);
        v[0] = w.x; v[1] = w.y;
    }
}
// Rounds to T; v becomes the rounded values
template <typename T, int V>
__device__ __forceinline__ void store_few(T* p, float (&v)[V])
{
    if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int k = 0; k < V; ++k) v[k] = __bfloat162float(__float2bfloat16_rn(v[k]));
    }
    if constexpr (V == 1) *p = from_float<T>(v[0]);
    else if constexpr (sizeof(T) == 2) *reinterpret_cast<uint32_t*>(p) = __float_as_uint(v[0]) >> 16 | (__float_as_uint(v[1]) & 0xFFFF0000u);
    else *reinterpret_cast<float2*>(p) = make_float2(v[0], v[1]);
}
template <int V>
__device__ __forceinline__ void params_few(const void* p, int64_t at, bool bf16, float (&v)[V])
{
    if (bf16) load_few<__nv_bfloat16, V>(static_cast<const __nv_bfloat16*>(p) + at, v);
    else load_few<float, V>(static_cast<const float*>(p) + at, v);
}

// T threads; SAME: the parameters have the stream's type.
template <typename Y, typename H, int V, int NE, int T, bool SAME>
__global__ void __launch_bounds__(T, NE == 16 ? 1024 / T : (T == 32 ? 24 : 1536 / T)) seam_forward_any_kernel(const SeamArgs a)
{
    __shared__ float area[2][SEAM_MAX_WARPS];
    constexpr int NV = NE / V;
    int turn = 0;
    const int t = threadIdx.x;
    const bool bf16 = SAME ? sizeof(H) == 2 : a.bf16_params;
    const float n_cols = (float)a.cols;
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const int64_t row = r * a.cols, gate = a.gate ? gate_row(a, r) * a.cols : 0;
        float n[NV][V], h[NV][V], s = 0.f, rp = 1.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (t + i * T) * V;
            if (c < a.cols) {
                load_few<Y, V>(static_cast<const Y*>(a.y) + row + c, n[i]);
                load_few<H, V>(static_cast<const H*>(a.h_in) + row + c, h[i]);
            } else
#pragma unroll
                for (int k = 0; k < V; ++k) n[i][k] = h[i][k] = 0.f;
        }
        if (a.gamma_post) {
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int k = 0; k < V; ++k) s = fmaf(n[i][k], n[i][k], s);
            rp = rstd_of(cta_sum(s, area, turn), n_cols, a.eps);
            if (t == 0) a.rstd_post[r] = rp;
        }
        s = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (t + i * T) * V;
            if (c >= a.cols) break;
            float w[V];
            if (a.gamma_post) {
                params_few<V>(a.gamma_post, c, bf16, w);
#pragma unroll
                for (int k = 0; k < V; ++k) n[i][k] = (n[i][k] * rp) * w[k];
            }
            if (a.gate) {
                params_few<V>(a.gate, gate + c, bf16, w);
#pragma unroll
                for (int k = 0; k < V; ++k) n[i][k] *= w[k];
            }
#pragma unroll
            for (int k = 0; k < V; ++k) h[i][k] = fmaf(a.branch_scale, n[i][k], a.residual_scale * h[i][k]);
            store_few<H, V>(static_cast<H*>(a.h) + row + c, h[i]);
#pragma unroll
            for (int k = 0; k < V; ++k) s = fmaf(h[i][k], h[i][k], s);
        }
        const float rn = rstd_of(cta_sum(s, area, turn), n_cols, a.eps);
        if (t == 0) a.rstd_pre[r] = rn;
        if (a.x)
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = (t + i * T) * V;
                if (c >= a.cols) break;
                float w[V];
                params_few<V>(a.gamma_pre, c, bf16, w);
#pragma unroll
                for (int k = 0; k < V; ++k) w[k] = (h[i][k] * rn) * w[k];
                store_few<Y, V>(static_cast<Y*>(a.x) + row + c, w);
            }
    }
}

// Backward.  One reduction per row: with t = dx gamma_pre, w = branch_scale gate gamma_post,
//   G = dh + rn (t - xh c1), c1 = S1 / cols,  S1 = sum t xh
//   mean(w G yh) = (S2 - rn c1 S3) / cols,     S2 = sum w yh (dh + rn t),  S3 = sum w yh xh
// A CTA takes `chunk` consecutive rows.  Its column sums go to the workspace ([CTA][cols] for each weight); those of the gate
// are put down whenever the row of the gate changes, at place CTA + row of the gate (no two CTAs share one: the next CTA begins
// with the same row of the gate or a later one), or in d_gate where one CTA holds all rows of it.
__device__ __forceinline__ float* gate_part(const SeamArgs& a, int64_t g)
{
    const int64_t first = g * a.rows_per_gate, last = min(first + a.rows_per_gate, a.rows) - 1;
    if (first / a.chunk == last / a.chunk) return a.d_gate + g * a.cols;
    const int64_t weights = (int64_t)gridDim.x * a.cols * ((a.d_gamma_pre != nullptr) + (a.d_gamma_post != nullptr));
    return a.ws + weights + (blockIdx.x + g) * a.cols;
}

// The CTA's column sums of the weights, [CTA][cols] for each
__device__ __forceinline__ float* weights_part(const SeamArgs& a, bool post)
{
    return a.ws + ((int64_t)blockIdx.x + (post && a.d_gamma_pre ? gridDim.x : 0)) * a.cols;
}

template <typename Y, typename H, int V, int NE, int T, bool SAME>
__global__ void __launch_bounds__(T, (NE == 4 ? 1024 : 512) / T) seam_grad_few_kernel(const SeamArgs a)
{
    __shared__ float4 area[2][SEAM_MAX_WARPS];
    constexpr int NV = NE / V;
    int turn = 0;
    const int t = threadIdx.x;
    const bool bf16 = SAME ? sizeof(H) == 2 : a.bf16_params;
    const int64_t r0 = blockIdx.x * a.chunk, r1 = min(r0 + a.chunk, a.rows);
    const float inv_cols = 1.0f / (float)a.cols;
    float pre[NV][V], post[NV][V], gates[NV][V];
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int k = 0; k < V; ++k) pre[i][k] = post[i][k] = gates[i][k] = 0.f;
    float rn_next = a.rstd_pre[r0], rp_next = a.gamma_post ? a.rstd_post[r0] : 1.f;             // a row ahead
    for (int64_t r = r0; r < r1; ++r) {
        const int64_t row = r * a.cols, g = a.gate ? gate_row(a, r) : 0;
        const float rn = rn_next, rp = rp_next;
        if (r + 1 < r1) {
            rn_next = a.rstd_pre[r + 1];
            if (a.gamma_post) rp_next = a.rstd_post[r + 1];
        }
        float dx[NV][V], dh[NV][V], y[NV][V], h[NV][V], s[3] = {0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (t + i * T) * V;
#pragma unroll
            for (int k = 0; k < V; ++k) dx[i][k] = dh[i][k] = y[i][k] = h[i][k] = 0.f;
            if (c >= a.cols) continue;
            if (a.dx) load_few<Y, V>(static_cast<const Y*>(a.dx) + row + c, dx[i]);
            load_few<Y, V>(static_cast<const Y*>(a.y) + row + c, y[i]);
            if (a.dh) load_few<H, V>(static_cast<const H*>(a.dh) + row + c, dh[i]);
            load_few<H, V>(static_cast<const H*>(static_cast<const void*>(a.h)) + row + c, h[i]);
        }
        // y, h become yh, xh
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (t + i * T) * V;
            if (c >= a.cols) break;
            float w[V], q[V];
            params_few<V>(a.gamma_pre, c, bf16, w);
#pragma unroll
            for (int k = 0; k < V; ++k) {
                h[i][k] *= rn;
                y[i][k] *= rp;
                w[k] *= dx[i][k];
                s[0] = fmaf(w[k], h[i][k], s[0]);
            }
            if (a.gamma_post) {
                float u[V];
                params_few<V>(a.gamma_post, c, bf16, u);
                if (a.gate) {
                    params_few<V>(a.gate, g * a.cols + c, bf16, q);
#pragma unroll
                    for (int k = 0; k < V; ++k) u[k] *= q[k];
                }
#pragma unroll
                for (int k = 0; k < V; ++k) {
                    u[k] *= y[i][k];
                    s[1] = fmaf(u[k], fmaf(rn, w[k], dh[i][k]), s[1]);
                    s[2] = fmaf(u[k], h[i][k], s[2]);
                }
            }
        }
        cta_sums(s, area, turn);
        const float c1 = s[0] * inv_cols, c2 = (s[1] - rn * c1 * s[2]) * a.branch_scale * inv_cols;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (t + i * T) * V;
            if (c >= a.cols) break;
            float w[V], G[V];
            params_few<V>(a.gamma_pre, c, bf16, w);
#pragma unroll
            for (int k = 0; k < V; ++k) {
                pre[i][k] = fmaf(dx[i][k], h[i][k], pre[i][k]);
                G[k] = fmaf(rn, fmaf(dx[i][k], w[k], -h[i][k] * c1), dh[i][k]);
                w[k] = a.residual_scale * G[k];
                G[k] *= a.branch_scale;
            }
            if (a.dh_in) store_few<H, V>(static_cast<H*>(a.dh_in) + row + c, w);
#pragma unroll
            for (int k = 0; k < V; ++k) w[k] = 1.f;
            if (a.gamma_post) params_few<V>(a.gamma_post, c, bf16, w);
            if (a.d_gate)
#pragma unroll
                for (int k = 0; k < V; ++k) gates[i][k] = fmaf(G[k], y[i][k] * w[k], gates[i][k]);
            if (a.gate) {
                float q[V];
                params_few<V>(a.gate, g * a.cols + c, bf16, q);
#pragma unroll
                for (int k = 0; k < V; ++k) G[k] *= q[k];
            }
            if (a.gamma_post)
#pragma unroll
                for (int k = 0; k < V; ++k) {
                    post[i][k] = fmaf(G[k], y[i][k], post[i][k]);
                    G[k] = rp * fmaf(G[k], w[k], -y[i][k] * c2);
                }
            if (a.dy) store_few<Y, V>(static_cast<Y*>(a.dy) + row + c, G);
        }
        if (a.d_gate && (r + 1 == r1 || (g + 1) * a.rows_per_gate == r + 1)) {
            float* part = gate_part(a, g);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = (t + i * T) * V;
#pragma unroll
                for (int k = 0; k < V; ++k) {
                    if (c < a.cols) part[c + k] = gates[i][k];
                    gates[i][k] = 0.f;
                }
            }
        }
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (t + i * T) * V;
        if (c >= a.cols) break;
#pragma unroll
        for (int k = 0; k < V; ++k) {
            if (a.d_gamma_pre) weights_part(a, false)[c + k] = pre[i][k];
            if (a.d_gamma_post) weights_part(a, true)[c + k] = post[i][k];
        }
    }
}

// The same for rows of any length: one element per thread at a time, column sums in shared memory, rows read a second time (from L2).
template <typename Y, typename H>
__global__ void __launch_bounds__(SEAM_THREADS) seam_grad_any_kernel(const SeamArgs a)
{
    extern __shared__ float column[];              // d_gamma_pre, d_gamma_post, d_gate: each column belongs to one thread
    __shared__ float4 area[2][SEAM_MAX_WARPS];
    int turn = 0;
    float *pre = column, *post = column + a.cols, *gates = column + 2 * a.cols;
    for (int c = threadIdx.x; c < 3 * a.cols; c += SEAM_THREADS) column[c] = 0.f;
    __syncthreads();
    const int64_t r0 = blockIdx.x * a.chunk, r1 = min(r0 + a.chunk, a.rows);
    const float inv_cols = 1.0f / (float)a.cols;
    for (int64_t r = r0; r < r1; ++r) {
        const Y* y = static_cast<const Y*>(a.y) + r * a.cols;
        const H* h = static_cast<const H*>(a.h) + r * a.cols;
        const Y* dx = a.dx ? static_cast<const Y*>(a.dx) + r * a.cols : nullptr;
        const H* dh = a.dh ? static_cast<const H*>(a.dh) + r * a.cols : nullptr;
        Y* dy = a.dy ? static_cast<Y*>(a.dy) + r * a.cols : nullptr;
        H* dh_in = a.dh_in ? static_cast<H*>(a.dh_in) + r * a.cols : nullptr;
        const int64_t g = a.gate ? gate_row(a, r) : 0;
        const float rn = a.rstd_pre[r], rp = a.gamma_post ? a.rstd_post[r] : 1.f;
        float s[3] = {0.f, 0.f, 0.f};
        for (int c = threadIdx.x; c < a.cols; c += SEAM_THREADS) {
            const float xh = to_float(h[c]) * rn, t = dx ? to_float(dx[c]) * param(a.gamma_pre, c, a.bf16_params) : 0.f;
            s[0] = fmaf(t, xh, s[0]);
            if (a.gamma_post) {
                float w = a.branch_scale * param(a.gamma_post, c, a.bf16_params);
                if (a.gate) w *= param(a.gate, g * a.cols + c, a.bf16_params);
                const float wy = w * (to_float(y[c]) * rp);
                s[1] = fmaf(wy, fmaf(rn, t, dh ? to_float(dh[c]) : 0.f), s[1]);
                s[2] = fmaf(wy, xh, s[2]);
            }
        }
        cta_sums(s, area, turn);
        const float c1 = s[0] * inv_cols, c2 = (s[1] - rn * c1 * s[2]) * inv_cols;
        for (int c = threadIdx.x; c < a.cols; c += SEAM_THREADS) {
            const float v = dx ? to_float(dx[c]) : 0.f, xh = to_float(h[c]) * rn;
            const float t = v * param(a.gamma_pre, c, a.bf16_params);
            const float G = fmaf(rn, t - xh * c1, dh ? to_float(dh[c]) : 0.f);
            pre[c] = fmaf(v, xh, pre[c]);
            if (dh_in) dh_in[c] = from_float<H>(a.residual_scale * G);
            const float yh = to_float(y[c]) * rp, branch = a.branch_scale * G;
            const float gamma = a.gamma_post ? param(a.gamma_post, c, a.bf16_params) : 1.f;
            gates[c] = fmaf(branch, yh * gamma, gates[c]);
            const float wG = a.gate ? branch * param(a.gate, g * a.cols + c, a.bf16_params) : branch;
            post[c] = fmaf(wG, yh, post[c]);
            if (dy) dy[c] = from_float<Y>(a.gamma_post ? rp * (wG * gamma - yh * c2) : wG);
        }
        if (a.d_gate && (r + 1 == r1 || (g + 1) * a.rows_per_gate == r + 1)) {
            float* to = gate_part(a, g);
            for (int c = threadIdx.x; c < a.cols; c += SEAM_THREADS) {
                to[c] = gates[c];
                gates[c] = 0.f;
            }
        }
    }
    for (int c = threadIdx.x; c < a.cols; c += SEAM_THREADS) {
        if (a.d_gamma_pre) weights_part(a, false)[c] = pre[c];
        if (a.d_gamma_post) weights_part(a, true)[c] = post[c];
    }
}

// ---------------------------------------------------------------------------------------------------------------------
// Rows that start on 16-byte boundaries.  A thread owns the vectors of eight columns threadIdx.x + i T of every row that its group
// takes (a warp for short rows, else the CTA of T threads).  It copies them itself, asynchronously, into places of shared memory that no other
// thread touches, STAGES - 1 rows ahead: no barrier guards them, only the thread's own wait for its copies.  Where shared memory holds one row of a CTA,
// STAGES is 1 and a row's loads are waited for (backward above 8192 columns, and above 4096 with FP32 on both sides; forward above 8192 with FP32 on both).
template <typename T> constexpr int PIECES = sizeof(T) / 2;            // 16-byte pieces of eight elements

__device__ __forceinline__ void copy16(uint32_t to, const void* from)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" :: "r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void copies_issued() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT>
__device__ __forceinline__ void copies_done() { asm volatile("cp.async.wait_group %0;" :: "n"(LEFT) : "memory"); }

// Eight FP32 values as four pairs: one instruction works on a pair (the same roundings as one at a time, half the issue slots).
struct Eight {
    float2 v[4];
};
__device__ __forceinline__ uint64_t bits(float2 v)
{
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(v.x), "f"(v.y));
    return r;
}
__device__ __forceinline__ float2 pair(uint64_t b)
{
    float2 v;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(v.x), "=f"(v.y) : "l"(b));
    return v;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c)
{
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(bits(a)), "l"(bits(b)), "l"(bits(c)));
    return pair(r);
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b)
{
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(bits(a)), "l"(bits(b)));
    return pair(r);
}
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }
__device__ __forceinline__ Eight zero8()
{
    Eight e;
#pragma unroll
    for (int k = 0; k < 4; ++k) e.v[k] = make_float2(0.f, 0.f);
    return e;
}

__device__ __forceinline__ Eight times(Eight e, float by)
{
#pragma unroll
    for (int k = 0; k < 4; ++k) e.v[k] = mul2(e.v[k], both(by));
    return e;
}

// Eight elements from 16-byte pieces, `apart` bytes from one another in shared memory / side by side in global memory
template <typename T>
__device__ __forceinline__ Eight unpack(const uint4 (&w)[PIECES<T>])
{
    const uint32_t* u = reinterpret_cast<const uint32_t*>(w);
    Eight e;
#pragma unroll
    for (int k = 0; k < 4; ++k)
        e.v[k] = sizeof(T) == 2 ? make_float2(__uint_as_float(u[k] << 16), __uint_as_float(u[k] & 0xFFFF0000u))
                                : make_float2(__uint_as_float(u[(2 * k) % (4 * PIECES<T>)]), __uint_as_float(u[(2 * k + 1) % (4 * PIECES<T>)]));
    return e;
}
template <typename T>
__device__ __forceinline__ Eight load_staged(const uint8_t* at, int apart)
{
    uint4 w[PIECES<T>];
#pragma unroll
    for (int p = 0; p < PIECES<T>; ++p) w[p] = *reinterpret_cast<const uint4*>(at + p * apart);
    return unpack<T>(w);
}
// Stores as T and returns the rounded values
template <typename T>
__device__ __forceinline__ Eight store8(T* to, const Eight& e)
{
    uint4* out = reinterpret_cast<uint4*>(to);
    if constexpr (sizeof(T) == 2) {
        uint32_t u[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const __nv_bfloat162 b = __floats2bfloat162_rn(e.v[k].x, e.v[k].y);
            u[k] = *reinterpret_cast<const uint32_t*>(&b);
        }
        const uint4 w[1] = {make_uint4(u[0], u[1], u[2], u[3])};
        out[0] = w[0];
        return unpack<__nv_bfloat16>(w);
    } else {
        out[0] = make_uint4(__float_as_uint(e.v[0].x), __float_as_uint(e.v[0].y), __float_as_uint(e.v[1].x), __float_as_uint(e.v[1].y));
        out[1] = make_uint4(__float_as_uint(e.v[2].x), __float_as_uint(e.v[2].y), __float_as_uint(e.v[3].x), __float_as_uint(e.v[3].y));
        return e;
    }
}
// Eight weights of a row of parameters; they stay in L1 from row to row
__device__ __forceinline__ Eight params8(const void* p, int64_t at, bool bf16)
{
    if (bf16) {
        const uint4 w[1] = {__ldg(reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(p) + at))};
        return unpack<__nv_bfloat16>(w);
    }
    const uint4* q = reinterpret_cast<const uint4*>(static_cast<const float*>(p) + at);
    const uint4 w[2] = {__ldg(q), __ldg(q + 1)};
    return unpack<float>(w);
}

// Largest magnitude of the finite elements as a bit pattern.  The maximum passes over NaN by itself; an infinity is looked at again.
__device__ __forceinline__ uint32_t finite_peak(const Eight& e)
{
    float peak = fmaxf(fabsf(e.v[0].x), fabsf(e.v[0].y));
#pragma unroll
    for (int k = 1; k < 4; ++k) peak = fmaxf(fmaxf(peak, fabsf(e.v[k].x)), fabsf(e.v[k].y));
    uint32_t bits = __float_as_uint(peak);
    if (bits >= 0x7F800000u) {                       // an infinity, or nothing but NaN
        bits = 0u;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t a = __float_as_uint(e.v[k].x) & 0x7FFFFFFFu, b = __float_as_uint(e.v[k].y) & 0x7FFFFFFFu;
            bits = max(bits, max(a < 0x7F800000u ? a : 0u, b < 0x7F800000u ? b : 0u));
        }
    }
    return bits;
}
// Scale byte of a block with this peak, and the eight codes under it
template <int ELEM>
__device__ __forceinline__ uint2 codes8(const Eight& x, uint32_t peak, int rule, uint32_t& byte)
{
    byte = scale_byte_from_amax_bits<ELEM>(peak, rule);
    const float2 inverse = both(inv_scale_from_byte(byte));
    float2 v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = mul2(x.v[k], inverse);
    return make_uint2(cvt_fp8x4<ELEM>(v[0].x, v[0].y, v[1].x, v[1].y), cvt_fp8x4<ELEM>(v[2].x, v[2].y, v[3].x, v[3].y));
}

// x of eight columns (c .. c + 7) rounded to the stream's type and converted: four lanes share a block, sixteen a word of four scale bytes.
// `codes`, `scales`: the row's.  All lanes of the warp take part; those without columns (in == false) store nothing.
template <typename H>
__device__ __forceinline__ void convert_row(const SeamArgs& a, uint8_t* codes, uint8_t* scales, int c, bool in, Eight x)
{
    if constexpr (sizeof(H) == 2) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const __nv_bfloat162 b = __floats2bfloat162_rn(x.v[k].x, x.v[k].y);
            const uint32_t u = *reinterpret_cast<const uint32_t*>(&b);
            x.v[k] = make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xFFFF0000u));
        }
    }
    uint32_t peak = finite_peak(x), byte;                                   // columns behind the row: zeros
    peak = max(peak, __shfl_xor_sync(0xFFFFFFFFu, peak, 1));
    peak = max(peak, __shfl_xor_sync(0xFFFFFFFFu, peak, 2));
    const uint2 q = a.elem == MXFP8_E4M3 ? codes8<MXFP8_E4M3>(x, peak, a.rule, byte) : codes8<MXFP8_E5M2>(x, peak, a.rule, byte);
    if (in) *reinterpret_cast<uint2*>(codes + c) = q;
    const int lane = threadIdx.x & 31;
    if (a.layout == MXFP8_SF_SWIZZLED) {                                    // whole words: the bytes behind the last block are zero
        uint32_t word = in ? byte << (8 * (lane >> 2 & 3)) : 0u;          // c / 32 % 4 == lane / 4 % 4
        word |= __shfl_xor_sync(0xFFFFFFFFu, word, 4);
        word |= __shfl_xor_sync(0xFFFFFFFFu, word, 8);
        if (in && (lane & 15) == 0) *reinterpret_cast<uint32_t*>(scales + (c >> 7) * 512) = word;
    } else if (in && (lane & 3) == 0) scales[c >> 5] = (uint8_t)byte;
}
// The rows that pad a swizzled scale array to 128, by the threads that took the last row
__device__ __forceinline__ void pad_scales(const SeamArgs& a, int t, int T)
{
    const int words = (a.cols / 32 + 3) / 4;
    const int64_t rest = (128 - a.rows % 128) % 128 * words;
    for (int64_t i = t; i < rest; i += T)
        *reinterpret_cast<uint32_t*>(a.s_row + sf_swizzled_offset(a.rows + i / words, i % words * 4, words * 4)) = 0u;
}

// Forward.  WARP: rows of a warp each (the CTA has four), else of the CTA.  CONVERT: x is converted (see convert_row) instead of stored.
// Rows go last to first: what reads h or x next begins with the first rows, and finds them in L2 (8192 x 4096 in BF16 with the conversion in
// both orientations behind it took 76 us that way and 79 us first to last; it takes 72 us now).
template <typename Y, typename H, int NV, bool WARP, int STAGES, int MODE, bool CONVERT>
__global__ void __launch_bounds__(WARP ? 128 : (NV == 1 ? 1024 : (NV == 2 ? 512 : 256)), WARP ? 8 : (NV == 1 ? 1 : 2)) seam_forward_kernel(const SeamArgs a)
{
    extern __shared__ __align__(16) uint8_t stage_mem[];
    __shared__ float area[2][SEAM_MAX_WARPS];
    constexpr int Q = PIECES<Y> + PIECES<H>;                // 16-byte pieces of a vector of both inputs
    const Known<MODE, H> known{a};
    int turn = 0;
    const int T = WARP ? 32 : blockDim.x, t = WARP ? threadIdx.x & 31 : threadIdx.x;
    const int64_t first = WARP ? (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5) : blockIdx.x, step = WARP ? (int64_t)gridDim.x * 4 : gridDim.x;
    const int piece = blockDim.x * 16;                      // bytes from a piece to the next one of the same thread
    uint8_t* mine = stage_mem + threadIdx.x * 16;
    const uint32_t mine_at = (uint32_t)__cvta_generic_to_shared(mine);
    const float n_cols = (float)a.cols;
    auto issue = [&](int64_t i, int stage) {
        if (i < a.rows) {
            const int64_t r = a.rows - 1 - i;
            const Y* y = static_cast<const Y*>(a.y) + r * a.cols;
            const H* h_in = static_cast<const H*>(a.h_in) + r * a.cols;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = (t + i * T) * 8;
                if (c >= a.cols) break;
                const uint32_t to = mine_at + (stage * NV + i) * Q * piece;
#pragma unroll
                for (int p = 0; p < PIECES<Y>; ++p) copy16(to + p * piece, reinterpret_cast<const uint4*>(y + c) + p);
#pragma unroll
                for (int p = 0; p < PIECES<H>; ++p) copy16(to + (PIECES<Y> + p) * piece, reinterpret_cast<const uint4*>(h_in + c) + p);
            }
        }
        copies_issued();
    };
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s) issue(first + s * step, s);
    int stage = 0;
    for (int64_t n = first; n < a.rows; n += step) {
        issue(n + (STAGES - 1) * step, (stage + STAGES - 1) % STAGES);
        const int64_t r = a.rows - 1 - n;
        copies_done<STAGES - 1>();
        const uint8_t* at = mine + stage * NV * Q * piece;
        float2 s = make_float2(0.f, 0.f);
        float rp = 1.f;
        if (known.post()) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                if ((t + i * T) * 8 >= a.cols) break;
                const Eight y = load_staged<Y>(at + i * Q * piece, piece);
#pragma unroll
                for (int k = 0; k < 4; ++k) s = fma2(y.v[k], y.v[k], s);
            }
            rp = rstd_of(WARP ? warp_sum(s.x + s.y) : cta_sum(s.x + s.y, area, turn), n_cols, a.eps);
            if (t == 0) a.rstd_post[r] = rp;
        }
        s = make_float2(0.f, 0.f);
        Eight h[NV];
        const int64_t gate = known.gate() ? gate_row(a, r) * a.cols : 0;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (t + i * T) * 8;
            if (c >= a.cols) break;
            Eight n = load_staged<Y>(at + i * Q * piece, piece);
            h[i] = load_staged<H>(at + (i * Q + PIECES<Y>) * piece, piece);
            if (known.post()) {
                const Eight w = params8(a.gamma_post, c, known.bf16());
#pragma unroll
                for (int k = 0; k < 4; ++k) n.v[k] = mul2(mul2(n.v[k], both(rp)), w.v[k]);
            }
            if (known.gate()) {
                const Eight w = params8(a.gate, gate + c, known.bf16());
#pragma unroll
                for (int k = 0; k < 4; ++k) n.v[k] = mul2(n.v[k], w.v[k]);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) h[i].v[k] = fma2(both(a.branch_scale), n.v[k], mul2(both(a.residual_scale), h[i].v[k]));
            h[i] = store8(static_cast<H*>(a.h) + r * a.cols + c, h[i]);
#pragma unroll
            for (int k = 0; k < 4; ++k) s = fma2(h[i].v[k], h[i].v[k], s);
        }
        const float rn = rstd_of(WARP ? warp_sum(s.x + s.y) : cta_sum(s.x + s.y, area, turn), n_cols, a.eps);
        if (t == 0) a.rstd_pre[r] = rn;
        if constexpr (CONVERT) {
            uint8_t* codes = a.q_row + r * a.cols;
            uint8_t* scales = a.s_row + (a.layout == MXFP8_SF_SWIZZLED ? sf_swizzled_offset(r, 0, a.cols / 32) : r * (a.cols / 32));
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = (t + i * T) * 8;
                if (c - t % 32 * 8 >= a.cols) break;                       // the whole warp is behind the row
                const bool in = c < a.cols;
                Eight x = zero8();
                if (in) {
                    const Eight w = params8(a.gamma_pre, c, known.bf16());
#pragma unroll
                    for (int k = 0; k < 4; ++k) x.v[k] = mul2(mul2(h[i].v[k], both(rn)), w.v[k]);
                }
                convert_row<H>(a, codes, scales, c, in, x);
            }
            if (r == a.rows - 1 && a.layout == MXFP8_SF_SWIZZLED) pad_scales(a, t, T);
        } else if (a.x) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = (t + i * T) * 8;
                if (c >= a.cols) break;
                const Eight w = params8(a.gamma_pre, c, known.bf16());
#pragma unroll
                for (int k = 0; k < 4; ++k) h[i].v[k] = mul2(mul2(h[i].v[k], both(rn)), w.v[k]);
                store8(static_cast<Y*>(a.x) + r * a.cols + c, h[i]);
            }
        }
        stage = stage + 1 == STAGES ? 0 : stage + 1;
    }
    copies_done<0>();
}

// Backward: same ownership and the same sums as seam_grad_any_kernel; column sums stay in registers.  With one vector per thread so do the
// parameters and, between the two passes over the row, its elements: 8192 x 4096 in BF16 took 82 us that
// way and 86 us with two vectors read twice from shared memory; it takes 76 to 81 us since statistics are read a row ahead and 16 warps join.
template <typename Y, typename H, int NV, int STAGES, int MODE>
__global__ void __launch_bounds__(512, 1) seam_grad_kernel(const SeamArgs a)
{
    extern __shared__ __align__(16) uint8_t stage_mem[];
    __shared__ float4 area[2][SEAM_MAX_WARPS];
    constexpr int Q = 2 * (PIECES<Y> + PIECES<H>);          // dx, y, dh, h
    constexpr int AT_Y = PIECES<Y>, AT_DH = 2 * PIECES<Y>, AT_H = 2 * PIECES<Y> + PIECES<H>;
    const Known<MODE, H> known{a};
    int turn = 0;
    const int T = blockDim.x, t = threadIdx.x, piece = T * 16;
    uint8_t* mine = stage_mem + t * 16;
    const uint32_t mine_at = (uint32_t)__cvta_generic_to_shared(mine);
    const int64_t r0 = blockIdx.x * a.chunk, r1 = min(r0 + a.chunk, a.rows);
    const float inv_cols = 1.0f / (float)a.cols;
    auto fetch = [&](uint32_t to, const auto* from) {
#pragma unroll
        for (int p = 0; p < PIECES<std::remove_cv_t<std::remove_reference_t<decltype(*from)>>>; ++p)
            copy16(to + p * piece, reinterpret_cast<const uint4*>(from) + p);
    };
    auto issue = [&](int64_t r, int stage) {
        if (r < r1)
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = (t + i * T) * 8;
                if (c >= a.cols) break;
                const uint32_t to = mine_at + (stage * NV + i) * Q * piece;
                const int64_t at = r * a.cols + c;
                if (known.dx()) fetch(to, static_cast<const Y*>(a.dx) + at);
                fetch(to + AT_Y * piece, static_cast<const Y*>(a.y) + at);
                if (known.dh()) fetch(to + AT_DH * piece, static_cast<const H*>(a.dh) + at);
                fetch(to + AT_H * piece, static_cast<const H*>(static_cast<const void*>(a.h)) + at);
            }
        copies_issued();
    };
    constexpr bool KEEP = NV == 1;
    Eight pre[NV], post[NV], gates[NV];                      // those of gamma_post and the gate without branch_scale
#pragma unroll
    for (int i = 0; i < NV; ++i) pre[i] = post[i] = gates[i] = zero8();
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s) issue(r0 + s, s);
    Eight keep_pre, keep_post, keep_gate, keep_xh, keep_dx, keep_sum, keep_yh;
    int64_t gate_kept = -1;
    if (KEEP && t * 8 < a.cols) {
        keep_pre = params8(a.gamma_pre, t * 8, known.bf16());
        if (known.post()) keep_post = params8(a.gamma_post, t * 8, known.bf16());
    }
    auto gamma_pre = [&](int c) { return KEEP ? keep_pre : params8(a.gamma_pre, c, known.bf16()); };
    auto gamma_post = [&](int c) { return KEEP ? keep_post : params8(a.gamma_post, c, known.bf16()); };
    auto gate_at = [&](int64_t g, int c) { return KEEP ? keep_gate : params8(a.gate, g * a.cols + c, known.bf16()); };
    int stage = 0;
    float rn_next = a.rstd_pre[r0], rp_next = known.post() ? a.rstd_post[r0] : 1.f;             // a row ahead
    for (int64_t r = r0; r < r1; ++r) {
        issue(r + STAGES - 1, (stage + STAGES - 1) % STAGES);
        const int64_t g = known.gate() ? gate_row(a, r) : 0;
        const float rn = rn_next, rp = rp_next;
        if (r + 1 < r1) {
            rn_next = a.rstd_pre[r + 1];
            if (known.post()) rp_next = a.rstd_post[r + 1];
        }
        if (KEEP && known.gate() && g != gate_kept) {
            if (t * 8 < a.cols) keep_gate = params8(a.gate, g * a.cols + t * 8, known.bf16());
            gate_kept = g;
        }
        copies_done<STAGES - 1>();
        const uint8_t* at = mine + stage * NV * Q * piece;
        // sums of products of normalised elements: with both statistics left out until the end, their squares leave FP32's range for small rows
        float2 s0 = make_float2(0.f, 0.f), s1 = s0, s2 = s0;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (t + i * T) * 8;
            if (c >= a.cols) break;
            const uint8_t* from = at + i * Q * piece;
            const Eight xh = times(load_staged<H>(from + AT_H * piece, piece), rn);
            keep_xh = xh;
            Eight d = zero8();
            if (known.dx()) {
                d = load_staged<Y>(from, piece);
                const Eight w = gamma_pre(c);
                keep_dx = d;
#pragma unroll
                for (int k = 0; k < 4; ++k) d.v[k] = mul2(d.v[k], w.v[k]);
            }
            Eight e = known.dh() ? load_staged<H>(from + AT_DH * piece, piece) : zero8();
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                s0 = fma2(d.v[k], xh.v[k], s0);
                e.v[k] = fma2(both(rn), d.v[k], e.v[k]);
            }
            keep_sum = e;
            if (known.post()) {
                Eight w = gamma_post(c);
                if (known.gate()) {
                    const Eight q = gate_at(g, c);
#pragma unroll
                    for (int k = 0; k < 4; ++k) w.v[k] = mul2(w.v[k], q.v[k]);
                }
                const Eight yh = times(load_staged<Y>(from + AT_Y * piece, piece), rp);
                keep_yh = yh;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    w.v[k] = mul2(w.v[k], yh.v[k]);
                    s1 = fma2(w.v[k], e.v[k], s1);
                    s2 = fma2(w.v[k], xh.v[k], s2);
                }
            }
        }
        float s[3] = {s0.x + s0.y, s1.x + s1.y, s2.x + s2.y};
        cta_sums(s, area, turn);
        // G = (dh + rn t) - k1 xh;  dy = kb G w - k2 yh
        const float k1 = rn * (s[0] * inv_cols), kb = a.branch_scale * rp, k2 = rp * ((s[1] - k1 * s[2]) * a.branch_scale * inv_cols);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (t + i * T) * 8;
            if (c >= a.cols) break;
            const uint8_t* from = at + i * Q * piece;
            const int64_t to = r * a.cols + c;
            const bool kept = KEEP && known.post();          // y is looked at in the first pass then
            const Eight xh = KEEP ? keep_xh : times(load_staged<H>(from + AT_H * piece, piece), rn);
            Eight G = KEEP ? keep_sum : (known.dh() ? load_staged<H>(from + AT_DH * piece, piece) : zero8());
            if (known.dx()) {
                const Eight d = KEEP ? keep_dx : load_staged<Y>(from, piece);
#pragma unroll
                for (int k = 0; k < 4; ++k) pre[i].v[k] = fma2(d.v[k], xh.v[k], pre[i].v[k]);
                if (!KEEP) {
                    const Eight w = gamma_pre(c);
#pragma unroll
                    for (int k = 0; k < 4; ++k) G.v[k] = fma2(both(rn), mul2(d.v[k], w.v[k]), G.v[k]);
                }
            }
            Eight out;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                G.v[k] = fma2(both(-k1), xh.v[k], G.v[k]);
                out.v[k] = mul2(both(a.residual_scale), G.v[k]);
            }
            if (known.dh_in()) store8(static_cast<H*>(a.dh_in) + to, out);
            Eight yh = kept ? keep_yh : load_staged<Y>(from + AT_Y * piece, piece);
            if (known.post() && !kept) yh = times(yh, rp);
            const Eight w = known.post() ? gamma_post(c) : zero8();
            if (known.d_gate())
#pragma unroll
                for (int k = 0; k < 4; ++k) gates[i].v[k] = fma2(G.v[k], known.post() ? mul2(yh.v[k], w.v[k]) : yh.v[k], gates[i].v[k]);
            if (known.gate()) {
                const Eight q = gate_at(g, c);
#pragma unroll
                for (int k = 0; k < 4; ++k) G.v[k] = mul2(G.v[k], q.v[k]);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float2 scaled = mul2(both(kb), G.v[k]);                  // without a norm after the block, dy
                out.v[k] = scaled;
                if (known.post()) {
                    post[i].v[k] = fma2(G.v[k], yh.v[k], post[i].v[k]);
                    out.v[k] = fma2(scaled, w.v[k], mul2(both(-k2), yh.v[k]));
                }
            }
            if (known.dy()) store8(static_cast<Y*>(a.dy) + to, out);
        }
        if (known.d_gate() && (r + 1 == r1 || (g + 1) * a.rows_per_gate == r + 1)) {
            float* part = gate_part(a, g);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = (t + i * T) * 8;
                if (c >= a.cols) break;
                store8(part + c, times(gates[i], a.branch_scale));
                gates[i] = zero8();
            }
        }
        stage = stage + 1 == STAGES ? 0 : stage + 1;
    }
    copies_done<0>();
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (t + i * T) * 8;
        if (c >= a.cols) break;
        if (a.d_gamma_pre) store8(weights_part(a, false) + c, pre[i]);
        if (a.d_gamma_post) store8(weights_part(a, true) + c, times(post[i], a.branch_scale));
    }
}

// Joins the CTAs' sums; 16 warps because the latency of the loads is what it waits for (3065 x 2048 with gates: 39.5 us, 41.1 with 8).
// blockIdx.y: 0 / 1 the weights, then the rows of the gate that several CTAs hold.
constexpr int JOIN_COLS = 32, JOIN_WARPS = 16;
__global__ void __launch_bounds__(32 * JOIN_WARPS) seam_join_kernel(const SeamArgs a, int parts)
{
    __shared__ float area[JOIN_WARPS][JOIN_COLS];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int c = blockIdx.x * JOIN_COLS + lane, weights = (a.d_gamma_pre != nullptr) + (a.d_gamma_post != nullptr);
    for (int64_t which = blockIdx.y; which < weights + (a.d_gate ? a.gates : 0); which += gridDim.y) {
        const float* from;
        float* to;
        int64_t count = parts;
        if (which < weights) {
            from = a.ws + which * (int64_t)parts * a.cols;
            to = (which == 0 && a.d_gamma_pre) ? a.d_gamma_pre : a.d_gamma_post;
        } else {
            const int64_t g = which - weights, first = g * a.rows_per_gate, last = min(first + a.rows_per_gate, a.rows) - 1;
            const int64_t b0 = first / a.chunk;
            count = last / a.chunk - b0 + 1;
            if (count == 1) continue;
            from = a.ws + ((int64_t)weights * parts + b0 + g) * a.cols;
            to = a.d_gate + g * a.cols;
        }
        float s = 0.f;
        if (c < a.cols) {
#pragma unroll 8
            for (int64_t p = warp; p < count; p += JOIN_WARPS) s += from[p * a.cols + c];
        }
        area[warp][lane] = s;
        __syncthreads();
        if (warp == 0) {
            s = 0.f;
#pragma unroll
            for (int w = 0; w < JOIN_WARPS; ++w) s += area[w][lane];
            if (c < a.cols) to[c] = s;
        }
        __syncthreads();
    }
}

int multiprocessors()
{
    static PerDeviceCache<int> cache;
    int n = 0;
    return cache.get(n, [](int dev, int& v) { return cudaDeviceGetAttribute(&v, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess; }) ? n : 148;
}

bool misaligned(const void* p, int dtype) { return (reinterpret_cast<uintptr_t>(p) & (dtype == MXFP8_BF16 ? 1u : 3u)) != 0; }

int seam_check(const mxfp8_seam* s)
{
    if (!s) return MXFP8_ERR_NULL;
    for (int d : {s->block_dtype, s->stream_dtype, s->param_dtype})
        if (d != MXFP8_FP32 && d != MXFP8_BF16) return MXFP8_ERR_ENUM;
    if (!s->gamma_pre) return MXFP8_ERR_NULL;
    if (s->rows <= 0 || s->cols <= 0 || !(s->eps >= 0.f) || (s->gate && s->rows_per_gate < 1)) return MXFP8_ERR_SHAPE;
    if (misaligned(s->gamma_pre, s->param_dtype) || misaligned(s->gamma_post, s->param_dtype) || misaligned(s->gate, s->param_dtype)) return MXFP8_ERR_ALIGN;
    if (s->cols > SEAM_MAX_COLS || s->rows > (1LL << 40)) return MXFP8_ERR_UNSUPPORTED;
    return MXFP8_OK;
}

SeamArgs seam_args(const mxfp8_seam* s)
{
    SeamArgs a{};
    a.rows = s->rows; a.cols = (int)s->cols;
    a.gamma_post = s->gamma_post; a.gate = s->gate; a.gamma_pre = s->gamma_pre;
    a.bf16_params = s->param_dtype == MXFP8_BF16;
    // one row of the gate for all is the same as rows_per_gate = rows
    a.rows_per_gate = s->gate ? (s->rows_per_gate < s->rows ? s->rows_per_gate : s->rows) : s->rows;
    a.gates = (s->rows + a.rows_per_gate - 1) / a.rows_per_gate;
    if (a.rows <= 0x7FFFFFFFLL) a.gate_magic = div_magic((uint32_t)a.rows_per_gate);
    a.branch_scale = s->branch_scale; a.residual_scale = s->residual_scale; a.eps = s->eps;
    return a;
}

// Calls f with two null pointers of the block's and the stream's element types.
template <typename F>
cudaError_t by_types(const mxfp8_seam* s, F f)
{
    using B = __nv_bfloat16;
    if (s->block_dtype == MXFP8_BF16)
        return s->stream_dtype == MXFP8_BF16 ? f((B*)nullptr, (B*)nullptr) : f((B*)nullptr, (float*)nullptr);
    return s->stream_dtype == MXFP8_BF16 ? f((float*)nullptr, (B*)nullptr) : f((float*)nullptr, (float*)nullptr);
}

// Rows on 16-byte boundaries everywhere
template <typename... P>
bool rows_aligned(const SeamArgs& a, const P*... p)
{
    return a.cols % 8 == 0 && (aligned16(p) && ...) && aligned16(a.gamma_post) && aligned16(a.gate) && aligned16(a.gamma_pre);
}

// Rows of an even number of elements that start on boundaries of two elements
template <typename Y, typename H>
bool even_rows(const SeamArgs& a, std::initializer_list<const void*> block, std::initializer_list<const void*> stream)
{
    uintptr_t off = 0;
    for (const void* p : block) off |= reinterpret_cast<uintptr_t>(p) & (2 * sizeof(Y) - 1);
    for (const void* p : stream) off |= reinterpret_cast<uintptr_t>(p) & (2 * sizeof(H) - 1);
    for (const void* p : {a.gamma_post, a.gate, a.gamma_pre}) off |= reinterpret_cast<uintptr_t>(p) & (a.bf16_params ? 3u : 7u);
    return a.cols % 2 == 0 && off == 0;
}

constexpr int SMEM_PER_SM = 224 * 1024;

// Whether the kernels that know the usual seam fit (see Known)
template <typename H>
int mode_of(const SeamArgs& a, bool backward)
{
    if (!a.gamma_post || a.bf16_params != (sizeof(H) == 2)) return 0;
    if (backward && (!a.dx || !a.dh || !a.dy || !a.dh_in || (a.gate != nullptr) != (a.d_gate != nullptr))) return 0;
    return a.gate ? 2 : 1;
}

template <typename Y, typename H, int NV, bool WARP, int STAGES, int MODE = 0, bool CONVERT = false>
cudaError_t launch_forward_rows(const SeamArgs& a, int threads, cudaStream_t st)
{
    if (!CONVERT && a.q_row) return launch_forward_rows<Y, H, NV, WARP, STAGES, MODE, true>(a, threads, st);
    if (MODE == 0 && !WARP && mode_of<H>(a, false) == 1) return launch_forward_rows<Y, H, NV, WARP, STAGES, MODE == 0 && !WARP ? 1 : MODE, CONVERT>(a, threads, st);
    auto kernel = seam_forward_kernel<Y, H, NV, WARP, STAGES, MODE, CONVERT>;
    const int smem = STAGES * NV * (PIECES<Y> + PIECES<H>) * 16 * threads;
    static unsigned long long set = 0;
    const cudaError_t err = ensure_dynamic_smem(kernel, SMEM_PER_SM, set);
    if (err != cudaSuccess) return err;
    const int by_threads = (NV == 8 ? 512 : 1024) / threads, by_smem = SMEM_PER_SM / (smem + 1024), per_sm = by_threads < by_smem ? by_threads : by_smem;
    const int64_t groups = WARP ? (a.rows + 3) / 4 : a.rows, most = (int64_t)multiprocessors() * (per_sm < 1 ? 1 : per_sm);
    kernel<<<(unsigned)(groups < most ? groups : most), threads, smem, st>>>(a);
    count_launch(1);
    return cudaGetLastError();
}

template <typename Y, typename H>
cudaError_t launch_forward(const SeamArgs& a, cudaStream_t st)
{
    if (!rows_aligned(a, a.y, a.h_in, a.h, a.x)) {
        const bool two = even_rows<Y, H>(a, {a.y, a.x}, {a.h_in, a.h}), same = a.bf16_params == (sizeof(H) == 2);
        auto go = [&](auto kernel, int threads) {
            const int64_t most = (int64_t)multiprocessors() * (1536 / threads < 24 ? 1536 / threads : 24);
            kernel<<<(unsigned)(a.rows < most ? a.rows : most), threads, 0, st>>>(a);
        };
        auto by_width = [&](auto v, auto s) {
            constexpr int V = decltype(v)::value;
            constexpr bool SAME = decltype(s)::value;
            if (a.cols <= 256) go(seam_forward_any_kernel<Y, H, V, 8, 32, SAME>, 32);
            else if (a.cols <= 2048) go(seam_forward_any_kernel<Y, H, V, 8, 256, SAME>, 256);
            else if (a.cols <= 8192) go(seam_forward_any_kernel<Y, H, V, 16, 512, SAME>, 512);
            else go(seam_forward_any_kernel<Y, H, V, 16, 1024, SAME>, 1024);
        };
        using one_t = std::integral_constant<int, 1>;
        using two_t = std::integral_constant<int, 2>;
        if (two) same ? by_width(two_t{}, std::true_type{}) : by_width(two_t{}, std::false_type{});
        else same ? by_width(one_t{}, std::true_type{}) : by_width(one_t{}, std::false_type{});
        count_launch(1);
        return cudaGetLastError();
    }
    const int vectors = a.cols / 8, warps = (vectors + 31) / 32;
    // Rows of one warp's width: a warp each (8192 x 256 BF16 6.0 us, 6.7 with a CTA each).
    // Wider ones, as long as CTAs of one vector per thread hold all rows at once: those (1184 x 1024 4.3 us, 5.0 with two vectors; 296 x 4096 4.7 and
    // 5.6).  With more rows two vectors per thread pay (2368 x 1024 6.6 us, 6.9 with one; 592 x 4096 6.6 and 7.0), up to 512 columns in a
    // warp per row (4736 x 512 6.5 us, 7.6 in a CTA per row; 8192 x 512 9.8 and 9.7; wider rows lose that way, 8192 x 1024 21 and 15).
    if (warps == 1) return launch_forward_rows<Y, H, 1, true, 4>(a, 128, st);
    if (warps <= 32 && a.rows <= (int64_t)multiprocessors() * (32 / warps)) return launch_forward_rows<Y, H, 1, false, 2>(a, 32 * warps, st);
    if (warps == 2) return launch_forward_rows<Y, H, 2, true, 3>(a, 128, st);
    if (warps <= 32) return launch_forward_rows<Y, H, 2, false, 2>(a, 32 * ((warps + 1) / 2), st);
    // 16384 columns of two FP32 inputs leave room for one row at a time
    return launch_forward_rows<Y, H, 8, false, PIECES<Y> + PIECES<H> == 4 ? 1 : 2>(a, 32 * ((warps + 7) / 8), st);
}

// CTAs of the backward pass per multiprocessor, by the width alone (the workspace's size follows from it): as many as registers allow.
// (16 warps of 128 registers)
int grad_ctas_per_sm(int64_t cols) { return cols > 2048 ? 1 : (cols > 1024 ? 2 : (cols > 512 ? 4 : 8)); }
int64_t grad_chunk(int64_t rows, int64_t cols)
{
    const int64_t ctas = (int64_t)grad_ctas_per_sm(cols) * multiprocessors();
    return (rows + ctas - 1) / ctas;
}

template <typename Y, typename H, int NV, int STAGES, int MODE = 0>
cudaError_t launch_grad_rows(const SeamArgs& a, int threads, unsigned ctas, cudaStream_t st)
{
    if (MODE == 0 && mode_of<H>(a, true) == 1) return launch_grad_rows<Y, H, NV, STAGES, MODE == 0 ? 1 : MODE>(a, threads, ctas, st);
    if (MODE == 0 && mode_of<H>(a, true) == 2) return launch_grad_rows<Y, H, NV, STAGES, MODE == 0 ? 2 : MODE>(a, threads, ctas, st);
    auto kernel = seam_grad_kernel<Y, H, NV, STAGES, MODE>;
    static unsigned long long set = 0;
    const cudaError_t err = ensure_dynamic_smem(kernel, SMEM_PER_SM, set);
    if (err != cudaSuccess) return err;
    kernel<<<ctas, threads, STAGES * NV * 2 * (PIECES<Y> + PIECES<H>) * 16 * threads, st>>>(a);
    return cudaGetLastError();
}

template <typename Y, typename H>
cudaError_t launch_grad(SeamArgs a, cudaStream_t st)
{
    const unsigned ctas = (unsigned)((a.rows + a.chunk - 1) / a.chunk);
    cudaError_t rc;
    // a row of the four inputs has to fit shared memory (it does but for rows of 16384 FP32 numbers)
    if (rows_aligned(a, a.dx, a.dh, a.y, a.h, a.dy, a.dh_in, a.d_gate) && a.cols * 2 * (int)(sizeof(Y) + sizeof(H)) <= SMEM_PER_SM) {
        constexpr int Q = PIECES<Y> + PIECES<H>;
        const int warps = (a.cols / 8 + 31) / 32;
        if (warps <= 16) rc = launch_grad_rows<Y, H, 1, Q == 2 ? 4 : (Q == 3 ? 4 : 3)>(a, 32 * warps, ctas, st);
        else if (warps <= 32) rc = launch_grad_rows<Y, H, 2, Q == 2 ? 3 : (Q == 3 ? 2 : 1)>(a, 32 * ((warps + 1) / 2), ctas, st);
        else rc = launch_grad_rows<Y, H, 4, 1>(a, 32 * ((warps + 3) / 4), ctas, st);
    } else if (a.cols <= 8192) {
        const bool two = even_rows<Y, H>(a, {a.dx, a.y, a.dy}, {a.dh, a.h, a.dh_in}), same = a.bf16_params == (sizeof(H) == 2);
        auto by_width = [&](auto v, auto s) {
            constexpr int V = decltype(v)::value;
            constexpr bool SAME = decltype(s)::value;
            if (a.cols <= 256) seam_grad_few_kernel<Y, H, V, 4, 64, SAME><<<ctas, 64, 0, st>>>(a);
            else if (a.cols <= 1024) seam_grad_few_kernel<Y, H, V, 4, 256, SAME><<<ctas, 256, 0, st>>>(a);
            else if (a.cols <= 2048) seam_grad_few_kernel<Y, H, V, 4, 512, SAME><<<ctas, 512, 0, st>>>(a);
            else if (a.cols <= 4096) seam_grad_few_kernel<Y, H, V, 8, 512, SAME><<<ctas, 512, 0, st>>>(a);
            else seam_grad_few_kernel<Y, H, V, 16, 512, SAME><<<ctas, 512, 0, st>>>(a);
        };
        using one_t = std::integral_constant<int, 1>;
        using two_t = std::integral_constant<int, 2>;
        if (two) same ? by_width(two_t{}, std::true_type{}) : by_width(two_t{}, std::false_type{});
        else same ? by_width(one_t{}, std::true_type{}) : by_width(one_t{}, std::false_type{});
        rc = cudaGetLastError();
    } else {
        auto kernel = seam_grad_any_kernel<Y, H>;
        static unsigned long long set = 0;
        const cudaError_t err = ensure_dynamic_smem(kernel, 3 * SEAM_MAX_COLS * (int)sizeof(float), set);
        if (err != cudaSuccess) return err;
        kernel<<<ctas, SEAM_THREADS, 3 * a.cols * sizeof(float), st>>>(a);
        rc = cudaGetLastError();
    }
    count_launch(1);
    const int64_t joins = (a.d_gamma_pre != nullptr) + (a.d_gamma_post != nullptr) + (a.d_gate ? a.gates : 0);
    if (rc != cudaSuccess || joins == 0) return rc;
    cudaLaunchConfig_t cfg{};                               // begins while the first launch ends, and waits for it itself
    cfg.gridDim = dim3((a.cols + JOIN_COLS - 1) / JOIN_COLS, (unsigned)(joins < 1024 ? joins : 1024));
    cfg.blockDim = dim3(32 * JOIN_WARPS);
    cfg.stream = st;
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    rc = cudaLaunchKernelEx(&cfg, seam_join_kernel, a, (int)ctas);
    if (rc == cudaSuccess) count_launch(1);
    return rc;
}

int seam_forward(const mxfp8_seam* s, const void* y, const void* h_in, void* h, void* x, float* rstd_post, float* rstd_pre, cudaStream_t st,
                 void* q_row = nullptr, void* s_row = nullptr, int elem = 0, int rule = 0, int layout = 0)
{
    SeamArgs a = seam_args(s);
    a.y = y; a.h_in = h_in; a.h = h; a.x = x; a.rstd_post = rstd_post; a.rstd_pre = rstd_pre;
    a.q_row = static_cast<uint8_t*>(q_row); a.s_row = static_cast<uint8_t*>(s_row); a.elem = elem; a.rule = rule; a.layout = layout;
    const cudaError_t err = by_types(s, [&](auto* yt, auto* ht) {
        return launch_forward<std::remove_pointer_t<decltype(yt)>, std::remove_pointer_t<decltype(ht)>>(a, st);
    });
    return err == cudaSuccess ? MXFP8_OK : MXFP8_ERR_CUDA;
}

int forward_check(const mxfp8_seam* s, const void* y, const void* h_in, const void* h, const float* rstd_post, const float* rstd_pre)
{
    const int bad = seam_check(s);
    if (bad != MXFP8_OK) return bad;
    if (!y || !h_in || !h || !rstd_pre || (s->gamma_post && !rstd_post)) return MXFP8_ERR_NULL;
    if (misaligned(y, s->block_dtype) || misaligned(h_in, s->stream_dtype) || misaligned(h, s->stream_dtype) ||
        misaligned(rstd_post, MXFP8_FP32) || misaligned(rstd_pre, MXFP8_FP32)) return MXFP8_ERR_ALIGN;
    return MXFP8_OK;
}

}  // namespace
}  // namespace mxfp8

using namespace mxfp8;

extern "C" int mxfp8_residual_rmsnorm(const mxfp8_seam* seam, const void* y, const void* h_in, void* h, void* x,
                                      float* rstd_post, float* rstd_pre, void* stream)
{
    const int bad = forward_check(seam, y, h_in, h, rstd_post, rstd_pre);
    if (bad != MXFP8_OK) return bad;
    if (misaligned(x, seam->block_dtype)) return MXFP8_ERR_ALIGN;
    return seam_forward(seam, y, h_in, h, x, rstd_post, rstd_pre, static_cast<cudaStream_t>(stream));
}

extern "C" int mxfp8_residual_rmsnorm_quantize(const mxfp8_seam* seam, const void* y, const void* h_in, void* h, float* rstd_post, float* rstd_pre,
                                               int orientation, int scale_rule, int elem, void* q_row, void* s_row, void* q_col, void* s_col,
                                               int sf_layout, void* stream)
{
    int bad = forward_check(seam, y, h_in, h, rstd_post, rstd_pre);
    if (bad != MXFP8_OK) return bad;
    if (seam->param_dtype != seam->stream_dtype) return MXFP8_ERR_UNSUPPORTED;
    bad = rmsnorm_check(h, seam->stream_dtype, seam->rows, seam->cols, seam->gamma_pre, seam->eps, rstd_pre, orientation, scale_rule, elem,
                        q_row, s_row, q_col, s_col, sf_layout);
    if (bad != MXFP8_OK) return bad;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    // row blocks alone, of 8-bit elements: converted where x is computed.  (Column blocks need 32 rows at a time: a second launch, which reads h.)
    if (orientation == MXFP8_ROW && fp8_elem(elem) && aligned16(y) && aligned16(h_in) && aligned16(seam->gamma_post) && aligned16(seam->gate))
        return seam_forward(seam, y, h_in, h, nullptr, rstd_post, rstd_pre, st, q_row, s_row, elem, scale_rule, sf_layout);
    bad = seam_forward(seam, y, h_in, h, nullptr, rstd_post, rstd_pre, st);
    if (bad != MXFP8_OK) return bad;
    const QuantizeItem item{h, seam->rows, seam->cols, q_row, s_row, q_col, s_col};
    return quantize_tma_batch(&item, 1, seam->stream_dtype, orientation, scale_rule, elem, sf_layout, st, false, MXFP8_ACT_NONE, rstd_pre, seam->gamma_pre);
}

extern "C" size_t mxfp8_residual_rmsnorm_grad_ws_bytes(const mxfp8_seam* seam)
{
    if (seam_check(seam) != MXFP8_OK) return 0;
    const SeamArgs a = seam_args(seam);
    const int64_t chunk = grad_chunk(a.rows, a.cols), ctas = (a.rows + chunk - 1) / chunk;
    const int64_t parts = ctas * (1 + (seam->gamma_post != nullptr)) + (seam->gate ? ctas + a.gates : 0);
    return (size_t)parts * (size_t)a.cols * sizeof(float);
}

extern "C" int mxfp8_residual_rmsnorm_grad(const mxfp8_seam* seam, const void* dx, const void* dh, const void* y, const void* h,
                                           const float* rstd_post, const float* rstd_pre, void* dy, void* dh_in,
                                           float* d_gamma_pre, float* d_gamma_post, float* d_gate, void* ws, size_t ws_bytes, void* stream)
{
    const int bad = seam_check(seam);
    if (bad != MXFP8_OK) return bad;
    if (!y || !h || !rstd_pre || (seam->gamma_post && !rstd_post) || (!seam->gamma_post && d_gamma_post) || (!seam->gate && d_gate)) return MXFP8_ERR_NULL;
    for (const void* p : {dx, y, static_cast<const void*>(dy)}) if (misaligned(p, seam->block_dtype)) return MXFP8_ERR_ALIGN;
    for (const void* p : {dh, h, static_cast<const void*>(dh_in)}) if (misaligned(p, seam->stream_dtype)) return MXFP8_ERR_ALIGN;
    for (const float* p : {rstd_post, rstd_pre, static_cast<const float*>(d_gamma_pre), static_cast<const float*>(d_gamma_post), static_cast<const float*>(d_gate)})
        if (misaligned(p, MXFP8_FP32)) return MXFP8_ERR_ALIGN;
    if (!ws || ws_bytes < mxfp8_residual_rmsnorm_grad_ws_bytes(seam)) return MXFP8_ERR_WORKSPACE;
    if (!aligned16(ws)) return MXFP8_ERR_ALIGN;
    SeamArgs a = seam_args(seam);
    a.dx = dx; a.dh = dh; a.y = y; a.h = const_cast<void*>(h);
    a.rstd_post = const_cast<float*>(rstd_post); a.rstd_pre = const_cast<float*>(rstd_pre);
    a.dy = dy; a.dh_in = dh_in; a.d_gamma_pre = d_gamma_pre; a.d_gamma_post = d_gamma_post; a.d_gate = d_gate;
    a.ws = static_cast<float*>(ws);
    a.chunk = grad_chunk(a.rows, a.cols);
    const cudaError_t err = by_types(seam, [&](auto* yt, auto* ht) {
        return launch_grad<std::remove_pointer_t<decltype(yt)>, std::remove_pointer_t<decltype(ht)>>(a, static_cast<cudaStream_t>(stream));
    });
    return err == cudaSuccess ? MXFP8_OK : MXFP8_ERR_CUDA;
}
