// A mixture-of-experts layer for a few tokens with packed E2M1 matrices (mxfp8_e2m1_moe), in two launches:
//   1. the choice of the experts from the router's logits, their gate / up products, m = act(gate) * up
//   2. the down products of the chosen experts and their weighted sum, straight into y
// Every CTA of both launches chooses for itself (a few hundred logits, cheaper than a launch in between).  Bound by the
// weights of the experts that are used, 17/32 byte each, which are read once.
#include "e2m1_tiles.cuh"
#include "mxfp8_host.h"

namespace mxfp8 {
namespace {

constexpr int MOE_MAX_TOKENS = 64, MOE_MAX_EXPERTS = 256, MOE_MAX_TOP_K = 16;
constexpr int MOE_WARPS = 8, MOE_THREADS = 32 * MOE_WARPS;

struct MoeArgs {
    const __nv_bfloat16* x;          // [tokens, cols]
    const float* logits;             // [tokens, experts]
    const uint8_t *gate_up, *down;   // packed
    void* y;                         // [tokens, cols]
    bool bf16_out;
    int32_t* ids;
    float* weights;
    __nv_bfloat16 *m_hi, *m_lo;      // [slots, inner]: m = m_hi + m_lo
    int tokens, experts, top_k, act, renormalize;
    int cols, inner;
    int col_tiles, inner_tiles;      // column tiles of gate_up and of down
};

// What a CTA knows of the choice.
struct Choice {
    float weight[MOE_MAX_TOKENS * MOE_MAX_TOP_K];
    short expert[MOE_MAX_TOKENS * MOE_MAX_TOP_K];         // -1: none
    uint32_t used[MOE_MAX_EXPERTS / 32];                  // one bit per expert
};

// Unsigned numbers in the order of the logits; 0 for one that is never chosen (-Inf, NaN).  Both zeros are equal.
__device__ __forceinline__ uint32_t order_of(float l)
{
    if (!(l > -INFINITY)) return 0u;
    const uint32_t u = __float_as_uint(l + 0.f);
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float logit_of(uint32_t o) { return __uint_as_float((o & 0x80000000u) ? (o ^ 0x80000000u) : ~o); }
// exp(l - top), with equal infinities at the top counting as equal
__device__ __forceinline__ float share_of(uint32_t o, uint32_t top) { return o == top ? 1.f : expf(logit_of(o) - logit_of(top)); }

// Chooses for all tokens, a warp for each in turn: top_k rounds of the largest remaining logit (the lowest expert among equals).
// Ends with a barrier.
__device__ __forceinline__ void choose(const MoeArgs& a, Choice& choice)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    if (threadIdx.x < MOE_MAX_EXPERTS / 32) choice.used[threadIdx.x] = 0u;
    __syncthreads();
    for (int t = warp; t < a.tokens; t += warps) {
        uint32_t left[MOE_MAX_EXPERTS / 32];
#pragma unroll
        for (int i = 0; i < MOE_MAX_EXPERTS / 32; ++i)
            left[i] = lane + 32 * i < a.experts ? order_of(a.logits[t * a.experts + lane + 32 * i]) : 0u;
        uint32_t top = 0u;
        float mine = 0.f, total = 0.f;               // lane j: the share of choice j
        for (int j = 0; j < a.top_k; ++j) {
            uint32_t best = 0u;
            int at = 0;
#pragma unroll
            for (int i = 0; i < MOE_MAX_EXPERTS / 32; ++i)
                if (left[i] > best) { best = left[i]; at = lane + 32 * i; }
            const uint32_t most = __reduce_max_sync(0xFFFFFFFFu, best);
            const int expert = (int)__reduce_min_sync(0xFFFFFFFFu, best == most ? (uint32_t)at : 0xFFFFu);
            if (j == 0) {
                top = most;
                if (!a.renormalize && top != 0u) {
#pragma unroll
                    for (int i = 0; i < MOE_MAX_EXPERTS / 32; ++i)
                        if (left[i] != 0u) total += share_of(left[i], top);
#pragma unroll
                    for (int off = 16; off > 0; off >>= 1) total += __shfl_xor_sync(0xFFFFFFFFu, total, off);
                }
            }
            const float share = most != 0u ? share_of(most, top) : 0.f;
            if (a.renormalize) total += share;
            if (lane == j) {
                mine = share;
                choice.expert[t * a.top_k + j] = (short)(most != 0u ? expert : -1);
                if (most != 0u) atomicOr(&choice.used[expert >> 5], 1u << (expert & 31));
            }
#pragma unroll
            for (int i = 0; i < MOE_MAX_EXPERTS / 32; ++i)
                if (most != 0u && lane + 32 * i == expert) left[i] = 0u;
        }
        if (lane < a.top_k) choice.weight[t * a.top_k + lane] = mine > 0.f ? mine / total : 0.f;
    }
    __syncthreads();
}

// The u-th used expert, or -1.
__device__ __forceinline__ int used_expert(const Choice& choice, int u)
{
    for (int w = 0; w < MOE_MAX_EXPERTS / 32; ++w) {
        uint32_t bits = choice.used[w];
        const int n = __popc(bits);
        if (u < n) {
            for (; u > 0; --u) bits &= bits - 1u;
            return 32 * w + __ffs(bits) - 1;
        }
        u -= n;
    }
    return -1;
}

// The slots that chose an expert, ascending, by one warp; returns their number.
__device__ __forceinline__ int slots_of(const MoeArgs& a, const Choice& choice, int expert, short* list)
{
    const int lane = threadIdx.x & 31, slots = a.tokens * a.top_k;
    int found = 0;
    for (int base = 0; base < slots; base += 32) {
        const bool hit = base + lane < slots && choice.expert[base + lane] == expert;
        const unsigned hits = __ballot_sync(0xFFFFFFFFu, hit);
        if (hit) list[found + __popc(hits & ((1u << lane) - 1u))] = (short)(base + lane);
        found += __popc(hits);
    }
    __syncwarp();
    return found;
}

__device__ __forceinline__ float activate(float x, int act)
{
    switch (act) {
        case MXFP8_ACT_RELU: return x > 0.f ? x : 0.f;
        case MXFP8_ACT_RELU2: return x > 0.f ? x * x : 0.f;
        case MXFP8_ACT_SILU: return __fdividef(x, 1.f + __expf(-x));
        case MXFP8_ACT_GELU_TANH: return __fdividef(x, 1.f + __expf(-1.5957691216057308f * (x + 0.044715f * x * x * x)));
        default: return x;
    }
}

// Products of one warp's column tiles (every `step`-th from `first`) with R row tiles, for up to 8 NT rows of `from`.
template <int R, int NT>
__device__ __forceinline__ void run_products(const uint8_t* const (&tile)[R], const __nv_bfloat16* const (&from)[NT], const bool (&has)[NT],
                                             int cols, int col_tiles, int first, int step, float (&acc)[R][NT][4])
{
    const int lane = threadIdx.x & 31, quarter = lane & 3;
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[r][t][i] = 0.f;
    for (int kt = first; kt < col_tiles; kt += step) {
        Operands<R, NT> o;
        bool none[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) none[t] = false;
        o.load(tile, (int64_t)kt * TILE_BYTES, from, none, 0, lane);
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int k = kt * TILE_COLS + g * 32;                  // columns behind the matrix are zeros
                o.x[t][g] = has[t] && k < cols ? *reinterpret_cast<const uint4*>(from[t] + k + quarter * 8) : make_uint4(0u, 0u, 0u, 0u);
            }
        product<R, NT>(o, acc);
    }
}

// CTA (p, u): rows 16 p .. of the gate and of the up projection of the u-th used expert.  Eight warps split the columns.
__global__ void __launch_bounds__(MOE_THREADS) moe_gate_up_kernel(const MoeArgs a)
{
    __shared__ Choice choice;
    __shared__ short list[MOE_MAX_TOKENS];
    __shared__ int listed;
    __shared__ float sums[MOE_WARPS][2][TILE_ROWS][9];
    choose(a, choice);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (blockIdx.x == 0 && blockIdx.y == 0)
        for (int s = tid; s < a.tokens * a.top_k; s += MOE_THREADS) {
            if (a.ids) a.ids[s] = choice.expert[s];
            if (a.weights) a.weights[s] = choice.weight[s];
        }
    const int expert = used_expert(choice, blockIdx.y);
    if (expert < 0) return;
    if (warp == 0) {
        const int n = slots_of(a, choice, expert, list);
        if (lane == 0) listed = n;
    }
    __syncthreads();
    const int pairs = a.inner / TILE_ROWS, count = listed;
    const uint8_t* matrix = a.gate_up + (int64_t)expert * 2 * pairs * a.col_tiles * TILE_BYTES + lane * 16;
    const uint8_t* tile[2] = {matrix + (int64_t)blockIdx.x * a.col_tiles * TILE_BYTES, matrix + (int64_t)(pairs + blockIdx.x) * a.col_tiles * TILE_BYTES};
    for (int s0 = 0; s0 < count; s0 += 8) {
        const bool has[1] = {s0 + (lane >> 2) < count};
        const __nv_bfloat16* from[1] = {a.x + (int64_t)(has[0] ? list[s0 + (lane >> 2)] / a.top_k : 0) * a.cols};
        float acc[2][1][4];
        run_products<2, 1>(tile, from, has, a.cols, a.col_tiles, warp, MOE_WARPS, acc);
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
            for (int i = 0; i < 4; ++i) sums[warp][r][(lane >> 2) + 8 * (i >> 1)][2 * (lane & 3) + (i & 1)] = acc[r][0][i];
        __syncthreads();
        if (tid < 8 * TILE_ROWS && s0 + (tid >> 4) < count) {
            const int n = tid & 15, s = tid >> 4;
            float g = 0.f, u = 0.f;
            for (int w = 0; w < MOE_WARPS; ++w) {
                g += sums[w][0][n][s];
                u += sums[w][1][n][s];
            }
            const float m = activate(g, a.act) * u;
            const __nv_bfloat16 hi = __float2bfloat16_rn(m);
            const int64_t at = (int64_t)list[s0 + s] * a.inner + blockIdx.x * TILE_ROWS + n;
            a.m_hi[at] = hi;
            a.m_lo[at] = __float2bfloat16_rn(m - __bfloat162float(hi));
        }
        __syncthreads();
    }
}

// CTA p: rows 16 p .. of all used experts' down projections.  The warps split the columns; each holds the weighted sums of its
// share for all tokens, and they are added at the end.
__global__ void __launch_bounds__(MOE_THREADS) moe_down_kernel(const MoeArgs a)
{
    extern __shared__ float total[];                     // [warp][token][row], rows padded to 17
    __shared__ Choice choice;
    __shared__ short list[MOE_WARPS][MOE_MAX_TOKENS];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    for (int i = tid; i < MOE_WARPS * a.tokens * 17; i += MOE_THREADS) total[i] = 0.f;
    choose(a, choice);
    float* mine = total + warp * a.tokens * 17;
    const int row_tiles = (a.cols + TILE_ROWS - 1) / TILE_ROWS;
    for (int w = 0; w < MOE_MAX_EXPERTS / 32; ++w)
        for (uint32_t bits = choice.used[w]; bits != 0u; bits &= bits - 1u) {
            const int expert = 32 * w + __ffs(bits) - 1;
            const int count = slots_of(a, choice, expert, list[warp]);
            const uint8_t* tile[1] = {a.down + ((int64_t)expert * row_tiles + blockIdx.x) * a.inner_tiles * TILE_BYTES + lane * 16};
            for (int s0 = 0; s0 < count; s0 += 8) {
                const bool in = s0 + (lane >> 2) < count, has[2] = {in, in};
                const int64_t at = (int64_t)(in ? list[warp][s0 + (lane >> 2)] : 0) * a.inner;
                const __nv_bfloat16* from[2] = {a.m_hi + at, a.m_lo + at};
                float acc[1][2][4];
                run_products<1, 2>(tile, from, has, a.inner, a.inner_tiles, warp, MOE_WARPS, acc);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int s = s0 + 2 * (lane & 3) + (i & 1);
                    if (s < count) {
                        float* to = mine + list[warp][s] / a.top_k * 17 + (lane >> 2) + 8 * (i >> 1);
                        *to = fmaf(choice.weight[list[warp][s]], acc[0][0][i] + acc[0][1][i], *to);
                    }
                }
                __syncwarp();
            }
        }
    __syncthreads();
    for (int i = tid; i < a.tokens * TILE_ROWS; i += MOE_THREADS) {
        const int n = i & 15, t = i >> 4, row = blockIdx.x * TILE_ROWS + n;
        float v = 0.f;
        for (int w = 0; w < MOE_WARPS; ++w) v += total[(w * a.tokens + t) * 17 + n];
        if (a.bf16_out) static_cast<__nv_bfloat16*>(a.y)[(int64_t)t * a.cols + row] = __float2bfloat16_rn(v);
        else static_cast<float*>(a.y)[(int64_t)t * a.cols + row] = v;
    }
}

}  // namespace
}  // namespace mxfp8

using namespace mxfp8;

extern "C" size_t mxfp8_e2m1_moe_ws_bytes(int64_t tokens, int top_k, int64_t inner)
{
    if (tokens <= 0 || top_k <= 0 || inner <= 0 || tokens > MOE_MAX_TOKENS || top_k > MOE_MAX_TOP_K) return 0;
    return (size_t)tokens * top_k * (size_t)inner * 2 * sizeof(__nv_bfloat16);
}

extern "C" int mxfp8_e2m1_moe(const void* x, const float* logits, int64_t tokens, int64_t cols, int num_experts, int top_k,
                              const void* gate_up, const void* down, int64_t inner, int act, int renormalize,
                              void* y, int y_dtype, int32_t* ids, float* weights, void* ws, size_t ws_bytes, void* stream)
{
    if (y_dtype != MXFP8_FP32 && y_dtype != MXFP8_BF16) return MXFP8_ERR_ENUM;
    if (act < MXFP8_ACT_NONE || act > MXFP8_ACT_GELU_TANH) return MXFP8_ERR_ENUM;
    if (!x || !logits || !gate_up || !down || !y) return MXFP8_ERR_NULL;
    if (tokens <= 0 || cols <= 0 || inner <= 0 || (cols % 32) || (inner % 32) || num_experts < 1 || top_k < 1 || top_k > num_experts) return MXFP8_ERR_SHAPE;
    if (!aligned16(x) || !aligned16(gate_up) || !aligned16(down)) return MXFP8_ERR_ALIGN;
    if ((reinterpret_cast<uintptr_t>(y) % (y_dtype == MXFP8_BF16 ? 2 : 4)) || (reinterpret_cast<uintptr_t>(logits) & 3u) ||
        (reinterpret_cast<uintptr_t>(ids) & 3u) || (reinterpret_cast<uintptr_t>(weights) & 3u)) return MXFP8_ERR_ALIGN;
    if (tokens > MOE_MAX_TOKENS || num_experts > MOE_MAX_EXPERTS || top_k > MOE_MAX_TOP_K || cols > (1 << 20) || inner > (1 << 20)) return MXFP8_ERR_UNSUPPORTED;
    if (!ws || ws_bytes < mxfp8_e2m1_moe_ws_bytes(tokens, top_k, inner)) return MXFP8_ERR_WORKSPACE;
    if (!aligned16(ws)) return MXFP8_ERR_ALIGN;
    MoeArgs a{};
    a.x = static_cast<const __nv_bfloat16*>(x);
    a.logits = logits;
    a.gate_up = static_cast<const uint8_t*>(gate_up); a.down = static_cast<const uint8_t*>(down);
    a.y = y; a.bf16_out = y_dtype == MXFP8_BF16; a.ids = ids; a.weights = weights;
    a.m_hi = static_cast<__nv_bfloat16*>(ws); a.m_lo = a.m_hi + tokens * top_k * inner;
    a.tokens = (int)tokens; a.experts = num_experts; a.top_k = top_k; a.act = act; a.renormalize = renormalize != 0;
    a.cols = (int)cols; a.inner = (int)inner;
    a.col_tiles = (int)((cols + TILE_COLS - 1) / TILE_COLS); a.inner_tiles = (int)((inner + TILE_COLS - 1) / TILE_COLS);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const int slots = a.tokens * a.top_k;
    moe_gate_up_kernel<<<dim3((unsigned)(inner / TILE_ROWS), (unsigned)(slots < num_experts ? slots : num_experts)), MOE_THREADS, 0, st>>>(a);
    count_launch(1);
    if (cudaGetLastError() != cudaSuccess) return MXFP8_ERR_CUDA;
    moe_down_kernel<<<(unsigned)(cols / TILE_ROWS), MOE_THREADS, MOE_WARPS * a.tokens * 17 * sizeof(float), st>>>(a);
    count_launch(1);
    return cudaGetLastError() == cudaSuccess ? MXFP8_OK : MXFP8_ERR_CUDA;
}
