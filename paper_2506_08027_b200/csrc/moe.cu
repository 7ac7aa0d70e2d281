// Mixture-of-experts token movement around mxfp8_grouped_gemm (App. A.4): sorting the routed tokens by expert into
// segments that start at multiples of 128 rows, gathering the experts' outputs back with the router's weights, and the
// gradient of that sum.  (The gather into the sorted order is fused with the conversion: quantize_tma_kernel.cuh.)
//
// A slot is one (token, choice) pair, numbered token * top_k + choice.
#include "mxfp8_device.cuh"
#include "mxfp8_host.h"

namespace mxfp8 {
namespace {

// ------------------------------------------------------------------------------------------------------------ sorting
constexpr int SORT_MAX_EXPERTS = 256;
constexpr int SORT_THREADS = 1024;
constexpr int SORT_WARPS = SORT_THREADS / 32;
constexpr int SORT_PAD = 128;                 // rows of a scale atom: what grouped products ask of a segment's start
constexpr int SORT_MAX_CHUNKS = 148;          // one CTA per multiprocessor
constexpr int SORT_ONE_CTA_SLOTS = 4096;      // up to here one CTA sorts alone

struct SortArgs {
    const int32_t* ids;
    int32_t* offsets;
    int32_t* row_of;
    int32_t* slot_of;
    int32_t* counts;        // [chunks][experts] slots of every expert in every chunk; null when one CTA holds all slots
    int slots, experts, rows, chunk;
};

// Slots of every expert in one chunk of consecutive slots (first of two launches; integer sums, so their order is free).
__global__ void __launch_bounds__(SORT_THREADS) moe_sort_count_kernel(const SortArgs a)
{
    __shared__ int hist[SORT_MAX_EXPERTS];
    for (int e = threadIdx.x; e < a.experts; e += SORT_THREADS) hist[e] = 0;
    __syncthreads();
    const int first = blockIdx.x * a.chunk, last = min(first + a.chunk, a.slots);
    for (int s = first + (int)threadIdx.x; s < last; s += SORT_THREADS) {
        const int id = a.ids[s];
        if ((unsigned)id < (unsigned)a.experts) atomicAdd(&hist[id], 1);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < a.experts; e += SORT_THREADS) a.counts[blockIdx.x * a.experts + e] = hist[e];
}

// Stable counting sort of the slots by expert.  Every warp owns a run of consecutive slots: it counts them per expert
// (shared memory), the counts are summed over the warps before it and, through `counts`, over the chunks before its
// own, the experts' totals rounded up to 128 give the segment starts, and a second walk over the run hands out rows in
// slot order: within 32 slots the rank among equal experts is a population count of the match mask.  No atomic decides
// an order, so the result is the stable sort, the same every time.
__global__ void __launch_bounds__(SORT_THREADS) moe_sort_kernel(const SortArgs a)
{
    __shared__ int hist[SORT_WARPS][SORT_MAX_EXPERTS];     // counts, then the next free rank of (warp, expert)
    __shared__ int total[SORT_MAX_EXPERTS];                // slots of the expert in all chunks
    __shared__ int before[4][SORT_MAX_EXPERTS];            // ... in the chunks before this one (four partial sums)
    __shared__ int part[4][SORT_MAX_EXPERTS];
    __shared__ int start[SORT_MAX_EXPERTS + 1];            // segment starts
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, E = a.experts;
    const int first = blockIdx.x * a.chunk, last = min(first + a.chunk, a.slots);
    const int run = ((last - first + SORT_THREADS - 1) / SORT_THREADS) * 32;       // slots of a warp, whole groups of 32
    const int w_first = min(first + warp * run, last), w_last = min(w_first + run, last);

    for (int i = tid; i < SORT_WARPS * SORT_MAX_EXPERTS; i += SORT_THREADS) (&hist[0][0])[i] = 0;
    __syncthreads();
    for (int s = w_first + lane; s < w_last; s += 32) {
        const int id = a.ids[s];
        if ((unsigned)id < (unsigned)E) atomicAdd(&hist[warp][id], 1);
    }
    __syncthreads();
    if (a.counts != nullptr) {
        const int e = tid & (SORT_MAX_EXPERTS - 1), quarter = tid / SORT_MAX_EXPERTS;
        int sum = 0, sum_before = 0;
        if (e < E)
#pragma unroll 8
            for (int c = quarter; c < (int)gridDim.x; c += 4) {
                const int v = a.counts[c * E + e];
                sum += v;
                sum_before += c < (int)blockIdx.x ? v : 0;
            }
        part[quarter][e] = sum;
        before[quarter][e] = sum_before;
    }
    __syncthreads();
    if (tid < E) {
        int acc = 0;
        if (a.counts != nullptr) {
            acc = before[0][tid] + before[1][tid] + before[2][tid] + before[3][tid];
            total[tid] = part[0][tid] + part[1][tid] + part[2][tid] + part[3][tid];
        }
#pragma unroll 8
        for (int w = 0; w < SORT_WARPS; ++w) {             // first rank of every warp's run within the expert
            const int v = hist[w][tid];
            hist[w][tid] = acc;
            acc += v;
        }
        if (a.counts == nullptr) total[tid] = acc;
    }
    __syncthreads();
    if (warp == 0) {                                       // exclusive sum of the padded totals, eight experts per lane
        int mine[8], sum = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int e = lane * 8 + i;
            mine[i] = e < E ? (total[e] + SORT_PAD - 1) / SORT_PAD * SORT_PAD : 0;
            sum += mine[i];
        }
        int incl = sum;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const int v = __shfl_up_sync(0xFFFFFFFFu, incl, off);
            if (lane >= off) incl += v;
        }
        int at = incl - sum;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int e = lane * 8 + i;
            if (e <= E) start[e] = at;
            at += mine[i];
        }
        if (lane == 31 && E == SORT_MAX_EXPERTS) start[E] = at;
    }
    __syncthreads();
    if (blockIdx.x == 0)
        for (int e = tid; e <= E; e += SORT_THREADS) a.offsets[e] = start[e];
    for (int base = w_first; base < w_last; base += 32) {
        const int s = base + lane;
        int id = s < w_last ? a.ids[s] : -1;
        if ((unsigned)id >= (unsigned)E) id = -1;
        const unsigned same = __match_any_sync(0xFFFFFFFFu, id);
        const int rank = __popc(same & ((1u << lane) - 1u));
        int row = -1;
        if (id >= 0) row = start[id] + hist[warp][id] + rank;
        __syncwarp();
        if (id >= 0 && rank == 0) hist[warp][id] += __popc(same);
        __syncwarp();
        if (s < w_last) {
            a.row_of[s] = row;
            if (row >= 0) a.slot_of[row] = s;
        }
    }
    // rows without a slot: the padding behind every expert, and everything behind the last segment
    for (int e = (int)blockIdx.x * 8 + (tid >> 7); e < E; e += (int)gridDim.x * 8) {
        const int row = start[e] + total[e] + (tid & 127);
        if (row < start[e + 1]) a.slot_of[row] = -1;
    }
    for (int row = start[E] + (int)(blockIdx.x * SORT_THREADS + tid); row < a.rows; row += (int)gridDim.x * SORT_THREADS) a.slot_of[row] = -1;
}

// Slots per CTA: all of them in one CTA while they are few, else chunks of whole 1024s over at most one CTA per SM.
int sort_chunk(int64_t slots)
{
    if (slots <= SORT_ONE_CTA_SLOTS) return SORT_ONE_CTA_SLOTS;
    const int64_t per = (slots + SORT_MAX_CHUNKS - 1) / SORT_MAX_CHUNKS;
    return (int)((per + SORT_THREADS - 1) / SORT_THREADS * SORT_THREADS);
}

// -------------------------------------------------------------------------------------------- gather, weight, sum
// V consecutive elements of a row as they lie in memory, read and written in pieces of up to 16 bytes.
template <int BYTES> struct Piece { using type = uint4; };
template <> struct Piece<8> { using type = uint2; };
template <> struct Piece<4> { using type = uint32_t; };
template <> struct Piece<2> { using type = uint16_t; };
template <int DTYPE, int V> struct Vec {
    static constexpr int ESZ = (DTYPE == MXFP8_BF16) ? 2 : 4;
    static constexpr int BYTES = V * ESZ;
    using P = typename Piece<(BYTES < 16 ? BYTES : 16)>::type;
    static constexpr int N = BYTES / (int)sizeof(P);
    P piece[N];
    __device__ __forceinline__ void load(const void* base, int64_t element)
    {
        const P* p = reinterpret_cast<const P*>(static_cast<const uint8_t*>(base) + element * ESZ);
#pragma unroll
        for (int i = 0; i < N; ++i) piece[i] = p[i];
    }
    __device__ __forceinline__ void store(void* base, int64_t element) const
    {
        P* p = reinterpret_cast<P*>(static_cast<uint8_t*>(base) + element * ESZ);
#pragma unroll
        for (int i = 0; i < N; ++i) p[i] = piece[i];
    }
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int i = 0; i < N; ++i) piece[i] = P{};
    }
    __device__ __forceinline__ float get(int i) const
    {
        if constexpr (DTYPE == MXFP8_BF16) {
            const uint32_t h = reinterpret_cast<const uint16_t*>(piece)[i];
            return __uint_as_float(h << 16);
        } else return reinterpret_cast<const float*>(piece)[i];
    }
    __device__ __forceinline__ void set(int i, float x)      // one rounding to nearest even for BF16
    {
        if constexpr (DTYPE == MXFP8_BF16) reinterpret_cast<__nv_bfloat16*>(piece)[i] = __float2bfloat16_rn(x);
        else reinterpret_cast<float*>(piece)[i] = x;
    }
};

struct MoveArgs {
    const void* src;          // [rows, cols] in sorted order
    const void* dy;           // [tokens, cols] (gradient)
    const int32_t* row_of;    // [tokens, top_k]
    const int32_t* slot_of;   // [rows] (gradient)
    const float* weights;     // [tokens, top_k] or null
    const int32_t* used;      // device: rows in use (gradient)
    void* dst;                // [tokens, cols]; gradient: [rows, cols]
    float* d_weights;         // gradient
    int* status;
    int64_t rows, cols, tokens;
    int64_t token_blocks;     // gradient: CTAs that walk tokens; those behind them clear padding rows
    int top_k, group;         // group: threads that share a token (a power of two, 32 .. 256)
};

constexpr int MOVE_THREADS = 256;
constexpr int MOVE_UNROLL = 8;        // rows in flight per thread

// Row of a slot, or -1.  Anything but -1 and a row of the tensor is an error of the caller's array: reported, not used.
__device__ __forceinline__ int64_t checked_row(int32_t r, int64_t rows, int* status)
{
    if (r >= 0 && r < rows) return r;
    if (r != -1) atomicExch(status, (int)MXFP8_ERR_DEVICE_ARGS);
    return -1;
}

// dst[t, c] = sum_j w[t, j] * src[row_of[t, j], c]: FP32 sums in the order of j, one rounding at the end.
template <int SRC, int DST, int V>
__global__ void __launch_bounds__(MOVE_THREADS) moe_combine_kernel(const MoveArgs a)
{
    const int per_block = MOVE_THREADS / a.group;
    const int64_t t = (int64_t)blockIdx.x * per_block + threadIdx.x / a.group;
    const int64_t c = ((int64_t)blockIdx.y * a.group + threadIdx.x % a.group) * V;
    if (t >= a.tokens || c >= a.cols) return;
    float acc[V];
#pragma unroll
    for (int i = 0; i < V; ++i) acc[i] = 0.f;
    for (int j0 = 0; j0 < a.top_k; j0 += MOVE_UNROLL) {
        Vec<SRC, V> x[MOVE_UNROLL];
        float w[MOVE_UNROLL];
        bool live[MOVE_UNROLL];
#pragma unroll
        for (int j = 0; j < MOVE_UNROLL; ++j) {
            live[j] = false;
            if (j0 + j < a.top_k) {
                const int64_t slot = t * a.top_k + j0 + j;
                const int64_t r = checked_row(a.row_of[slot], a.rows, a.status);
                live[j] = r >= 0;
                if (live[j]) {
                    w[j] = a.weights ? a.weights[slot] : 1.f;
                    x[j].load(a.src, r * a.cols + c);
                }
            }
        }
#pragma unroll
        for (int j = 0; j < MOVE_UNROLL; ++j)
            if (live[j])
#pragma unroll
                for (int i = 0; i < V; ++i) acc[i] = fmaf(w[j], x[j].get(i), acc[i]);
    }
    Vec<DST, V> y;
#pragma unroll
    for (int i = 0; i < V; ++i) y.set(i, acc[i]);
    y.store(a.dst, t * a.cols + c);
}

// d_src[row_of[t, j], c] = w[t, j] * dy[t, c] (one FP32 product, rounded to src's type) and
// d_weights[t, j] = sum_c dy[t, c] * src[row_of[t, j], c] (FP32: lane-strided partial sums, then a fixed tree), so dy is
// read once per token.  CTAs behind the tokens' clear the padding rows of the segments.
template <int DY, int SRC, int V>
__global__ void __launch_bounds__(MOVE_THREADS) moe_combine_grad_kernel(const MoveArgs a)
{
    __shared__ float sums[MOVE_THREADS / 32][MOVE_UNROLL];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if ((int64_t)blockIdx.x >= a.token_blocks) {
        const int used = *a.used;
        if (used < 0 || used > a.rows) {
            if (tid == 0) atomicExch(a.status, (int)MXFP8_ERR_DEVICE_ARGS);
            return;
        }
        const int64_t row0 = ((int64_t)blockIdx.x - a.token_blocks) * 32 + warp * 4;
        for (int64_t r = row0; r < row0 + 4 && r < used; ++r) {
            if (a.slot_of[r] >= 0) continue;
            Vec<SRC, V> z;
            z.zero();
            for (int64_t c = (int64_t)lane * V; c < a.cols; c += 32 * V) z.store(a.dst, r * a.cols + c);
        }
        return;
    }
    const int per_block = MOVE_THREADS / a.group, member = tid % a.group;
    const int64_t t = (int64_t)blockIdx.x * per_block + tid / a.group;
    for (int j0 = 0; j0 < a.top_k; j0 += MOVE_UNROLL) {
        int64_t row[MOVE_UNROLL];
        float w[MOVE_UNROLL], acc[MOVE_UNROLL];
#pragma unroll
        for (int j = 0; j < MOVE_UNROLL; ++j) {
            acc[j] = 0.f;
            row[j] = -1;
            w[j] = 0.f;
            if (t < a.tokens && j0 + j < a.top_k) {
                const int64_t slot = t * a.top_k + j0 + j;
                row[j] = checked_row(a.row_of[slot], a.rows, a.status);
                w[j] = a.weights ? a.weights[slot] : 1.f;
            }
        }
        if (t < a.tokens)
            for (int64_t c = (int64_t)member * V; c < a.cols; c += (int64_t)a.group * V) {
                Vec<DY, V> g;
                g.load(a.dy, t * a.cols + c);
                Vec<SRC, V> x[MOVE_UNROLL];
                if (a.d_weights != nullptr)
#pragma unroll
                    for (int j = 0; j < MOVE_UNROLL; ++j)
                        if (row[j] >= 0) x[j].load(a.src, row[j] * a.cols + c);
#pragma unroll
                for (int j = 0; j < MOVE_UNROLL; ++j) {
                    if (row[j] < 0) continue;
                    if (a.d_weights != nullptr)
#pragma unroll
                        for (int i = 0; i < V; ++i) acc[j] = fmaf(g.get(i), x[j].get(i), acc[j]);
                    if (a.dst != nullptr) {
                        Vec<SRC, V> d;
#pragma unroll
                        for (int i = 0; i < V; ++i) d.set(i, w[j] * g.get(i));
                        d.store(a.dst, row[j] * a.cols + c);
                    }
                }
            }
        if (a.d_weights == nullptr) continue;
#pragma unroll
        for (int j = 0; j < MOVE_UNROLL; ++j)
#pragma unroll
            for (int off = 16; off > 0; off >>= 1) acc[j] += __shfl_xor_sync(0xFFFFFFFFu, acc[j], off);
        if (lane == 0)
#pragma unroll
            for (int j = 0; j < MOVE_UNROLL; ++j) sums[warp][j] = acc[j];
        __syncthreads();
        if (member < MOVE_UNROLL && t < a.tokens && j0 + member < a.top_k) {
            const int w0 = (tid / a.group) * (a.group / 32);
            float s = 0.f;
            for (int k = 0; k < a.group / 32; ++k) s += sums[w0 + k][member];
            a.d_weights[t * a.top_k + j0 + member] = s;
        }
        __syncthreads();
    }
}

// Largest vector (8, 4, 2 or 1 elements) that every row of every tensor starts on: it has to divide cols, and each base
// has to lie on a boundary of its pieces.
int vector_width(int64_t cols, const void* const* ptrs, const int* esz, int count)
{
    for (int v = 8; v > 1; v >>= 1) {
        bool ok = cols % v == 0;
        for (int i = 0; ok && i < count; ++i) {
            const int bytes = v * esz[i] < 16 ? v * esz[i] : 16;
            ok = (reinterpret_cast<uintptr_t>(ptrs[i]) % bytes) == 0;
        }
        if (ok) return v;
    }
    return 1;
}

int group_threads(int64_t vectors)
{
    int g = 32;
    while (g < MOVE_THREADS && g < vectors) g <<= 1;
    return g;
}

}  // namespace
}  // namespace mxfp8

using namespace mxfp8;

extern "C" int64_t mxfp8_moe_rows(int64_t tokens, int top_k, int num_experts)
{
    if (tokens <= 0 || top_k <= 0 || num_experts <= 0 || tokens > 0x7FFFFFFFLL) return 0;
    const int64_t slots = tokens * top_k;
    return (slots + (SORT_PAD - 1) * (slots < num_experts ? slots : num_experts)) / SORT_PAD * SORT_PAD;
}

extern "C" size_t mxfp8_moe_sort_ws_bytes(int64_t tokens, int top_k, int num_experts)
{
    if (tokens <= 0 || top_k <= 0 || num_experts <= 0 || tokens > 0x7FFFFFFFLL) return 0;
    const int64_t slots = tokens * top_k;
    if (slots > 0x7F000000LL || slots <= SORT_ONE_CTA_SLOTS) return 0;
    const int chunk = sort_chunk(slots);
    return (size_t)((slots + chunk - 1) / chunk) * num_experts * sizeof(int32_t);
}

extern "C" int mxfp8_moe_sort(const int32_t* expert_ids, int64_t tokens, int top_k, int num_experts,
                              int32_t* group_offsets, int32_t* row_of, int32_t* slot_of, int64_t rows,
                              void* ws, size_t ws_bytes, void* stream)
{
    if (tokens < 0 || top_k < 1 || num_experts < 1 || rows < 0) return MXFP8_ERR_SHAPE;
    if (!group_offsets || (tokens > 0 && (!expert_ids || !row_of)) || (rows > 0 && !slot_of)) return MXFP8_ERR_NULL;
    if (num_experts > SORT_MAX_EXPERTS || tokens > 0x7F000000LL || tokens * top_k > 0x7F000000LL || rows > 0x7FFFFFFFLL) return MXFP8_ERR_UNSUPPORTED;
    if (rows < mxfp8_moe_rows(tokens, top_k, num_experts)) return MXFP8_ERR_SHAPE;
    for (const void* p : {(const void*)expert_ids, (const void*)group_offsets, (const void*)row_of, (const void*)slot_of, (const void*)ws})
        if (reinterpret_cast<uintptr_t>(p) & 3u) return MXFP8_ERR_ALIGN;
    const size_t need = mxfp8_moe_sort_ws_bytes(tokens, top_k, num_experts);
    if (need > 0 && (!ws || ws_bytes < need)) return MXFP8_ERR_WORKSPACE;
    SortArgs a{};
    a.ids = expert_ids; a.offsets = group_offsets; a.row_of = row_of; a.slot_of = slot_of;
    a.slots = (int)(tokens * top_k); a.experts = num_experts; a.rows = (int)rows;
    a.chunk = sort_chunk(a.slots);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (need == 0) {
        moe_sort_kernel<<<1, SORT_THREADS, 0, st>>>(a);
        count_launch(1);
    } else {
        a.counts = static_cast<int32_t*>(ws);
        const int chunks = (a.slots + a.chunk - 1) / a.chunk;
        moe_sort_count_kernel<<<chunks, SORT_THREADS, 0, st>>>(a);
        moe_sort_kernel<<<chunks, SORT_THREADS, 0, st>>>(a);
        count_launch(2);
    }
    return cudaGetLastError() == cudaSuccess ? MXFP8_OK : MXFP8_ERR_CUDA;
}

namespace {
template <int A, int B>
cudaError_t launch_combine(int v, dim3 grid, const MoveArgs& m, cudaStream_t st)
{
    if (v == 8) moe_combine_kernel<A, B, 8><<<grid, MOVE_THREADS, 0, st>>>(m);
    else if (v == 4) moe_combine_kernel<A, B, 4><<<grid, MOVE_THREADS, 0, st>>>(m);
    else if (v == 2) moe_combine_kernel<A, B, 2><<<grid, MOVE_THREADS, 0, st>>>(m);
    else moe_combine_kernel<A, B, 1><<<grid, MOVE_THREADS, 0, st>>>(m);
    count_launch(1);
    return cudaGetLastError();
}
template <int A, int B>
cudaError_t launch_grad(int v, unsigned grid, const MoveArgs& m, cudaStream_t st)
{
    if (v == 8) moe_combine_grad_kernel<A, B, 8><<<grid, MOVE_THREADS, 0, st>>>(m);
    else if (v == 4) moe_combine_grad_kernel<A, B, 4><<<grid, MOVE_THREADS, 0, st>>>(m);
    else if (v == 2) moe_combine_grad_kernel<A, B, 2><<<grid, MOVE_THREADS, 0, st>>>(m);
    else moe_combine_grad_kernel<A, B, 1><<<grid, MOVE_THREADS, 0, st>>>(m);
    count_launch(1);
    return cudaGetLastError();
}
bool misaligned(const void* p, int bytes) { return (reinterpret_cast<uintptr_t>(p) % bytes) != 0; }
bool bad_dtype(int d) { return d != MXFP8_FP32 && d != MXFP8_BF16; }
int esize(int d) { return d == MXFP8_BF16 ? 2 : 4; }
}  // namespace

extern "C" int mxfp8_moe_combine(const void* src, int src_dtype, int64_t rows, int64_t cols, const int32_t* row_of,
                                 const float* weights, int64_t tokens, int top_k, void* dst, int dst_dtype, void* stream)
{
    if (bad_dtype(src_dtype) || bad_dtype(dst_dtype)) return MXFP8_ERR_ENUM;
    if (rows < 0 || cols <= 0 || tokens < 0 || top_k < 1) return MXFP8_ERR_SHAPE;
    if (tokens == 0) return MXFP8_OK;
    if ((rows > 0 && !src) || !row_of || !dst) return MXFP8_ERR_NULL;
    if (misaligned(src, esize(src_dtype)) || misaligned(dst, esize(dst_dtype)) || misaligned(row_of, 4) || misaligned(weights, 4)) return MXFP8_ERR_ALIGN;
    MoveArgs m{};
    m.src = src; m.row_of = row_of; m.weights = weights; m.dst = dst;
    m.rows = rows; m.cols = cols; m.tokens = tokens; m.top_k = top_k;
    const void* ptrs[2] = {src, dst};
    const int esz[2] = {esize(src_dtype), esize(dst_dtype)};
    const int v = vector_width(cols, ptrs, esz, 2);
    m.group = group_threads(cols / v);
    const int64_t gx = (tokens + MOVE_THREADS / m.group - 1) / (MOVE_THREADS / m.group), gy = (cols / v + m.group - 1) / m.group;
    if (gx > 0x7FFFFFFFLL || gy > 65535 || tokens > 0x7FFFFFFFFFFFLL / top_k) return MXFP8_ERR_UNSUPPORTED;
    if (!(m.status = device_status_word())) return MXFP8_ERR_CUDA;
    const dim3 grid((unsigned)gx, (unsigned)gy);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t err;
    if (src_dtype == MXFP8_BF16) err = dst_dtype == MXFP8_BF16 ? launch_combine<MXFP8_BF16, MXFP8_BF16>(v, grid, m, st) : launch_combine<MXFP8_BF16, MXFP8_FP32>(v, grid, m, st);
    else err = dst_dtype == MXFP8_BF16 ? launch_combine<MXFP8_FP32, MXFP8_BF16>(v, grid, m, st) : launch_combine<MXFP8_FP32, MXFP8_FP32>(v, grid, m, st);
    return err == cudaSuccess ? MXFP8_OK : MXFP8_ERR_CUDA;
}

extern "C" int mxfp8_moe_combine_grad(const void* dy, int dy_dtype, int64_t tokens, int64_t cols, const void* src, int src_dtype, int64_t rows,
                                      const int32_t* row_of, const int32_t* slot_of, int top_k, const float* weights,
                                      const int32_t* group_offsets, int num_groups, void* d_src, float* d_weights, void* stream)
{
    if (bad_dtype(dy_dtype) || bad_dtype(src_dtype)) return MXFP8_ERR_ENUM;
    if (rows < 0 || cols <= 0 || tokens < 0 || top_k < 1 || num_groups < 1) return MXFP8_ERR_SHAPE;
    if (tokens == 0) return MXFP8_OK;
    if (!dy || !row_of || (!d_src && !d_weights)) return MXFP8_ERR_NULL;
    if ((d_weights && rows > 0 && !src) || (d_src && rows > 0 && (!slot_of || !group_offsets))) return MXFP8_ERR_NULL;
    if (misaligned(dy, esize(dy_dtype)) || misaligned(src, esize(src_dtype)) || misaligned(d_src, esize(src_dtype)) || misaligned(row_of, 4) ||
        misaligned(slot_of, 4) || misaligned(weights, 4) || misaligned(group_offsets, 4) || misaligned(d_weights, 4))
        return MXFP8_ERR_ALIGN;
    MoveArgs m{};
    m.src = src; m.dy = dy; m.row_of = row_of; m.slot_of = slot_of; m.weights = weights; m.dst = d_src; m.d_weights = d_weights;
    m.rows = rows; m.cols = cols; m.tokens = tokens; m.top_k = top_k;
    m.used = group_offsets ? group_offsets + num_groups : nullptr;
    const void* ptrs[3] = {dy, src, d_src};
    const int esz[3] = {esize(dy_dtype), esize(src_dtype), esize(src_dtype)};
    const int v = vector_width(cols, ptrs, esz, 3);
    m.group = group_threads(cols / v);
    m.token_blocks = (tokens + MOVE_THREADS / m.group - 1) / (MOVE_THREADS / m.group);
    const int64_t blocks = m.token_blocks + (d_src ? (rows + 31) / 32 : 0);
    if (blocks > 0x7FFFFFFFLL || tokens > 0x7FFFFFFFFFFFLL / top_k) return MXFP8_ERR_UNSUPPORTED;
    if (!(m.status = device_status_word())) return MXFP8_ERR_CUDA;
    const unsigned grid = (unsigned)blocks;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t err;
    if (dy_dtype == MXFP8_BF16) err = src_dtype == MXFP8_BF16 ? launch_grad<MXFP8_BF16, MXFP8_BF16>(v, grid, m, st) : launch_grad<MXFP8_BF16, MXFP8_FP32>(v, grid, m, st);
    else err = src_dtype == MXFP8_BF16 ? launch_grad<MXFP8_FP32, MXFP8_BF16>(v, grid, m, st) : launch_grad<MXFP8_FP32, MXFP8_FP32>(v, grid, m, st);
    return err == cudaSuccess ? MXFP8_OK : MXFP8_ERR_CUDA;
}
