// Mixture-of-experts token movement around mxfp8_grouped_gemm (App. A.4): sorting the routed tokens by expert into
// segments that start at multiples of 128 rows, gathering the experts' outputs back with the router's weights, and the
// gradient of that sum.  (The gather into the sorted order is fused with the conversion: quantize_gather.cu.)
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
constexpr int SORT_MAX_CHUNKS = 148;          // one CTA per multiprocessor of a B200 (a size without a device: mxfp8_moe_sort_ws_bytes needs it)
constexpr int SORT_ONE_CTA_SLOTS = 4096;      // up to here one CTA sorts alone
constexpr int SORT_CHUNK_STEP = 512;          // chunks of several CTAs are multiples of this

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
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");      // the second launch may start on its own counting
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
// What bounds it is the chain of dependent steps (two launches, the chunks' counts, five CTA barriers), not the bytes: 6 of
// 64 experts for 8192 tokens 6.4 us, 8 of 256 for 131071 tokens 17 us.  (Putting a chunk's slots in order
// in shared memory first, for fewer scattered stores, took longer, and so did one cluster of eight CTAs that exchanges
// counts through shared memory in place of two launches.)
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
    // eight groups of 32 slots at a time, their loads in flight together; a run of one such block stays in registers
    int id[8];
    auto fetch = [&](int base) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int s = base + i * 32 + lane;
            id[i] = s < w_last ? a.ids[s] : -1;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if ((unsigned)id[i] >= (unsigned)E) id[i] = -1;
    };
    fetch(w_first);
    __syncthreads();
    for (int base = w_first;;) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (id[i] >= 0) atomicAdd(&hist[warp][id[i]], 1);
        base += 256;
        if (base >= w_last) break;
        fetch(base);
    }
    __syncthreads();
    if (a.counts != nullptr) {
        asm volatile("griddepcontrol.wait;" ::: "memory");             // the first launch's counts are there
        const int e = tid & (SORT_MAX_EXPERTS - 1), quarter = tid / SORT_MAX_EXPERTS;
        int sum = 0, sum_before = 0;
        if (e < E)
#pragma unroll 20
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
    const int bits = 32 - __clz(E - 1);                     // of an expert's number
    for (int base = w_first; base < w_last; base += 256) {
        if (run > 256) fetch(base);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int s = base + i * 32 + lane;
            if (base + i * 32 >= w_last) break;
            // lanes with the same expert, bit by bit (the match instruction walks the distinct values and takes longer once
            // there are many)
            unsigned same = __ballot_sync(0xFFFFFFFFu, id[i] >= 0);
            for (int b = 0; b < bits; ++b) {
                const unsigned set = __ballot_sync(0xFFFFFFFFu, id[i] >> b & 1);
                same &= (id[i] >> b & 1) ? set : ~set;
            }
            const int rank = __popc(same & ((1u << lane) - 1u));
            int place = 0;                                  // among the expert's slots of all chunks
            if (id[i] >= 0) place = hist[warp][id[i]] + rank;
            __syncwarp();
            if (id[i] >= 0 && rank == 0) hist[warp][id[i]] += __popc(same);
            __syncwarp();
            if (s < w_last) {
                const int row = id[i] >= 0 ? start[id[i]] + place : -1;
                a.row_of[s] = row;
                if (row >= 0) a.slot_of[row] = s;
            }
        }
    }
    // rows without a slot: the padding behind every expert, and everything behind the last segment
    for (int e = (int)blockIdx.x * 8 + (tid >> 7); e < E; e += (int)gridDim.x * 8) {
        const int row = start[e] + total[e] + (tid & 127);
        if (row < start[e + 1]) a.slot_of[row] = -1;
    }
    for (int row = start[E] + (int)(blockIdx.x * SORT_THREADS + tid); row < a.rows; row += (int)gridDim.x * SORT_THREADS) a.slot_of[row] = -1;
}

// Slots per CTA: all of them in one CTA while they are few, else equal chunks over at most one CTA per multiprocessor
// (49152 slots: 6.4 us in chunks of 512, 7.2 to 7.9 us in chunks of 1024 or 2048).
int sort_chunk(int64_t slots)
{
    if (slots <= SORT_ONE_CTA_SLOTS) return SORT_ONE_CTA_SLOTS;
    const int64_t per = (slots + SORT_MAX_CHUNKS - 1) / SORT_MAX_CHUNKS;
    return (int)((per + SORT_CHUNK_STEP - 1) / SORT_CHUNK_STEP * SORT_CHUNK_STEP);
}

// -------------------------------------------------------------------------------------------- gather, weight, sum
// V consecutive elements of a row as they lie in memory, read and written in pieces of up to 16 bytes.  Results are stored the
// ordinary way, so that L2 keeps what it can of them for the call that reads them: with evict-first stores too, the layer's sum (8192
// tokens, top-6, 2048 BF16 columns) alone takes 39.2 us in place of 40.2, but followed by an elementwise sum 56.2 in place of 55.2; its
// gradient alone 76.9 in place of 79.7, but followed by the conversion of the rows that it wrote 167.4 in place of 159.8.
// STREAM: rows that are read leave L2 before anything else.  In the sum that pays where a lane has up to eight rows in flight (the
// layer: 40.2 us | 42.5 with ordinary loads, followed by the sum 55.2 | 57.9; 1024 tokens 13.7 | 13.2, 16.8 | 17.2) and costs where it has
// two (8192 tokens, top-2, 4096 columns: 61.0 | 53.7, followed by the sum 94.2 | 85.7); in the gradient it pays with two (4096 tokens of
// these 32.9 | 36.5, followed by the conversion 56.5 | 62.3) and makes no difference with more (the layer 79.7 | 79.1, 159.8 | 159.5).
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
    template <bool STREAM>
    __device__ __forceinline__ void load(const void* base, int64_t element)
    {
        const P* p = reinterpret_cast<const P*>(static_cast<const uint8_t*>(base) + element * ESZ);
#pragma unroll
        for (int i = 0; i < N; ++i) piece[i] = STREAM ? __ldcs(p + i) : p[i];
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

constexpr int MOVE_THREADS = 256, MOVE_WARPS = MOVE_THREADS / 32;

// Row of a slot, or -1.  Anything but -1 and a row of the tensor is an error of the caller's array: reported, not used.
__device__ __forceinline__ int checked_row(int32_t r, int64_t rows, int* status)
{
    if (r >= 0 && r < rows) return r;
    if (r != -1) atomicExch(status, (int)MXFP8_ERR_DEVICE_ARGS);
    return -1;
}
// Rows that the gradient may touch: those in use where the caller names their end, none where that end cannot be one.
__device__ __forceinline__ int64_t rows_in_use(const MoveArgs& a)
{
    if (a.used == nullptr) return a.rows;
    const int used = *a.used;
    if (used >= 0 && used <= a.rows) return used;
    atomicExch(a.status, (int)MXFP8_ERR_DEVICE_ARGS);
    return 0;
}

// Vectors per lane and row when there is plenty to do: a lane asks for 256 bytes of the K rows before it uses any, which
// with 16 warps on a multiprocessor keeps more than 100 KB in flight.  Layer as above: 86 % of the rate of a plain copy, its gradient
// 84 %.  With one or two choices per token it reaches less (8192 tokens of 4096 columns, top-2: 57 %), for a cause not yet found.
template <int DTYPE, int V, int K> constexpr int MANY = (256 / K / (V * (DTYPE == MXFP8_BF16 ? 2 : 4))) < 1 ? 1
                                                      : (256 / K / (V * (DTYPE == MXFP8_BF16 ? 2 : 4))) > 8 ? 8 : (256 / K / (V * (DTYPE == MXFP8_BF16 ? 2 : 4)));
template <int U> constexpr int COMBINE_CTAS = U == 1 ? 4 : 2;       // per multiprocessor

// dst[t, c] = sum_j w[t, j] * src[row_of[t, j], c]: FP32 sums in the order of j, one rounding at the end.
// A warp takes one token's run of 32 * V * U columns at a time; lane j fetches the j-th row number and weight of its next
// item while the current one is summed, so that the two dependent loads of a gather are paid once per warp, not per item.
template <int SRC, int DST, int V, int K, int U>
__global__ void __launch_bounds__(MOVE_THREADS, COMBINE_CTAS<U>) moe_combine_kernel(const MoveArgs a)
{
    constexpr int RUN = 32 * V * U;
    constexpr bool STREAM_ROWS = K > 2;                // see Vec
    const int lane = threadIdx.x & 31;
    const uint32_t runs = (uint32_t)((a.cols + RUN - 1) / RUN), items = (uint32_t)a.tokens * runs, step = gridDim.x * MOVE_WARPS;
    const bool one_round = a.top_k <= K;
    auto lookup = [&](uint32_t t, int j, int& row, float& w) {
        row = -1;
        w = 0.f;
        if (j < a.top_k) {
            const int64_t slot = (int64_t)t * a.top_k + j;
            row = checked_row(a.row_of[slot], a.rows, a.status);
            w = a.weights ? a.weights[slot] : 1.f;
        }
    };
    uint32_t item = blockIdx.x * MOVE_WARPS + (threadIdx.x >> 5);
    if (item >= items) return;
    uint32_t t = item / runs, run = item - t * runs;                           // token and run of the item, carried on by additions
    const uint32_t t_step = step / runs, run_step = step - t_step * runs;
    int my_row = -1, next_row = -1;
    float my_w = 0.f, next_w = 0.f;
    if (lane < K) lookup(t, lane, my_row, my_w);
    for (; item < items; item += step) {
        const int64_t c0 = (int64_t)run * RUN + lane * V;
        uint32_t next_t = t + t_step, next_run = run + run_step;
        if (next_run >= runs) { next_run -= runs; ++next_t; }
        if (one_round && item + step < items && lane < K) lookup(next_t, lane, next_row, next_w);
        float acc[U][V];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < V; ++i) acc[u][i] = 0.f;
        for (int j0 = 0; j0 < a.top_k; j0 += K) {
            if (!one_round) {
                my_row = -1;
                if (lane < K) lookup(t, j0 + lane, my_row, my_w);
            }
            Vec<SRC, V> x[K][U];
            bool live[K];
#pragma unroll
            for (int j = 0; j < K; ++j) {
                const int r = __shfl_sync(0xFFFFFFFFu, my_row, j);
                live[j] = r >= 0;
                if (live[j])
#pragma unroll
                    for (int u = 0; u < U; ++u)
                        if (c0 + u * 32 * V < a.cols) x[j][u].template load<STREAM_ROWS>(a.src, (int64_t)r * a.cols + c0 + u * 32 * V);
            }
#pragma unroll
            for (int j = 0; j < K; ++j) {
                const float w = __shfl_sync(0xFFFFFFFFu, my_w, j);
                if (live[j])
#pragma unroll
                    for (int u = 0; u < U; ++u)
#pragma unroll
                        for (int i = 0; i < V; ++i) acc[u][i] = fmaf(w, x[j][u].get(i), acc[u][i]);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (c0 + u * 32 * V < a.cols) {
                Vec<DST, V> y;
#pragma unroll
                for (int i = 0; i < V; ++i) y.set(i, acc[u][i]);
                y.store(a.dst, (int64_t)t * a.cols + c0 + u * 32 * V);
            }
        my_row = next_row;
        my_w = next_w;
        t = next_t;
        run = next_run;
    }
}

// d_src[row_of[t, j], c] = w[t, j] * dy[t, c] (one FP32 product, rounded to src's type) and
// d_weights[t, j] = sum_c dy[t, c] * src[row_of[t, j], c] (FP32: lane-strided partial sums, then a fixed tree), so dy is
// read once per token and K choices.  Rows have to lie among those in use.  `group` threads share a token: one warp while tokens fill the machine, which
// leaves the sums to shuffles; up to a whole CTA for few tokens.  CTAs behind the tokens' clear the padding rows.
template <int DY, int SRC, int V, int K>
__global__ void __launch_bounds__(MOVE_THREADS) moe_combine_grad_kernel(const MoveArgs a)
{
    constexpr int U = MANY<SRC, V, K> < 2 ? 1 : 2;
    __shared__ float sums[MOVE_WARPS][K];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if ((int64_t)blockIdx.x >= a.token_blocks) {
        const int64_t used = rows_in_use(a);
        const int64_t row0 = ((int64_t)blockIdx.x - a.token_blocks) * 32 + warp * 4;
        for (int64_t r = row0; r < row0 + 4 && r < used; ++r) {
            const int slot = a.slot_of[r];
            if (slot >= 0 && slot < a.tokens * a.top_k) continue;
            if (slot != -1) atomicExch(a.status, (int)MXFP8_ERR_DEVICE_ARGS);
            Vec<SRC, V> z;
            z.zero();
            for (int64_t c = (int64_t)lane * V; c < a.cols; c += 32 * V) z.store(a.dst, r * a.cols + c);
        }
        return;
    }
    const int per_block = MOVE_THREADS / a.group, member = tid % a.group;
    const int64_t t = (int64_t)blockIdx.x * per_block + tid / a.group;
    const int64_t stride = (int64_t)a.group * V;
    const int64_t rows = rows_in_use(a);
    for (int j0 = 0; j0 < a.top_k; j0 += K) {
        int my_row = -1;
        float my_w = 0.f;
        if (t < a.tokens && lane < K && j0 + lane < a.top_k) {
            const int64_t slot = t * a.top_k + j0 + lane;
            my_row = checked_row(a.row_of[slot], rows, a.status);
            my_w = a.weights ? a.weights[slot] : 1.f;
        }
        int row[K];
        float w[K], acc[K];
#pragma unroll
        for (int j = 0; j < K; ++j) {
            row[j] = __shfl_sync(0xFFFFFFFFu, my_row, j);
            w[j] = __shfl_sync(0xFFFFFFFFu, my_w, j);
            acc[j] = 0.f;
        }
        if (t < a.tokens)
            for (int64_t c0 = (int64_t)member * V; c0 < a.cols; c0 += U * stride) {
                Vec<DY, V> g[U];
                Vec<SRC, V> x[K][U];
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (c0 + u * stride < a.cols) g[u].template load<true>(a.dy, t * a.cols + c0 + u * stride);
                if (a.d_weights != nullptr)
#pragma unroll
                    for (int j = 0; j < K; ++j)
                        if (row[j] >= 0)
#pragma unroll
                            for (int u = 0; u < U; ++u)
                                if (c0 + u * stride < a.cols) x[j][u].template load<true>(a.src, (int64_t)row[j] * a.cols + c0 + u * stride);
#pragma unroll
                for (int j = 0; j < K; ++j) {
                    if (row[j] < 0) continue;
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        if (c0 + u * stride >= a.cols) continue;
                        if (a.d_weights != nullptr)
#pragma unroll
                            for (int i = 0; i < V; ++i) acc[j] = fmaf(g[u].get(i), x[j][u].get(i), acc[j]);
                        if (a.dst != nullptr) {
                            Vec<SRC, V> d;
#pragma unroll
                            for (int i = 0; i < V; ++i) d.set(i, w[j] * g[u].get(i));
                            d.store(a.dst, (int64_t)row[j] * a.cols + c0 + u * stride);
                        }
                    }
                }
            }
        if (a.d_weights == nullptr) continue;
        float mine = 0.f;                                  // lane j ends with the sum of choice j
#pragma unroll
        for (int j = 0; j < K; ++j) {
            float v = acc[j];
#pragma unroll
            for (int off = 16; off > 0; off >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, off);
            if (lane == j) mine = v;
        }
        if (a.group == 32) {
            if (t < a.tokens && lane < K && j0 + lane < a.top_k) a.d_weights[t * a.top_k + j0 + lane] = mine;
            continue;
        }
        if (lane < K) sums[warp][lane] = mine;
        __syncthreads();
        if (member < K && t < a.tokens && j0 + member < a.top_k) {
            const int w0 = (tid / a.group) * (a.group / 32);
            float v = 0.f;
            for (int k = 0; k < a.group / 32; ++k) v += sums[w0 + k][member];
            a.d_weights[t * a.top_k + j0 + member] = v;
        }
        __syncthreads();
    }
}

// Largest vector (8, 4, 2 or 1 elements, at most `most`) that every row of every tensor starts on: it has to divide cols,
// and each base has to lie on a boundary of its pieces.
int vector_width(int64_t cols, const void* const* ptrs, const int* esz, int count, int most)
{
    for (int v = most; v > 1; v >>= 1) {
        bool ok = cols % v == 0;
        for (int i = 0; ok && i < count; ++i) {
            const int bytes = v * esz[i] < 16 ? v * esz[i] : 16;
            ok = (reinterpret_cast<uintptr_t>(ptrs[i]) % bytes) == 0;
        }
        if (ok) return v;
    }
    return 1;
}

int sm_count()
{
    static PerDeviceCache<int> cache;
    int n = 0;
    return cache.get(n, [](int dev, int& v) { return cudaDeviceGetAttribute(&v, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess && v > 0; }) ? n : 0;
}

// Threads that share a token in the gradient: as few as keep 24 warps on every multiprocessor, at most what a row has
// vectors for.
int group_threads(int64_t tokens, int64_t vectors, int sms)
{
    int g = 32;
    while (g < MOVE_THREADS && g < vectors && tokens * (g / 32) < 24 * sms) g <<= 1;
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
    if (num_experts > SORT_MAX_EXPERTS || tokens > 0x7F000000LL || tokens * top_k > 0x7F000000LL || rows > 0x7FF00000LL) return MXFP8_ERR_UNSUPPORTED;   // 32-bit counters
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
        if (cudaGetLastError() != cudaSuccess) return MXFP8_ERR_CUDA;
        // the second launch starts beside the first one (its own counting needs nothing of it) and waits for it in the kernel
        cudaLaunchConfig_t cfg{};
        cfg.gridDim = dim3((unsigned)chunks);
        cfg.blockDim = dim3(SORT_THREADS);
        cfg.stream = st;
        cudaLaunchAttribute attr{};
        attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr.val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = &attr;
        cfg.numAttrs = 1;
        if (cudaLaunchKernelEx(&cfg, moe_sort_kernel, a) != cudaSuccess) return MXFP8_ERR_CUDA;
        count_launch(2);
    }
    return cudaGetLastError() == cudaSuccess ? MXFP8_OK : MXFP8_ERR_CUDA;
}

namespace {
// Two or eight rows in flight per lane; several vectors of each where the rows are long enough and the items fill the machine
template <int A, int B, int V, int K>
cudaError_t launch_combine_k(const MoveArgs& m, int sms, cudaStream_t st)
{
    auto go = [&](auto kernel, int run, int ctas) {
        const int64_t items = m.tokens * ((m.cols + run - 1) / run), blocks = (items + MOVE_WARPS - 1) / MOVE_WARPS;
        kernel<<<(unsigned)(blocks < (int64_t)ctas * sms ? blocks : (int64_t)ctas * sms), MOVE_THREADS, 0, st>>>(m);
    };
    constexpr int U = MANY<A, V, K>, RUN = 32 * V * U;
    if (U > 1 && m.cols >= RUN && m.tokens * (m.cols / RUN) >= (int64_t)2 * MOVE_WARPS * COMBINE_CTAS<U> * sms)
        go(moe_combine_kernel<A, B, V, K, U>, RUN, COMBINE_CTAS<U>);
    else go(moe_combine_kernel<A, B, V, K, 1>, 32 * V, COMBINE_CTAS<1>);
    count_launch(1);
    return cudaGetLastError();
}
template <int A, int B, int V>
cudaError_t launch_combine_v(const MoveArgs& m, int sms, cudaStream_t st)
{
    return m.top_k <= 2 ? launch_combine_k<A, B, V, 2>(m, sms, st) : launch_combine_k<A, B, V, 8>(m, sms, st);
}
template <int A, int B>
cudaError_t launch_combine(int v, const MoveArgs& m, int sms, cudaStream_t st)
{
    if constexpr (A == MXFP8_BF16)
        if (v == 8) return launch_combine_v<A, B, 8>(m, sms, st);
    if (v >= 4) return launch_combine_v<A, B, 4>(m, sms, st);
    if (v == 2) return launch_combine_v<A, B, 2>(m, sms, st);
    return launch_combine_v<A, B, 1>(m, sms, st);
}
template <int A, int B, int V>
cudaError_t launch_grad_v(unsigned grid, const MoveArgs& m, cudaStream_t st)
{
    if (m.top_k <= 2) moe_combine_grad_kernel<A, B, V, 2><<<grid, MOVE_THREADS, 0, st>>>(m);
    else if (m.top_k <= 4) moe_combine_grad_kernel<A, B, V, 4><<<grid, MOVE_THREADS, 0, st>>>(m);
    else moe_combine_grad_kernel<A, B, V, 8><<<grid, MOVE_THREADS, 0, st>>>(m);
    count_launch(1);
    return cudaGetLastError();
}
template <int A, int B>
cudaError_t launch_grad(int v, unsigned grid, const MoveArgs& m, cudaStream_t st)
{
    if constexpr (B == MXFP8_BF16)
        if (v == 8) return launch_grad_v<A, B, 8>(grid, m, st);
    if (v >= 4) return launch_grad_v<A, B, 4>(grid, m, st);
    if (v == 2) return launch_grad_v<A, B, 2>(grid, m, st);
    return launch_grad_v<A, B, 1>(grid, m, st);
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
    if (rows > 0x7FFFFFFFLL || cols > 0x7FFFFFFFLL || tokens > 0x7FFFFFFFLL) return MXFP8_ERR_UNSUPPORTED;
    if ((rows > 0 && !src) || !row_of || !dst) return MXFP8_ERR_NULL;
    if (misaligned(src, esize(src_dtype)) || misaligned(dst, esize(dst_dtype)) || misaligned(row_of, 4) || misaligned(weights, 4)) return MXFP8_ERR_ALIGN;
    MoveArgs m{};
    m.src = src; m.row_of = row_of; m.weights = weights; m.dst = dst;
    m.rows = rows; m.cols = cols; m.tokens = tokens; m.top_k = top_k;
    const void* ptrs[2] = {src, dst};
    const int esz[2] = {esize(src_dtype), esize(dst_dtype)};
    const int v = vector_width(cols, ptrs, esz, 2, 16 / esize(src_dtype));
    if (tokens * ((cols + 32 * v - 1) / (32 * v)) >= 0x7FFF0000LL) return MXFP8_ERR_UNSUPPORTED;      // items are counted in 32 bits
    const int sms = sm_count();
    if (sms <= 0 || !(m.status = device_status_word())) return MXFP8_ERR_CUDA;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t err;
    if (src_dtype == MXFP8_BF16) err = dst_dtype == MXFP8_BF16 ? launch_combine<MXFP8_BF16, MXFP8_BF16>(v, m, sms, st) : launch_combine<MXFP8_BF16, MXFP8_FP32>(v, m, sms, st);
    else err = dst_dtype == MXFP8_BF16 ? launch_combine<MXFP8_FP32, MXFP8_BF16>(v, m, sms, st) : launch_combine<MXFP8_FP32, MXFP8_FP32>(v, m, sms, st);
    return err == cudaSuccess ? MXFP8_OK : MXFP8_ERR_CUDA;
}

extern "C" int mxfp8_moe_combine_grad(const void* dy, int dy_dtype, int64_t tokens, int64_t cols, const void* src, int src_dtype, int64_t rows,
                                      const int32_t* row_of, const int32_t* slot_of, int top_k, const float* weights,
                                      const int32_t* group_offsets, int num_groups, void* d_src, float* d_weights, void* stream)
{
    if (bad_dtype(dy_dtype) || bad_dtype(src_dtype)) return MXFP8_ERR_ENUM;
    if (rows < 0 || cols <= 0 || tokens < 0 || top_k < 1 || num_groups < 1) return MXFP8_ERR_SHAPE;
    if (tokens == 0) return MXFP8_OK;
    if (rows > 0x7FFFFFFFLL || cols > 0x7FFFFFFFLL || tokens > 0x7FFFFFFFLL) return MXFP8_ERR_UNSUPPORTED;
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
    const int v = vector_width(cols, ptrs, esz, 3, 16 / esize(src_dtype));
    const int sms = sm_count();
    if (sms <= 0) return MXFP8_ERR_CUDA;
    m.group = group_threads(tokens, cols / v, sms);
    m.token_blocks = (tokens + MOVE_THREADS / m.group - 1) / (MOVE_THREADS / m.group);
    const int64_t blocks = m.token_blocks + (d_src ? (rows + 31) / 32 : 0);
    if (blocks > 0x7FFFFFFFLL) return MXFP8_ERR_UNSUPPORTED;
    if (!(m.status = device_status_word())) return MXFP8_ERR_CUDA;
    const unsigned grid = (unsigned)blocks;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t err;
    if (dy_dtype == MXFP8_BF16) err = src_dtype == MXFP8_BF16 ? launch_grad<MXFP8_BF16, MXFP8_BF16>(v, grid, m, st) : launch_grad<MXFP8_BF16, MXFP8_FP32>(v, grid, m, st);
    else err = src_dtype == MXFP8_BF16 ? launch_grad<MXFP8_FP32, MXFP8_BF16>(v, grid, m, st) : launch_grad<MXFP8_FP32, MXFP8_FP32>(v, grid, m, st);
    return err == cudaSuccess ? MXFP8_OK : MXFP8_ERR_CUDA;
}
