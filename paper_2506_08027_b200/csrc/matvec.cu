// Products of a few tokens with E2M1 (MXFP4) matrices: the conversion's 4-bit codes and UE8M0 scales (Sec. 2, Table 1) as
// stored weights, BF16 activations, FP32 sums.  One matrix for all tokens or one chosen per (token, choice) slot, which
// is what a mixture-of-experts layer (App. A.4) computes when it answers a few tokens.
//
//   y[s, n] = sum over groups g of 32 columns of  2^(b[n,g] - 127) * sum_{k in g} code[n,k] * x[s / slots_per_token, k]
//
// The floor is the weight bytes, 17/32 byte per weight.  They are read and decoded once per eight slots of a matrix that is chosen, and
// once per 8, 16 or 32 tokens of a matrix that serves all: made for a few tokens.  The codes become BF16 registers (exact) and go
// through the warp-level tensor instructions with the tokens as the narrow side.  (The block-scaled tensor instructions would take
// the 4-bit codes as they are, but not BF16 activations.)
// Weights from HBM, us, beside mxfp8_gemm of E4M3 activations and the same codes in their 16-byte slots with the conversion of the
// activations: 28672 x 4096, 1 token 19.8 (34.5), 16 tokens 27.6 (33.8), 17 tokens 40.7 (34.5), 32 tokens 44.7 (29.5), 128 tokens 160 (32);
// 4096 x 4096, 1 token 5.9 (19.0), 32 tokens 11.1 (17.3), 64 tokens 19.1 (17.6), 128 tokens 35 (18).
//
// The packed layout and its decoding: e2m1_tiles.cuh.
#include "e2m1_tiles.cuh"
#include "mxfp8_host.h"

namespace mxfp8 {
namespace {

constexpr int MV_MAX_SLOTS = 1024;              // (token, choice) pairs of one call

struct MatvecArgs {
    const __nv_bfloat16* x;      // [tokens, cols]
    const uint8_t* packed;       // [matrices][row tiles][column tiles][1088]
    const int32_t* ids;          // [slots] or null: matrix 0 for all
    void* y;                     // [slots, rows]
    int slots, per_token, matrices, by_matrix;
    int64_t rows, cols;
    int row_tiles, col_tiles;
    int split_log;               // 2^split_log warps share a row group and split its columns (1, 2, 4 or 8)
    uint32_t per_token_magic;
};

template <typename T> __device__ __forceinline__ T to_out(float v);
template <> __device__ __forceinline__ float to_out<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 to_out<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

template <int R, int NT> constexpr int WARP_SUMS = R * TILE_ROWS * (8 * NT + 1);      // floats of a warp's sums, padded

// CTA (i, u): groups of R row tiles times the slots that chose a matrix, 8 NT at a time.  `split` warps share a group and
// take its column tiles in turn; their sums meet in shared memory and are added in a fixed order.  Weights and activations go
// from global memory to the registers that the tensor instructions read them from; other warps cover the latency, or,
// where registers leave few of them (AHEAD), the next tile's loads run under this tile's products.
// u counts slots (the first slot with a matrix works for all of them, the others leave) or, where there are fewer
// matrices than slots, matrices.
template <typename OUT, int R, int NT, int WARPS, int PER_SM, bool AHEAD>
__global__ void __launch_bounds__(32 * WARPS, PER_SM) matvec_kernel(const MatvecArgs a)
{
    constexpr int THREADS = 32 * WARPS;
    extern __shared__ float sums[];
    __shared__ int list[MV_MAX_SLOTS];
    __shared__ int listed;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, u = blockIdx.y;
    const int split = 1 << a.split_log, groups = WARPS >> a.split_log;  // row groups of this CTA
    static_assert((R & (R - 1)) == 0 && (WARPS & (WARPS - 1)) == 0, "rows of a CTA are a power of two");
    const int cta_rows = groups * R * TILE_ROWS, cta_rows_log = 31 - __clz(cta_rows);
    const int64_t row0 = (int64_t)blockIdx.x * cta_rows;                   // its first row
    OUT* y = static_cast<OUT*>(a.y);
    int matrix = 0, count = a.slots;
    if (a.ids != nullptr) {
        matrix = a.by_matrix ? u : a.ids[u];
        if ((unsigned)matrix >= (unsigned)a.matrices) {
            // no such matrix: this slot's rows are zero
            for (int n = tid; n < cta_rows; n += THREADS)
                if (row0 + n < a.rows) y[(int64_t)u * a.rows + row0 + n] = to_out<OUT>(0.f);
            return;
        }
        if (warp == 0) {
            int found = 0, first = -1;
            for (int base = 0; base < a.slots; base += 32) {
                const int s = base + lane;
                const unsigned hit = __ballot_sync(0xFFFFFFFFu, s < a.slots && a.ids[min(s, a.slots - 1)] == matrix);
                if (hit && first < 0) first = base + __ffs(hit) - 1;
                if (hit >> lane & 1u) list[found + __popc(hit & ((1u << lane) - 1u))] = s;
                found += __popc(hit);
            }
            if (lane == 0) listed = (a.by_matrix || first == u) ? found : 0;
        }
        if (a.by_matrix && u == 0)                      // slots without a matrix: theirs are zero
            for (int s = warp; s < a.slots; s += WARPS)
                if ((unsigned)a.ids[s] >= (unsigned)a.matrices)
                    for (int n = lane; n < cta_rows; n += 32)
                        if (row0 + n < a.rows) y[(int64_t)s * a.rows + row0 + n] = to_out<OUT>(0.f);
        __syncthreads();
        count = listed;
    }
    auto slot = [&](int i) { return a.ids ? list[i] : i; };
    const int token = lane >> 2, quarter = lane & 3;    // as columns of the tensor instructions' second operand
    const int group = warp >> a.split_log, part = warp & (split - 1);
    const int rt0 = (blockIdx.x * groups + group) * R;  // this warp's first row tile
    const uint8_t* tile[R];
#pragma unroll
    for (int r = 0; r < R; ++r)                         // rows behind the matrix repeat its last tile and are not stored
        tile[r] = a.packed + ((int64_t)matrix * a.row_tiles + min(rt0 + r, a.row_tiles - 1)) * a.col_tiles * TILE_BYTES + lane * 16;
    const int whole = (int)(a.cols / TILE_COLS);        // column tiles without padding
    for (int s0 = 0; s0 < count; s0 += 8 * NT) {
        const int tokens = min(8 * NT, count - s0);
        const __nv_bfloat16* x[NT];
        bool has[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            has[t] = 8 * t + token < tokens;
            int row = 0, choice = 0;
            if (has[t]) divmod((uint32_t)slot(s0 + 8 * t + token), (uint32_t)a.per_token, a.per_token_magic, row, choice);
            x[t] = a.x + (int64_t)row * a.cols + quarter * 8;
        }
        float acc[R][NT][4];
        Operands<R, NT> now;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int g = 0; g < 4; ++g) now.x[t][g] = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[r][t][i] = 0.f;
        int kt = part;
        if constexpr (!AHEAD) {
            for (; kt < whole; kt += split) {
                now.load(tile, (int64_t)kt * TILE_BYTES, x, has, (int64_t)kt * TILE_COLS, lane);
                product<R, NT>(now, acc);
            }
        } else {
            Operands<R, NT> next = now;
            if (kt < whole) now.load(tile, (int64_t)kt * TILE_BYTES, x, has, (int64_t)kt * TILE_COLS, lane);
            while (kt < whole) {
                kt += split;
                if (kt < whole) next.load(tile, (int64_t)kt * TILE_BYTES, x, has, (int64_t)kt * TILE_COLS, lane);
                product<R, NT>(now, acc);
                if (kt >= whole) break;
                kt += split;
                if (kt < whole) now.load(tile, (int64_t)kt * TILE_BYTES, x, has, (int64_t)kt * TILE_COLS, lane);
                product<R, NT>(next, acc);
            }
        }
        if (whole < a.col_tiles && (whole & (split - 1)) == part) {      // the columns end inside the last tile
            bool none[NT];
#pragma unroll
            for (int t = 0; t < NT; ++t) none[t] = false;
            now.load(tile, (int64_t)whole * TILE_BYTES, x, none, 0, lane);
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const int64_t k = (int64_t)whole * TILE_COLS + g * 32;
                    now.x[t][g] = make_uint4(0u, 0u, 0u, 0u);
                    if (has[t] && k < a.cols) now.x[t][g] = *reinterpret_cast<const uint4*>(x[t] + k);
                }
            product<R, NT>(now, acc);
        }
        constexpr int P = 8 * NT + 1;
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                float* to = sums + warp * WARP_SUMS<R, NT> + (r * TILE_ROWS + token) * P + 8 * t + 2 * quarter;
                to[0] = acc[r][t][0];
                to[1] = acc[r][t][1];
                to[8 * P] = acc[r][t][2];
                to[8 * P + 1] = acc[r][t][3];
            }
        __syncthreads();
        for (int i = tid; i < cta_rows * tokens; i += THREADS) {
            const int n = i & (cta_rows - 1), j = i >> cta_rows_log;
            const int g = n / (R * TILE_ROWS), m = n % (R * TILE_ROWS);
            const float* from = sums + (g << a.split_log) * WARP_SUMS<R, NT> + m * P + j;
            float v = 0.f;
#pragma unroll
            for (int w = 0; w < WARPS; ++w)
                if (w < split) v += from[w * WARP_SUMS<R, NT>];
            if (row0 + n < a.rows) y[(int64_t)slot(s0 + j) * a.rows + row0 + n] = to_out<OUT>(v);
        }
        __syncthreads();
    }
}

template <typename OUT, int R, int NT, int WARPS, int PER_SM, bool AHEAD>
cudaError_t launch_matvec(MatvecArgs a, unsigned grid_y, cudaStream_t st)
{
    auto kernel = matvec_kernel<OUT, R, NT, WARPS, PER_SM, AHEAD>;
    constexpr int SUMS = WARPS * WARP_SUMS<R, NT> * (int)sizeof(float);
    static unsigned long long set = 0;
    cudaError_t err = ensure_dynamic_smem(kernel, SUMS, set);
    if (err != cudaSuccess) return err;
    a.split_log = 0;
    while ((1 << a.split_log) < WARPS && (1 << a.split_log) < a.col_tiles) ++a.split_log;
    a.per_token_magic = div_magic((uint32_t)a.per_token);
    auto ctas = [&](int log) { return (int64_t)((a.row_tiles + (WARPS >> log) * R - 1) / ((WARPS >> log) * R)); };
    // Longer runs per warp wherever at least two full waves of CTAs (148 multiprocessors) remain: 2816 x 2048 matrices of six experts
    // for eight tokens take 32.8 us with two warps to a row group, 36.4 us with four and 33.4 us with one; one 28672 x 4096 matrix
    // for eight tokens, whose waves would run out, 19.5 us with four, 21.3 us with two and 25.8 us with one.
    while (a.split_log > 0 && ctas(a.split_log - 1) * grid_y >= 2 * PER_SM * 148) --a.split_log;
    kernel<<<dim3((unsigned)ctas(a.split_log), grid_y), 32 * WARPS, SUMS, st>>>(a);
    count_launch(1);
    return cudaGetLastError();
}

// Tokens worked on together: 8, 16 or 32 (a matrix's slots are seldom more than a few when they choose).  Many row tiles: two
// to a warp, which halves the reads of the activations, in small CTAs that end one by one; few: one to a warp and eight
// warps to its columns, which keeps more multiprocessors busy.  28672 x 4096: 8 tokens 19.3 us (eight-warp CTAs 21.6),
// 16 tokens 26.6 us (29.7), 32 tokens 45 us (49); 6144 x 4096 for one token: 5.7 us with few, 6.5 us with many.  Chosen matrices take
// the variant of eight slots whatever their number: most have a few, and one with more is walked again per eight.
template <typename OUT>
cudaError_t launch_matvec(const MatvecArgs& a, unsigned grid_y, cudaStream_t st)
{
    const bool few = (int64_t)(a.row_tiles + 1) / 2 * grid_y < 4 * 148;
    if (a.slots <= 8 || a.ids) return few ? launch_matvec<OUT, 1, 1, 8, 4, false>(a, grid_y, st) : launch_matvec<OUT, 2, 1, 4, 4, true>(a, grid_y, st);
    if (a.slots <= 16) return few ? launch_matvec<OUT, 1, 2, 8, 3, false>(a, grid_y, st) : launch_matvec<OUT, 2, 2, 4, 4, false>(a, grid_y, st);
    return few ? launch_matvec<OUT, 1, 4, 8, 2, false>(a, grid_y, st) : launch_matvec<OUT, 2, 4, 4, 2, true>(a, grid_y, st);
}

// One thread per word of eight codes of the packed layout, from the library's own slots (16 codes to 16 bytes, code i
// in bits 4i .. 4i + 3 of the first eight); the first 64 bytes' worth of threads of a tile also move its scales.
__global__ void __launch_bounds__(256) e2m1_pack_kernel(const uint8_t* __restrict__ q, const uint8_t* __restrict__ s, uint8_t* __restrict__ packed,
                                                        int64_t rows, int64_t cols, int64_t row_tiles, int64_t col_tiles)
{
    const int64_t tile = blockIdx.x;                    // over matrices x row tiles x column tiles
    const int64_t kt = tile % col_tiles, rt = tile / col_tiles % row_tiles, m = tile / (col_tiles * row_tiles);
    const int t = threadIdx.x, g = t & 3, c = (t >> 2) & 3, r = t >> 4;      // word t of the tile
    uint8_t* out = packed + tile * TILE_BYTES;
    const int64_t row = rt * TILE_ROWS + r, col = kt * TILE_COLS + g * 32 + c * 8;
    uint32_t codes = 0u;                                // nibble i = column col + i
    if (row < rows && col < cols)
        codes = *reinterpret_cast<const uint32_t*>(q + (m * rows + row) * cols + col / 16 * 16 + (col % 16) / 2);
    constexpr int SIGN[4] = {15, 12, 14, 13}, VALUE[4] = {6, 3, 0, 9};
    uint32_t word = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t code = codes >> (4 * i);
        word |= ((code >> 3 & 1u) << SIGN[i / 2] | (code & 7u) << VALUE[i / 2]) << (16 * (i & 1));
    }
    reinterpret_cast<uint32_t*>(out)[t] = word;
    if (t < 64) {
        const int64_t srow = rt * TILE_ROWS + t / 4, group = kt * 4 + t % 4;
        out[TILE_CODES + t] = (srow < rows && group * 32 < cols) ? s[(m * rows + srow) * (cols / 32) + group] : (uint8_t)0;
    }
}

}  // namespace
}  // namespace mxfp8

using namespace mxfp8;

extern "C" size_t mxfp8_e2m1_packed_bytes(int64_t num_matrices, int64_t rows, int64_t cols)
{
    if (num_matrices <= 0 || rows <= 0 || cols <= 0) return 0;
    return (size_t)num_matrices * (size_t)((rows + TILE_ROWS - 1) / TILE_ROWS) * (size_t)((cols + TILE_COLS - 1) / TILE_COLS) * TILE_BYTES;
}

extern "C" int mxfp8_e2m1_pack(const void* q, const void* s, int64_t num_matrices, int64_t rows, int64_t cols, void* packed, void* stream)
{
    if (!q || !s || !packed) return MXFP8_ERR_NULL;
    if (num_matrices <= 0 || rows <= 0 || cols <= 0 || (cols % 32)) return MXFP8_ERR_SHAPE;
    if (!aligned16(q) || !aligned16(packed)) return MXFP8_ERR_ALIGN;
    const int64_t rt = (rows + TILE_ROWS - 1) / TILE_ROWS, kt = (cols + TILE_COLS - 1) / TILE_COLS;
    if (rt > 0x7FFFFFFFLL || kt > 0x7FFFFFFFLL || rt * kt > 0x7FFFFFFFLL / num_matrices) return MXFP8_ERR_UNSUPPORTED;
    e2m1_pack_kernel<<<(unsigned)(rt * kt * num_matrices), 256, 0, static_cast<cudaStream_t>(stream)>>>(
        static_cast<const uint8_t*>(q), static_cast<const uint8_t*>(s), static_cast<uint8_t*>(packed), rows, cols, rt, kt);
    count_launch(1);
    return cudaGetLastError() == cudaSuccess ? MXFP8_OK : MXFP8_ERR_CUDA;
}

extern "C" int mxfp8_e2m1_matvec(const void* x, int64_t tokens, int64_t cols, const void* packed, int64_t num_matrices, int64_t rows,
                                 const int32_t* matrix_ids, int slots_per_token, void* y, int y_dtype, void* stream)
{
    if (y_dtype != MXFP8_FP32 && y_dtype != MXFP8_BF16) return MXFP8_ERR_ENUM;
    if (!x || !packed || !y) return MXFP8_ERR_NULL;
    if (tokens <= 0 || rows <= 0 || cols <= 0 || (cols % 32) || num_matrices <= 0 || slots_per_token < 1) return MXFP8_ERR_SHAPE;
    if (!matrix_ids && (num_matrices != 1 || slots_per_token != 1)) return MXFP8_ERR_SHAPE;
    if (!aligned16(x) || !aligned16(packed)) return MXFP8_ERR_ALIGN;
    if ((reinterpret_cast<uintptr_t>(y) % (y_dtype == MXFP8_BF16 ? 2 : 4)) || (reinterpret_cast<uintptr_t>(matrix_ids) & 3u)) return MXFP8_ERR_ALIGN;
    if (tokens > MV_MAX_SLOTS || tokens * slots_per_token > MV_MAX_SLOTS || num_matrices > 65535) return MXFP8_ERR_UNSUPPORTED;
    MatvecArgs a{};
    const int64_t rt = (rows + TILE_ROWS - 1) / TILE_ROWS, kt = (cols + TILE_COLS - 1) / TILE_COLS;
    if (rt > 0x7FFFFFFLL || kt > 0x7FFFFFFLL) return MXFP8_ERR_UNSUPPORTED;
    a.x = static_cast<const __nv_bfloat16*>(x);
    a.packed = static_cast<const uint8_t*>(packed);
    a.ids = matrix_ids; a.y = y;
    a.slots = (int)(tokens * slots_per_token); a.per_token = slots_per_token; a.matrices = (int)num_matrices;
    a.rows = rows; a.cols = cols; a.row_tiles = (int)rt; a.col_tiles = (int)kt;
    a.by_matrix = matrix_ids && num_matrices < a.slots;
    const unsigned grid_y = (unsigned)(!matrix_ids ? 1 : (a.by_matrix ? num_matrices : a.slots));
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const cudaError_t err = y_dtype == MXFP8_BF16 ? launch_matvec<__nv_bfloat16>(a, grid_y, st) : launch_matvec<float>(a, grid_y, st);
    return err == cudaSuccess ? MXFP8_OK : MXFP8_ERR_CUDA;
}
