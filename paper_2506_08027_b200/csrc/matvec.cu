// Products of a few tokens with E2M1 (MXFP4) matrices: the conversion's 4-bit codes and UE8M0 scales (Sec. 2, Table 1) as
// stored weights, BF16 activations, FP32 sums.  One matrix for all tokens or one chosen per (token, choice) slot, which
// is what a mixture-of-experts layer (App. A.4) computes when it answers a few tokens.
//
//   y[s, n] = sum over groups g of 32 columns of  2^(b[n,g] - 127) * sum_{k in g} code[n,k] * x[s / slots_per_token, k]
//
// Bound by the weight bytes: 17/32 byte per weight, read once.  The codes become BF16 registers (exact) and go through
// the warp-level tensor instructions with the tokens as the narrow side.  (The block-scaled tensor instructions would take the
// 4-bit codes as they are, but not BF16 activations.)
//
// Packed layout: a matrix of N rows and K columns is cut into tiles of 16 rows x 128 columns, column tiles innermost,
// rows and columns padded with zero codes under zero scale bytes.  A tile is 1088 bytes:
//   1024 bytes of codes: words of 8 codes, word (h, r, c, g) for row 8h + r, columns 32 g + 8 c .. + 7 of the tile, at
//        ((h * 8 + r) * 4 + c) * 4 + g: lane (r, c) of a warp finds its words of the four groups in 16 bytes.
//        In a word the even columns lie in the low half, the odd ones in the high half; columns 2p, 2p + 1 have their sign
//        at bit 15, 12, 14, 13 and their three value bits from bit 6, 3, 0, 9 of the half for p = 0, 1, 2, 3.
//   64 bytes of scales: byte 4 r + g for row r, group g.
// A BF16 number whose three value bits are its two lowest exponent bits and its highest mantissa bit (bits 8 .. 6) and whose
// other exponent bits are zero is the E2M1 value times 2^-126, subnormals included: two shifts and two masks at most
// and one exact product by 2^126 turn a pair of codes into a register of two BF16 values.
#include "mxfp8_device.cuh"
#include "mxfp8_host.h"

namespace mxfp8 {
namespace {

constexpr int TILE_ROWS = 16, TILE_COLS = 128, TILE_CODES = 1024, TILE_BYTES = 1088;
constexpr int MV_WARPS = 8, MV_THREADS = 32 * MV_WARPS;
constexpr int MV_MAX_SLOTS = 1024;       // (token, choice) pairs of one call

struct MatvecArgs {
    const __nv_bfloat16* x;      // [tokens, cols]
    const uint8_t* packed;       // [matrices][row tiles][column tiles][1088]
    const int32_t* ids;          // [slots] or null: matrix 0 for all
    void* y;                     // [slots, rows]
    int slots, per_token, matrices;
    int64_t rows, cols;
    int row_tiles, col_tiles;
};

// Code pairs p = 0 .. 3 of a word as BF16 pairs (column 2p in the low half).
__device__ __forceinline__ void decode_word(uint32_t w, uint32_t (&out)[4])
{
    constexpr uint32_t V = 0x01C001C0u, S = 0x80008000u;
    out[0] = w & (V | S);
    out[1] = (w << 3) & (V | S);
    out[2] = ((w << 6) & V) | ((w << 1) & S);
    out[3] = ((w >> 3) & V) | ((w << 2) & S);
    const __nv_bfloat162 up = __halves2bfloat162(__ushort_as_bfloat16(0x7E80), __ushort_as_bfloat16(0x7E80));      // 2^126
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const __nv_bfloat162 v = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&out[p]), up);
        out[p] = *reinterpret_cast<const uint32_t*>(&v);
    }
}

__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// 2^(b - 127): b = 0 is the subnormal 2^-127, b = 255 is NaN
__device__ __forceinline__ float scale_value(uint32_t b)
{
    return __uint_as_float(b == 0u ? 0x00400000u : (b == 255u ? 0x7FC00000u : b << 23));
}

template <typename T> __device__ __forceinline__ T to_out(float v);
template <> __device__ __forceinline__ float to_out<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 to_out<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// CTA (i, u): 16 rows of a matrix times the slots that chose it, eight at a time; the eight warps split the columns and
// add their sums in a fixed order.  u counts slots (the first slot with a matrix works for all of them, the others
// leave) or, where there are fewer matrices than slots, matrices.
template <typename OUT>
__global__ void __launch_bounds__(MV_THREADS) matvec_kernel(const MatvecArgs a, int by_matrix)
{
    __shared__ int list[MV_MAX_SLOTS];
    __shared__ float sums[MV_WARPS][TILE_ROWS][9];      // 8 tokens per row, padded
    __shared__ int listed;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, u = blockIdx.y;
    int matrix = 0;
    if (a.ids == nullptr) {
        for (int i = tid; i < a.slots; i += MV_THREADS) list[i] = i;
        if (tid == 0) listed = a.slots;
    } else {
        matrix = by_matrix ? u : a.ids[u];
        if ((unsigned)matrix >= (unsigned)a.matrices) {
            // no such matrix: this slot's rows are zero
            const int64_t n = (int64_t)blockIdx.x * TILE_ROWS + tid;
            if (tid < TILE_ROWS && n < a.rows) static_cast<OUT*>(a.y)[(int64_t)u * a.rows + n] = to_out<OUT>(0.f);
            return;
        }
        if (warp == 0) {
            int count = 0, first = -1;
            for (int base = 0; base < a.slots; base += 32) {
                const int s = base + lane;
                const unsigned hit = __ballot_sync(0xFFFFFFFFu, s < a.slots && a.ids[min(s, a.slots - 1)] == matrix);
                if (hit && first < 0) first = base + __ffs(hit) - 1;
                if (hit >> lane & 1u) list[count + __popc(hit & ((1u << lane) - 1u))] = s;
                count += __popc(hit);
            }
            if (lane == 0) listed = (by_matrix || first == u) ? count : 0;
        }
        if (by_matrix && blockIdx.y == 0) {             // slots without a matrix: theirs are zero
            const int64_t n = (int64_t)blockIdx.x * TILE_ROWS + (tid & 15);
            for (int s = tid >> 4; s < a.slots; s += MV_THREADS / 16)
                if ((unsigned)a.ids[s] >= (unsigned)a.matrices && n < a.rows) static_cast<OUT*>(a.y)[(int64_t)s * a.rows + n] = to_out<OUT>(0.f);
        }
    }
    __syncthreads();
    const int count = listed;
    const int row = lane >> 2, quarter = lane & 3;      // of the tensor instructions' operands
    const uint8_t* tiles = a.packed + ((int64_t)matrix * a.row_tiles + blockIdx.x) * a.col_tiles * TILE_BYTES;
    for (int s0 = 0; s0 < count; s0 += 8) {
        const bool has = s0 + row < count;
        const __nv_bfloat16* x = a.x + (has ? (int64_t)(list[s0 + row] / a.per_token) * a.cols : 0) + quarter * 8;
        float acc[4] = {0.f, 0.f, 0.f, 0.f};
        for (int kt = warp; kt < a.col_tiles; kt += MV_WARPS) {
            const uint8_t* tile = tiles + (int64_t)kt * TILE_BYTES;
            const uint4 lo = *reinterpret_cast<const uint4*>(tile + lane * 16), hi = *reinterpret_cast<const uint4*>(tile + 512 + lane * 16);
            const uint32_t s_lo = *reinterpret_cast<const uint32_t*>(tile + TILE_CODES + row * 4), s_hi = *reinterpret_cast<const uint32_t*>(tile + TILE_CODES + 32 + row * 4);
            const uint32_t w_lo[4] = {lo.x, lo.y, lo.z, lo.w}, w_hi[4] = {hi.x, hi.y, hi.z, hi.w};
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int64_t k = (int64_t)kt * TILE_COLS + g * 32;
                uint4 b = make_uint4(0u, 0u, 0u, 0u);
                if (has && k < a.cols) b = *reinterpret_cast<const uint4*>(x + k);
                uint32_t al[4], ah[4];
                decode_word(w_lo[g], al);
                decode_word(w_hi[g], ah);
                float d[4] = {0.f, 0.f, 0.f, 0.f};
                mma_bf16(d, al[0], ah[0], al[1], ah[1], b.x, b.y);
                mma_bf16(d, al[2], ah[2], al[3], ah[3], b.z, b.w);
                const float f_lo = scale_value(s_lo >> (8 * g) & 255u), f_hi = scale_value(s_hi >> (8 * g) & 255u);
                acc[0] = fmaf(f_lo, d[0], acc[0]);
                acc[1] = fmaf(f_lo, d[1], acc[1]);
                acc[2] = fmaf(f_hi, d[2], acc[2]);
                acc[3] = fmaf(f_hi, d[3], acc[3]);
            }
        }
        sums[warp][row][2 * quarter] = acc[0];
        sums[warp][row][2 * quarter + 1] = acc[1];
        sums[warp][row + 8][2 * quarter] = acc[2];
        sums[warp][row + 8][2 * quarter + 1] = acc[3];
        __syncthreads();
        if (tid < 8 * TILE_ROWS) {
            const int r = tid & 15, j = tid >> 4;
            const int64_t n = (int64_t)blockIdx.x * TILE_ROWS + r;
            float v = 0.f;
#pragma unroll
            for (int w = 0; w < MV_WARPS; ++w) v += sums[w][r][j];
            if (s0 + j < count && n < a.rows) static_cast<OUT*>(a.y)[(int64_t)list[s0 + j] * a.rows + n] = to_out<OUT>(v);
        }
        __syncthreads();
    }
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
    if (rt > 0x7FFFFFFFLL || kt > 0x7FFFFFFFLL / MV_THREADS) return MXFP8_ERR_UNSUPPORTED;
    a.x = static_cast<const __nv_bfloat16*>(x);
    a.packed = static_cast<const uint8_t*>(packed);
    a.ids = matrix_ids; a.y = y;
    a.slots = (int)(tokens * slots_per_token); a.per_token = slots_per_token; a.matrices = (int)num_matrices;
    a.rows = rows; a.cols = cols; a.row_tiles = (int)rt; a.col_tiles = (int)kt;
    const int by_matrix = matrix_ids && num_matrices < a.slots;
    const dim3 grid((unsigned)rt, (unsigned)(!matrix_ids ? 1 : (by_matrix ? num_matrices : a.slots)));
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (y_dtype == MXFP8_BF16) matvec_kernel<__nv_bfloat16><<<grid, MV_THREADS, 0, st>>>(a, by_matrix);
    else matvec_kernel<float><<<grid, MV_THREADS, 0, st>>>(a, by_matrix);
    count_launch(1);
    return cudaGetLastError() == cudaSuccess ? MXFP8_OK : MXFP8_ERR_CUDA;
}
