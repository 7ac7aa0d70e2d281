// mxfp8_moe_dispatch_quantize: the conversion of rows gathered by an index (tokens in the order of their experts, App. A.4),
// optionally weighted.  Tile, slab and order of the scale bytes are those of the fast path (quantize_tma_kernel.cuh), and so
// is the careful path for slabs with Inf or NaN or columns behind the tensor; the rest is made for rows that mostly come from L2,
// where the conversion's instructions, not its bytes, set the pace:
//   loads  : a warp fetches its own 32-row slab with 16-byte asynchronous copies, two rows per instruction, straight from
//            the tokens' rows (a gathering tensor copy was tried first: its issue runs through the lanes one by one, some
//            2000 cycles of one warp per tile with the other three waiting: 88 us for the row-blocked copy of 53248 x 2048
//            rows against 55 us with these copies and all else alike).  Rows without a slot and columns behind the tensor are zero-filled by the copies.
//   order  : slots of the tile after next are asked for under the current slab, its copies go out as soon as the slab
//            is done; no warp waits for another but the one that stores a tile's scale bytes, a different one each tile
//   rows   : lane r takes the whole of row r, 16 bytes at a time: weights it (one FP32 product and one rounding per element,
//            back in place) and finds the row's block maxima without a shuffle; 16-byte piece c of row r lies at c ^ (r mod
//            16), so that this walk and the walk by columns both read shared memory without conflicts
//   columns: lane l owns 8 bytes of every row, as in the fast path; the 32 rows stay in registers for the conversion
//   cast   : products of two elements per instruction
// Measured at 53248 x 2048 BF16 rows of 8192 tokens, top-6, with the HBM time of the tokens read once and the outputs written:
// 38 us for the row-blocked copy (22), 37 us by columns (22), 53 us for both (39), 63 us for both with weights; mxfp8_quantize
// of the same rows already sorted takes 88 us for both.  6272 x 4096 FP32 rows of 2999 tokens, weighted, both: 26.4 us (15).
// No unit is at its limit: for both from BF16 the integer pipe, the busiest, is taken 62 % of the cycles, a multiprocessor issues 2.45
// of four instructions a cycle from twelve warps, L2 works at 42 % of its throughput and HBM at 46 %.  One slab per warp instead of two, with 16 warps on a multiprocessor instead of 12, took 10 % more by columns and
// 2 % less for both; 20 warps spill.
#include "quantize_tma_kernel.cuh"

namespace mxfp8 {
namespace {

// Order of the tiles.  A token is read once per expert that it went to, from L2 as long as the tokens stay there.  Up to
// ONE_GROUP bytes of tokens the tiles are taken by rows; larger sources in groups of tile columns under which the tokens
// have at most GROUP_BYTES, in a group by rows.  Top-6, by rows | in groups, us: 16384 x 4096 BF16, row-blocked 196 | 139, both
// copies 284 | 246; 8192 x 4096 BF16 both 131 | 120, row-blocked 74.5 | 73.7; 8192 x 2048 FP32 both 84.6 | 84.6, row-blocked
// 63.7 | 67.2 (64 MiB: one copy alone stays by rows).  Groups of 32 and 40 MiB take 1 % less to 4 % more.
template <bool BOTH> constexpr int64_t ONE_GROUP = (int64_t)(BOTH ? 48 : 64) << 20;
constexpr int64_t GROUP_BYTES = (int64_t)24 << 20;
// Both copies together push the tokens out of L2 before their last expert has read them, unless the codes leave first: the call alone
// takes 53 us in place of 57 for 8192 tokens, top-6, 2048 BF16 columns (one copy alone is 2 % faster without: 38.1 us, 38.9).  The
// products that follow read the codes, though, so the codes of up to FIRST_OUT_BYTES, which L2 can hold in part, stay: weighted
// conversion, DGRAD and WGRAD together 153.9 us with codes that leave first | 152.2 without, of 512 tokens, 175.0 | 173.2 of 1024,
// 221.9 | 220.3 of 2048, 312.2 | 310.9 of 4096 (conversion and FPROP 0 to 0.7 % less; from FP32 0.6 to 1.8 % less).  From 8192 tokens on (200 MB of codes) the
// two are within 0.6 % of each other either way, and 24576 tokens of 4096 columns take 0.2 to 0.7 % less with codes that leave first.
constexpr int64_t FIRST_OUT_BYTES = (int64_t)128 << 20;
struct Walk {
    uint32_t group, group_magic, last, last_magic;     // tile columns of a group and of the last one
    int groups;
};
struct GatherArgs {
    QParams t;                                // the converted tensor [rows, cols]
    const void* src;                          // [tokens, cols]
    const int32_t* slot_of;                   // slot of every row, -1: none
    const float* weights;                     // per slot, or null
    const int32_t* used;                      // device: rows in use
    int* status;                              // reports a bad array
    uint32_t top_k, top_k_magic, slots;       // slots per token and of all tokens
    int tiles;                                // of all rows
};
constexpr int SLAB_BYTES = 32 * T_BYTES;
// Scale bytes of the last eight tiles.  Warp i mod 4 stores those of the CTA's i-th tile once it has converted its slab of
// tile i + 1, by when the other three have mostly announced their slabs of tile i and need not be waited for (waiting right
// behind tile i cost 9 % of the warps' time, 15 % from FP32).  Why eight buffers and barriers are enough: when a warp writes
// the bytes of tile i + 8, the last tile m that it stored is at least i + 3, so all others had announced tile m, and who
// stored tile i had done so before it announced tile i + 1 or any later one.
constexpr int STORERS = QT_THREADS / 32, STAGES = 8;

// The larger magnitude of each half; the sign bits are of no meaning.  A NaN gives way to the other operand.
__device__ __forceinline__ uint32_t max_magnitude2(uint32_t a, uint32_t b)
{
    uint32_t m;
    asm("max.xorsign.abs.bf16x2 %0, %1, %2;" : "=r"(m) : "r"(a), "r"(b));
    return m;
}
// Two FP32 products, each rounded to nearest even
__device__ __forceinline__ float2 mul2(float2 a, float2 b)
{
    float2 d;
    asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmul.rn.f32x2 z, x, y;\n\tmov.b64 {%0, %1}, z;\n\t}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ float2 bf16_pair(uint32_t w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u)); }
__device__ __forceinline__ uint32_t weigh_pair(uint32_t w, float f)
{
    const float2 p = mul2(bf16_pair(w), make_float2(f, f));
    const __nv_bfloat162 r = __floats2bfloat162_rn(p.x, p.y);
    return *reinterpret_cast<const uint32_t*>(&r);
}

// A slab lies at a multiple of 256 bytes of shared memory, so that the place of a piece is an exclusive-or of an address that
// the lane computes once with a constant.
template <typename T> __device__ __forceinline__ T& shared_at(uint32_t address) { return *static_cast<T*>(__cvta_shared_to_generic(address)); }
// The 8 bytes of row j that belong to this lane, from own = own_bytes(slab, lane)
__device__ __forceinline__ uint32_t own_bytes(uint32_t slab, int lane) { return slab | (lane >> 1) << 4 | (lane & 1) << 3; }
__device__ __forceinline__ uint32_t in_row(uint32_t own, int j) { return (own ^ (j & 15) << 4) + j * T_BYTES; }
// Piece c of this lane's row, from row = own_row(slab, lane)
__device__ __forceinline__ uint32_t own_row(uint32_t slab, int lane) { return slab + lane * T_BYTES + (lane & 15) * 16; }
__device__ __forceinline__ uint32_t piece(uint32_t row, int c) { return row ^ c << 4; }

// First walk: row `lane` of the slab is weighted in place and its block maxima become scale bytes (staged) and factors 1/X
// (in `inv`, four per row).  Returns whether a maximum is Inf (NaN elements do not enter it).
template <int DTYPE, int ELEM, bool DO_ROW>
__device__ __forceinline__ bool walk_row(uint32_t slab, float* inv, float weight, bool weighted, uint8_t* my_scales, int lane, uint32_t rule_offset)
{
    constexpr bool BF = (DTYPE == MXFP8_BF16);
    constexpr int NKB = BF ? 4 : 2, PIECES = 16 / NKB;       // blocks of the row, pieces of a block
    const uint32_t row = own_row(slab, lane);
    uint32_t top[NKB];
#pragma unroll
    for (int b = 0; b < NKB; ++b) {
        uint32_t m = 0u;
        float f = 0.f;
#pragma unroll
        for (int c = 0; c < PIECES; ++c) {
            uint4& at = shared_at<uint4>(piece(row, b * PIECES + c));
            uint4 v = at;
            if (weighted) {
                if constexpr (BF) {
                    v.x = weigh_pair(v.x, weight); v.y = weigh_pair(v.y, weight);
                    v.z = weigh_pair(v.z, weight); v.w = weigh_pair(v.w, weight);
                } else {
                    const float2 w2 = make_float2(weight, weight);
                    const float2 lo = mul2(make_float2(__uint_as_float(v.x), __uint_as_float(v.y)), w2);
                    const float2 hi = mul2(make_float2(__uint_as_float(v.z), __uint_as_float(v.w)), w2);
                    v = make_uint4(__float_as_uint(lo.x), __float_as_uint(lo.y), __float_as_uint(hi.x), __float_as_uint(hi.y));
                }
                at = v;
            }
            if constexpr (!DO_ROW) continue;
            if constexpr (BF) m = max_magnitude2(max_magnitude2(max_magnitude2(max_magnitude2(m, v.x), v.y), v.z), v.w);
            else f = fmaxf(fmaxf(f, fmaxf(fabsf(__uint_as_float(v.x)), fabsf(__uint_as_float(v.y)))),
                           fmaxf(fabsf(__uint_as_float(v.z)), fabsf(__uint_as_float(v.w))));
        }
        if constexpr (BF) top[b] = max(m & 0x7FFFu, (m >> 16) & 0x7FFFu);
        else top[b] = __float_as_uint(f);
    }
    if constexpr (!DO_ROW) return false;
    if constexpr (BF) {
        const uint32_t z01 = top[0] | (top[1] << 16), z23 = top[NKB - 2] | (top[NKB - 1] << 16), off2 = (rule_offset >> 16) * 0x00010001u;
        const uint32_t e01 = inv_exp_field2<ELEM>(z01, off2), e23 = inv_exp_field2<ELEM>(z23, off2);
        *reinterpret_cast<uint32_t*>(my_scales) = __byte_perm(0x00FE00FEu - e01, 0x00FE00FEu - e23, 0x6420);
        *reinterpret_cast<float4*>(inv + lane * 4) = make_float4(__uint_as_float(e01 << 23), __uint_as_float((e01 & 0xFFFF0000u) << 7),
                                                                  __uint_as_float(e23 << 23), __uint_as_float((e23 & 0xFFFF0000u) << 7));
        return (nonfinite2(z01) | nonfinite2(z23)) != 0u;
    } else {
        const uint32_t e0 = inv_exp_field<ELEM>(top[0], rule_offset), e1 = inv_exp_field<ELEM>(top[1], rule_offset);
        *reinterpret_cast<uint16_t*>(my_scales) = (uint16_t)((254u - e0) | (254u - e1) << 8);
        *reinterpret_cast<float2*>(inv + lane * 4) = make_float2(__uint_as_float(e0 << 23), __uint_as_float(e1 << 23));
        return top[0] == 0x7F800000u || top[1] == 0x7F800000u;
    }
}

// This lane's VEC elements of a row times the factors, as codes (FIRST_OUT: they leave L2 before anything else; see FIRST_OUT_BYTES)
template <int ELEM, int VEC, bool FIRST_OUT>
__device__ __forceinline__ void store_codes(uint8_t* to, const float2 (&x)[VEC / 2], const float2 (&f)[VEC / 2], int lane)
{
    constexpr bool SUB = (ELEM != MXFP8_E4M3 && ELEM != MXFP8_E5M2);
    if constexpr (VEC == 4) {
        const float2 a = mul2(x[0], f[0]), b = mul2(x[1], f[1]);
        uint32_t c;
        if constexpr (ELEM == MXFP8_E4M3)      // one block: the two conversions are moved into one register by one instruction
            asm("{\n\t.reg .b16 l, h;\n\tcvt.rn.satfinite.e4m3x2.f32 l, %2, %1;\n\tcvt.rn.satfinite.e4m3x2.f32 h, %4, %3;\n\tmov.b32 %0, {l, h};\n\t}"
                : "=r"(c) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
        else if constexpr (ELEM == MXFP8_E5M2)
            asm("{\n\t.reg .b16 l, h;\n\tcvt.rn.satfinite.e5m2x2.f32 l, %2, %1;\n\tcvt.rn.satfinite.e5m2x2.f32 h, %4, %3;\n\tmov.b32 %0, {l, h};\n\t}"
                : "=r"(c) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
        else c = cvt_fp8x4<ELEM>(a.x, a.y, b.x, b.y);
        if constexpr (SUB) c = pack_slot<ELEM, VEC>(c, lane);
        if constexpr (FIRST_OUT) __stcs(reinterpret_cast<uint32_t*>(to), c);
        else *reinterpret_cast<uint32_t*>(to) = c;
    } else {
        const float2 a = mul2(x[0], f[0]);
        uint32_t c = cvt_fp8x2<ELEM>(a.x, a.y);
        if constexpr (SUB) c = pack_slot<ELEM, VEC>(c, lane);
        if constexpr (FIRST_OUT) __stcs(reinterpret_cast<uint16_t*>(to), (uint16_t)c);
        else *reinterpret_cast<uint16_t*>(to) = (uint16_t)c;
    }
}

// One slab whose columns all lie inside the tensor.  Returns true, with nothing stored but staged scale bytes, when an Inf
// takes part (or a whole column of NaN); the slab then holds the weighted rows.
template <int DTYPE, int ELEM, bool DO_ROW, bool DO_COL, bool FIRST_OUT>
__device__ __forceinline__ bool convert_slab(uint32_t slab, float* inv, uint8_t* my_qrow, uint8_t* my_qcol, uint32_t pitch, uint8_t* my_row_scales,
                                             uint8_t* my_sm_col, float weight, bool weighted, int lane, uint32_t rule_offset)
{
    constexpr bool BF = (DTYPE == MXFP8_BF16);
    constexpr int VEC = BF ? 4 : 2;
    bool special = false;
    if (DO_ROW || weighted) {
        special = walk_row<DTYPE, ELEM, DO_ROW>(slab, inv, weight, weighted, my_row_scales, lane, rule_offset);
        __syncwarp();
    }
    const uint32_t own = own_bytes(slab, lane);
    uint2 raw[DO_COL ? 32 : 1];
    float2 col[VEC / 2];
    if constexpr (DO_COL) {
        uint32_t bits[VEC];
        if constexpr (BF) {
            uint32_t m0 = 0u, m1 = 0u;
#pragma unroll
            for (int j = 0; j < 32; ++j) {
                raw[j] = shared_at<const uint2>(in_row(own, j));
                m0 = max_magnitude2(m0, raw[j].x);
                m1 = max_magnitude2(m1, raw[j].y);
            }
            bits[0] = (m0 & 0x7FFFu) << 16; bits[1] = m0 & 0x7FFF0000u;
            bits[2] = (m1 & 0x7FFFu) << 16; bits[3] = m1 & 0x7FFF0000u;
        } else {
            float m0 = 0.f, m1 = 0.f;
#pragma unroll
            for (int j = 0; j < 32; ++j) {
                raw[j] = shared_at<const uint2>(in_row(own, j));
                m0 = fmaxf(m0, fabsf(__uint_as_float(raw[j].x)));
                m1 = fmaxf(m1, fabsf(__uint_as_float(raw[j].y)));
            }
            bits[0] = __float_as_uint(m0); bits[1] = __float_as_uint(m1);
        }
        float f[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            special = special || bits[i] >= 0x7F800000u;
            const uint32_t e = inv_exp_field<ELEM>(bits[i], rule_offset);
            f[i] = __uint_as_float(e << 23);
            my_sm_col[i * STAGE_PITCH] = (uint8_t)(254u - e);
        }
#pragma unroll
        for (int i = 0; i < VEC / 2; ++i) col[i] = make_float2(f[2 * i], f[2 * i + 1]);
    }
    if (__any_sync(0xFFFFFFFFu, special)) return true;
#pragma unroll
    for (int j = 0; j < 32; ++j) {
        uint2 w;
        if constexpr (DO_COL) w = raw[j];
        else w = shared_at<const uint2>(in_row(own, j));
        float2 x[VEC / 2];
        if constexpr (BF) {
            x[0] = bf16_pair(w.x);
            x[VEC / 2 - 1] = bf16_pair(w.y);
        } else x[0] = make_float2(__uint_as_float(w.x), __uint_as_float(w.y));
        if constexpr (DO_ROW) {
            const float r = inv[j * 4 + lane / (32 / VEC)];
            float2 f[VEC / 2];
#pragma unroll
            for (int i = 0; i < VEC / 2; ++i) f[i] = make_float2(r, r);
            store_codes<ELEM, VEC, FIRST_OUT>(my_qrow + (uint64_t)j * pitch, x, f, lane);
        }
        if constexpr (DO_COL) store_codes<ELEM, VEC, FIRST_OUT>(my_qcol + (uint64_t)j * pitch, x, col, lane);
    }
    return false;
}

// The slab back in plain order, for the careful path
__device__ __noinline__ void plain_order(uint32_t slab, int lane)
{
    const uint32_t own = own_bytes(slab, lane);
    for (int j = 0; j < 32; ++j) {
        const uint2 v = shared_at<const uint2>(in_row(own, j));
        __syncwarp();
        shared_at<uint2>(slab + j * T_BYTES + lane * 8) = v;
        __syncwarp();
    }
}

// A quarter of the scale bytes of one tile, row and column `tid` of it, leaves from the staging arrays (both in the order of a
// swizzled atom).  A tile's rows are all inside the tensor, its columns may not be.  (The fast path's kernel has such code inside:
// shared between the two as a function, it cost that kernel up to 10 %, 15.3 against 16.7 us for both copies of 4096 x 4096 BF16.)
template <bool BF, bool DO_ROW, bool DO_COL>
__device__ __forceinline__ void store_scales(const QParams& p, int tile_x, int tile_y, const uint8_t* sm_row, const uint8_t* sm_col, int tid, int lane, int quarter)
{
    constexpr int T_COLS = T_BYTES / (BF ? 2 : 4), NKB = T_COLS / 32;
    const int64_t gcol0 = (int64_t)tile_x * T_COLS;
    if (BF && p.sf_layout == MXFP8_SF_SWIZZLED && gcol0 + T_COLS <= p.cols) {      // exactly one atom per orientation, 16 bytes per lane
        if (DO_ROW && quarter == 0) {
            const int64_t atoms_k = ((p.cols >> 5) + 3) >> 2;
            *reinterpret_cast<uint4*>(p.s_row + ((int64_t)tile_y * atoms_k + tile_x) * 512 + lane * 16) = *reinterpret_cast<const uint4*>(sm_row + lane * 16);
        }
        if (DO_COL && quarter == (DO_ROW ? 1 : 0))
            *reinterpret_cast<uint4*>(p.s_col + ((int64_t)tile_x * (p.rows >> 7) + tile_y) * 512 + lane * 16) = *reinterpret_cast<const uint4*>(sm_col + lane * 16);
        return;
    }
    if constexpr (DO_ROW) {
        const int64_t r = (int64_t)tile_y * T_ROWS + tid, blocks = p.cols >> 5, kb0 = (int64_t)tile_x * NKB;
        const int nkb = (int)min((int64_t)NKB, blocks - kb0);
        uint32_t v = *reinterpret_cast<const uint32_t*>(sm_row + stage_offset(tid));
        if (nkb < 4) v &= (1u << (8 * nkb)) - 1u;          // bytes behind the last block are zero
        if (p.sf_layout == MXFP8_SF_SWIZZLED) {
            // a 64-column FP32 tile owns half of the atom's four blocks; without a right neighbour it clears that half too
            uint8_t* d = p.s_row + ((int64_t)tile_y * ((blocks + 3) >> 2) + (kb0 >> 2)) * 512 + stage_offset(tid) + (kb0 & 3);
            if (NKB == 4 || ((kb0 & 3) == 0 && kb0 + NKB >= blocks)) *reinterpret_cast<uint32_t*>(d) = v;
            else *reinterpret_cast<uint16_t*>(d) = (uint16_t)v;
        } else {
            uint8_t* d = p.s_row + r * blocks + kb0;
            for (int kb = 0; kb < nkb; ++kb) d[kb] = (uint8_t)(v >> (8 * kb));
        }
    }
    if (DO_COL && tid < T_COLS) {
        const int64_t c = gcol0 + tid, atoms_r = p.rows >> 7;
        const uint32_t v = c < p.cols ? *reinterpret_cast<const uint32_t*>(sm_col + stage_offset(tid)) : 0u;
        if (p.sf_layout == MXFP8_SF_SWIZZLED) {
            const int64_t padded_cols = ((p.cols + 127) >> 7) << 7;
            *reinterpret_cast<uint32_t*>(p.s_col + ((c >> 7) * atoms_r + tile_y) * 512 + (c & 31) * 16 + ((c >> 5) & 3) * 4) = v;
            // columns of the atom that no 64-column FP32 tile covers
            if (T_COLS == 64 && tile_x == p.tiles_x - 1 && c + 64 < padded_cols)
                *reinterpret_cast<uint32_t*>(p.s_col + (((c + 64) >> 7) * atoms_r + tile_y) * 512 + ((c + 64) & 31) * 16 + (((c + 64) >> 5) & 3) * 4) = 0u;
        } else if (c < p.cols) {
            for (int w = 0; w < 4; ++w) p.s_col[((int64_t)tile_y * 4 + w) * p.cols + c] = (uint8_t)(v >> (8 * w));
        }
    }
}

template <int DTYPE, int ELEM, bool DO_ROW, bool DO_COL, bool GROUPED, bool FIRST_OUT>
__global__ void __launch_bounds__(QT_THREADS, QT_CTAS_PER_SM)
quantize_gather_kernel(const __grid_constant__ GatherArgs a, const Walk walk)
{
    constexpr bool BF = (DTYPE == MXFP8_BF16);
    constexpr int VEC = BF ? 4 : 2;                 // elements per lane per row
    constexpr int ESZ = BF ? 2 : 4;
    constexpr int T_COLS = T_BYTES / ESZ;           // 128 or 64
    constexpr int LPB = 32 / VEC;                   // lanes per row block: 8 or 16

    extern __shared__ __align__(256) uint8_t gather_smem[];
    uint8_t* sm_scales = gather_smem + RING * IN_BYTES;    // STAGES x (row scales + column scales of one tile, 512 bytes each)
    float* row_inv = reinterpret_cast<float*>(sm_scales + STAGES * 1024) + (threadIdx.x >> 5) * 128;      // this warp's row factors, four per row

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;   // warp = 32-row slab of the tile
    const QParams& p = a.t;
    const uint32_t rule_offset = (p.rule == MXFP8_RULE_PAPER) ? paper_offset<ELEM>() : 0u;
    const uint32_t my_slabs = smem_addr(gather_smem) + warp * SLAB_BYTES;   // + IN_BYTES for the ring's second slot

    // rows in use: whole 128-row tiles by construction of the sort; anything else is reported and nothing is stored
    const int used = *a.used;
    int num_tiles = 0;
    if (used < 0 || used > p.rows || used % T_ROWS) {
        if (tid == 0 && blockIdx.x == 0) atomicExch(a.status, (int)MXFP8_ERR_DEVICE_ARGS);
    } else num_tiles = (used / T_ROWS) * p.tiles_x;

    [[maybe_unused]] const uint32_t group = walk.group * (uint32_t)(num_tiles ? used / T_ROWS : 1);      // tiles of a whole group
    [[maybe_unused]] const uint32_t group_magic = GROUPED ? div_magic(group) : 0u;
    auto locate = [&](int t, int& y, int& x) {
        if constexpr (GROUPED) {
            int g, in, rest;
            divmod((uint32_t)t, group, group_magic, g, in);
            const bool last = g == walk.groups - 1;
            divmod((uint32_t)in, last ? walk.last : walk.group, last ? walk.last_magic : walk.group_magic, y, rest);
            x = g * (int)walk.group + rest;
        } else divmod((uint32_t)t, (uint32_t)p.tiles_x, p.tiles_x_magic, y, x);
    };
    // slot of this lane's row of tile t (-1: none), and that row's weight
    auto slot_in = [&](int t) {
        int lx, ly;
        locate(t, ly, lx);
        return a.slot_of[(int64_t)ly * T_ROWS + warp * 32 + lane];
    };
    auto checked = [&](int slot) {
        if ((uint32_t)slot < a.slots) return slot;
        if (slot != -1) atomicExch(a.status, (int)MXFP8_ERR_DEVICE_ARGS);
        return -1;
    };
    // this warp's slab of tile t -> ring slot buf: 16 copies of two rows; lane l carries 16 bytes of row l / 16 of each pair
    auto issue = [&](int t, int slot, int buf) {
        int lx, ly, token, rest;
        locate(t, ly, lx);
        divmod(slot < 0 ? 0u : (uint32_t)slot, a.top_k, a.top_k_magic, token, rest);
        const int64_t col = (int64_t)lx * T_COLS + (lane & 15) * (16 / ESZ);
        const bool col_ok = col < p.cols;
        const uint8_t* src = static_cast<const uint8_t*>(a.src) + (col_ok ? col : 0) * ESZ;
        const uint32_t src_pitch = (uint32_t)p.cols * ESZ;
        const int upper = lane >> 4;
        const uint32_t to = my_slabs + buf * IN_BYTES + upper * T_BYTES + ((lane & 15) ^ upper) * 16;      // its piece of row `upper`
        if (slot < 0) token = -1;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int tk = __shfl_sync(0xFFFFFFFFu, token, 2 * i + upper);
            const uint32_t bytes = (tk >= 0 && col_ok) ? 16u : 0u;               // 0: the 16 bytes are filled with zeros
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;"
                         ::"r"((to ^ (2 * i & 15) << 4) + 2 * i * T_BYTES), "l"(src + (uint64_t)(uint32_t)max(tk, 0) * src_pitch), "r"(bytes) : "memory");
        }
    };
    auto commit = [] { asm volatile("cp.async.commit_group;" ::: "memory"); };
    auto weight_of = [&](int slot) { return (a.weights != nullptr && slot >= 0) ? a.weights[slot] : 0.f; };
    int next_slot = -1;                             // of this lane's row in the next tile
    float my_weight = 0.f;                          // of this lane's row in this tile (a row without a slot holds zeros and has the weight 0)
#pragma unroll
    for (int k = 0; k < RING; ++k) {
        const int t = blockIdx.x + k * gridDim.x;
        int slot = -1;
        if (t < num_tiles) {
            slot = checked(slot_in(t));
            issue(t, slot, k);
        }
        commit();
        if (k == 0) my_weight = weight_of(slot);
        else next_slot = slot;
    }
    auto store_tile = [&](int i, int x, int y) {    // one warp does the whole CTA's part
        if (i % STORERS != warp) return;
        asm volatile("bar.sync %0, %1;" ::"r"(1 + i % STAGES), "n"(QT_THREADS) : "memory");
        const uint8_t* at = sm_scales + (i % STAGES) * 1024;
#pragma unroll 1
        for (int k = 0; k < QT_THREADS / 32; ++k) store_scales<BF, DO_ROW, DO_COL>(p, x, y, at, at + 512, k * 32 + lane, lane, k);
    };
    int it = 0, before_x = 0, before_y = 0;         // the tile before this one
    for (int tile = blockIdx.x; tile < num_tiles; tile += gridDim.x, ++it) {
        const int buf = it & 1;
        const int after = tile + RING * (int)gridDim.x;         // the tile that will refill this slab
        int raw = -1;
        if (after < num_tiles) raw = slot_in(after);            // asked for here, needed behind the slab; so is the next tile's weight
        const float next_weight = weight_of(next_slot);
        uint8_t* sm_row = sm_scales + (it % STAGES) * 1024;     // 128 rows x 4 blocks, at stage_offset(row)
        uint8_t* sm_col = sm_row + 512;                         // T_COLS columns x 4 blocks, at stage_offset(column)
        int tile_x, tile_y;
        locate(tile, tile_y, tile_x);
        const int64_t gcol0 = (int64_t)tile_x * T_COLS, grow0 = (int64_t)tile_y * T_ROWS;

        asm volatile("cp.async.wait_group 1;" ::: "memory");
        __syncwarp();
        const uint32_t slab = my_slabs + buf * IN_BYTES;
        const bool weighted = a.weights != nullptr;
        const int64_t my_col = gcol0 + lane * VEC;
        const bool col_ok = my_col < p.cols;                                         // cols % 16 == 0: a lane's bytes are all in or all out
        uint8_t* my_qrow = p.q_row + ((grow0 + warp * 32) * p.cols + my_col);
        uint8_t* my_qcol = p.q_col + ((grow0 + warp * 32) * p.cols + my_col);
        const uint32_t pitch = (uint32_t)p.cols;
        uint8_t* my_sm_col = sm_col + stage_offset(lane * VEC) + warp;         // column lane * VEC + i: + i * STAGE_PITCH
        const bool whole = __all_sync(0xFFFFFFFFu, col_ok);
        bool special = !whole;
        if (whole)
            special = convert_slab<DTYPE, ELEM, DO_ROW, DO_COL, FIRST_OUT>(slab, row_inv, my_qrow, my_qcol, pitch, sm_row + stage_offset(warp * 32 + lane), my_sm_col,
                                                                my_weight, weighted, lane, rule_offset);
        else if (weighted) {
            walk_row<DTYPE, ELEM, false>(slab, row_inv, my_weight, true, nullptr, lane, rule_offset);
            __syncwarp();
        }
        if (special) {
            plain_order(slab, lane);
            slab_careful<DTYPE, ELEM, DO_ROW, DO_COL, false>(gather_smem + warp * SLAB_BYTES + buf * IN_BYTES + lane * 8, my_qrow, my_qcol, pitch, sm_row + warp * 4 + lane / LPB, my_sm_col, lane,
                                                             rule_offset, 32, col_ok);
        }
        __syncwarp();
        if (after < num_tiles) {
            raw = checked(raw);
            issue(after, raw, buf);
        }
        my_weight = next_weight;
        next_slot = raw;
        commit();
        if (it > 0) store_tile(it - 1, before_x, before_y);
        if (it % STORERS != warp) asm volatile("bar.arrive %0, %1;" ::"r"(1 + it % STAGES), "n"(QT_THREADS) : "memory");
        before_x = tile_x;
        before_y = tile_y;
    }
    if (it > 0) store_tile(it - 1, before_x, before_y);
    asm volatile("cp.async.wait_group 0;" ::: "memory");
}

template <int DTYPE, int ELEM, bool R, bool C, bool GROUPED, bool FIRST_OUT>
cudaError_t launch_gather(const GatherArgs& a, const Walk& walk, cudaStream_t stream)
{
    constexpr int SMEM = RING * IN_BYTES + STAGES * 1024 + QT_THREADS * 16;      // ring, scale staging, row factors
    auto kernel = quantize_gather_kernel<DTYPE, ELEM, R, C, GROUPED, FIRST_OUT>;
    static_assert(STAGES == 2 * STORERS, "see STAGES");
    static unsigned long long smem_set = 0;
    cudaError_t err = ensure_dynamic_smem(kernel, SMEM, smem_set);
    if (err != cudaSuccess) return err;
    const int sms = qt_sm_count();
    if (sms <= 0) return cudaErrorInvalidDevice;
    const int tiles = a.tiles, most = sms * QT_CTAS_PER_SM;
    kernel<<<tiles < most ? tiles : most, QT_THREADS, SMEM, stream>>>(a, walk);
    count_launch(1);
    return cudaGetLastError();
}
template <int DTYPE, int ELEM, bool R, bool C, bool GROUPED>
cudaError_t launch_gather(const GatherArgs& a, const Walk& walk, cudaStream_t stream)
{
    if constexpr (R && C)
        if ((int64_t)a.slots * a.t.cols * 2 > FIRST_OUT_BYTES) return launch_gather<DTYPE, ELEM, R, C, GROUPED, true>(a, walk, stream);
    return launch_gather<DTYPE, ELEM, R, C, GROUPED, false>(a, walk, stream);
}
template <int DTYPE, int ELEM, bool R, bool C>
cudaError_t launch_gather(const GatherArgs& a, cudaStream_t stream)
{
    const int64_t strip = (int64_t)(a.slots / a.top_k) * T_BYTES;      // bytes of the tokens under one tile column
    const uint32_t tiles_x = (uint32_t)a.t.tiles_x;
    Walk w{};
    if (strip * tiles_x <= ONE_GROUP<R && C>) return launch_gather<DTYPE, ELEM, R, C, false>(a, w, stream);
    const uint32_t fit = (uint32_t)(strip >= GROUP_BYTES ? 1 : GROUP_BYTES / strip), groups = (tiles_x + fit - 1) / fit;
    w.group = (tiles_x + groups - 1) / groups;
    w.groups = (int)((tiles_x + w.group - 1) / w.group);
    w.last = tiles_x - w.group * (uint32_t)(w.groups - 1);
    w.group_magic = div_magic(w.group);
    w.last_magic = div_magic(w.last);
    return launch_gather<DTYPE, ELEM, R, C, true>(a, w, stream);
}
template <int DTYPE, int ELEM>
cudaError_t launch_gather_o(int orientation, const GatherArgs& a, cudaStream_t st)
{
    if (orientation == MXFP8_ROW) return launch_gather<DTYPE, ELEM, true, false>(a, st);
    if (orientation == MXFP8_COL) return launch_gather<DTYPE, ELEM, false, true>(a, st);
    return launch_gather<DTYPE, ELEM, true, true>(a, st);
}

cudaError_t launch_gather_e(int elem, bool bf16_src, int orientation, const GatherArgs& a, cudaStream_t st)
{
#define MXFP8_GATHER_CASE(E) \
    case E: return bf16_src ? launch_gather_o<MXFP8_BF16, E>(orientation, a, st) : launch_gather_o<MXFP8_FP32, E>(orientation, a, st);
    switch (elem) {
        MXFP8_GATHER_CASE(MXFP8_E4M3)
        MXFP8_GATHER_CASE(MXFP8_E5M2)
        MXFP8_GATHER_CASE(MXFP8_E2M3)
        MXFP8_GATHER_CASE(MXFP8_E3M2)
        MXFP8_GATHER_CASE(MXFP8_E2M1)
        default: return cudaErrorInvalidValue;
    }
#undef MXFP8_GATHER_CASE
}

}  // namespace
}  // namespace mxfp8

extern "C" int mxfp8_moe_dispatch_quantize(const void* src, int src_dtype, int64_t tokens, int64_t cols,
                                           const int32_t* slot_of, int64_t rows, int top_k, const float* weights,
                                           const int32_t* group_offsets, int num_groups,
                                           int orientation, int scale_rule, int elem,
                                           void* q_row, void* s_row, void* q_col, void* s_col,
                                           int sf_layout, void* stream)
{
    using namespace mxfp8;
    if (src_dtype != MXFP8_FP32 && src_dtype != MXFP8_BF16) return MXFP8_ERR_ENUM;
    if (orientation < MXFP8_ROW || orientation > MXFP8_BOTH) return MXFP8_ERR_ENUM;
    if (scale_rule != MXFP8_RULE_PAPER && scale_rule != MXFP8_RULE_OCP) return MXFP8_ERR_ENUM;
    if (!valid_elem(elem)) return MXFP8_ERR_ENUM;
    if (sf_layout != MXFP8_SF_LINEAR && sf_layout != MXFP8_SF_SWIZZLED) return MXFP8_ERR_ENUM;
    if (tokens < 0 || rows < 0 || cols <= 0 || top_k < 1 || num_groups < 1) return MXFP8_ERR_SHAPE;
    if ((rows % T_ROWS) || ((orientation & MXFP8_ROW) && (cols % 32))) return MXFP8_ERR_SHAPE;
    if (tokens == 0 || rows == 0) return MXFP8_OK;                       // no token, no segment
    if (!src || !slot_of || !group_offsets) return MXFP8_ERR_NULL;
    if ((orientation & MXFP8_ROW) && (!q_row || !s_row)) return MXFP8_ERR_NULL;
    if ((orientation & MXFP8_COL) && (!q_col || !s_col)) return MXFP8_ERR_NULL;
    if (!aligned16(src) || !aligned16(slot_of)) return MXFP8_ERR_ALIGN;
    if ((reinterpret_cast<uintptr_t>(weights) & 3u) || (reinterpret_cast<uintptr_t>(group_offsets) & 3u)) return MXFP8_ERR_ALIGN;
    if ((orientation & MXFP8_ROW) && (!aligned16(q_row) || !aligned16(s_row))) return MXFP8_ERR_ALIGN;
    if ((orientation & MXFP8_COL) && (!aligned16(q_col) || !aligned16(s_col))) return MXFP8_ERR_ALIGN;
    if (tokens > 0x7F000000LL || tokens * top_k > 0x7F000000LL || cols > 0x3FFFFFFFLL) return MXFP8_ERR_UNSUPPORTED;      // 32-bit counters and pitches
    if (!quantize_tma_eligible(src_dtype, rows, cols)) return MXFP8_ERR_UNSUPPORTED;   // needs cols % 16 == 0
    const uint32_t t_cols = src_dtype == MXFP8_BF16 ? 128 : 64;
    GatherArgs a{};
    QParams& q = a.t;
    q.rows = rows; q.cols = cols; q.rule = scale_rule; q.sf_layout = sf_layout;
    q.tiles_x = (int)((cols + t_cols - 1) / t_cols);
    q.tiles_x_magic = div_magic((uint32_t)q.tiles_x);
    q.tiles_y = (int)(rows / T_ROWS);
    q.q_row = static_cast<uint8_t*>(q_row);
    q.q_col = static_cast<uint8_t*>(q_col);
    q.s_row = static_cast<uint8_t*>(s_row);
    q.s_col = static_cast<uint8_t*>(s_col);
    a.src = src; a.slot_of = slot_of; a.weights = weights; a.used = group_offsets + num_groups;
    a.top_k = (uint32_t)top_k;
    a.top_k_magic = div_magic(a.top_k);
    a.slots = (uint32_t)(tokens * top_k);
    a.tiles = q.tiles_x * q.tiles_y;                                     // fits: quantize_tma_eligible
    if (!(a.status = device_status_word())) return MXFP8_ERR_CUDA;
    return launch_gather_e(elem, src_dtype == MXFP8_BF16, orientation, a, static_cast<cudaStream_t>(stream)) == cudaSuccess ? MXFP8_OK : MXFP8_ERR_CUDA;
}
