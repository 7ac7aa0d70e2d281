// Packed E2M1 (MXFP4) matrices and their products with BF16 activations on the warp-level tensor instructions: what matvec.cu and
// moe_tokens.cu share.
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
// and one exact product by 2^126 turn a pair of codes into a register of two BF16 values.  (Widening a small float by placing its
// bits across the exponent / mantissa boundary and multiplying by a power of two is a published method, used by open-source code for
// 4-bit weights; the order of a word's bits and the scale inside the product are this file's.)
#pragma once

#include "mxfp8_device.cuh"

namespace mxfp8 {
namespace {

constexpr int TILE_ROWS = 16, TILE_COLS = 128, TILE_CODES = 1024, TILE_BYTES = 1088;

// Code pairs p = 0 .. 3 of a word as BF16 pairs (column 2p in the low half), times `scale` (both halves: 2^126 X).
__device__ __forceinline__ void decode_word(uint32_t w, uint32_t scale, uint32_t (&out)[4])
{
    constexpr uint32_t V = 0x01C001C0u, S = 0x80008000u;
    out[0] = w & (V | S);
    out[1] = (w << 3) & (V | S);
    out[2] = ((w << 6) & V) | ((w << 1) & S);
    out[3] = ((w >> 3) & V) | ((w << 2) & S);
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const __nv_bfloat162 v = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&out[p]), *reinterpret_cast<const __nv_bfloat162*>(&scale));
        out[p] = *reinterpret_cast<const uint32_t*>(&v);
    }
}

__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// 2^(b - c), what a scale byte b leaves to the sums when its weights took c = b clamped to 64 .. 127 (weights are BF16 then,
// and a sum of 32 products only passes FP32's range where the scaled one does); b = 255 is NaN
__device__ __forceinline__ float scale_rest(uint32_t b, uint32_t c)
{
    return __uint_as_float(b == 255u ? 0x7FC00000u : (b + 127u - c) << 23);
}
// 2^126 * 2^(b - 127) as BF16, for b <= 127: exponent field b + 126.  Two words hold a row's four factors, one per half, and
// the product names the half that it takes.
template <int G>
__device__ __forceinline__ __nv_bfloat162 half_of(const uint32_t (&f)[2])
{
    const __nv_bfloat162 v = *reinterpret_cast<const __nv_bfloat162*>(&f[G & 1]);
    return (G >> 1) ? __high2bfloat162(v) : __low2bfloat162(v);
}
__device__ __forceinline__ void factors(uint32_t bytes, uint32_t (&f)[2])
{
    f[0] = (bytes & 0x00FF00FFu) * 128u + 0x3F003F00u;              // groups 0 and 2
    f[1] = ((bytes >> 8) & 0x00FF00FFu) * 128u + 0x3F003F00u;       // groups 1 and 3
}
// One lane's share of R row tiles and of the activations under them.
template <int R, int NT>
struct Operands {
    uint4 lo[R], hi[R];           // rows (lane / 4) and (lane / 4) + 8: a word of eight codes per group
    uint32_t s_lo[R], s_hi[R];    // their scale bytes, one per group
    uint4 x[NT][4];               // token lane / 4 of every block: eight columns per group
    __device__ __forceinline__ void load(const uint8_t* const (&tile)[R], int64_t w_at, const __nv_bfloat16* const (&from)[NT], const bool (&has)[NT], int64_t x_at, int lane)
    {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            lo[r] = __ldcs(reinterpret_cast<const uint4*>(tile[r] + w_at));
            hi[r] = __ldcs(reinterpret_cast<const uint4*>(tile[r] + w_at + 512));
            s_lo[r] = __ldcs(reinterpret_cast<const uint32_t*>(tile[r] + w_at + TILE_CODES - lane * 16 + (lane >> 2) * 4));
            s_hi[r] = __ldcs(reinterpret_cast<const uint32_t*>(tile[r] + w_at + TILE_CODES - lane * 16 + (lane >> 2) * 4 + 32));
        }
#pragma unroll
        for (int t = 0; t < NT; ++t)
            if (has[t])
#pragma unroll
                for (int g = 0; g < 4; ++g) x[t][g] = *reinterpret_cast<const uint4*>(from[t] + x_at + g * 32);
    }
};

template <int R, int NT>
__device__ __forceinline__ void product(const Operands<R, NT>& o, float (&acc)[R][NT][4])
{
    uint32_t any = 0u, all = 0xFFFFFFFFu;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        any |= o.s_lo[r] | o.s_hi[r];
        all &= o.s_lo[r] & o.s_hi[r];
    }
    const bool wide = ((any & 0x80808080u) | (~all & 0x40404040u)) != 0u;             // a byte outside 64 .. 127
    if (!__any_sync(0xFFFFFFFFu, wide)) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const uint32_t wl[4] = {o.lo[r].x, o.lo[r].y, o.lo[r].z, o.lo[r].w}, wh[4] = {o.hi[r].x, o.hi[r].y, o.hi[r].z, o.hi[r].w};
            float d[NT][4];
            uint32_t fl[2], fh[2];
            factors(o.s_lo[r], fl);
            factors(o.s_hi[r], fh);
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) d[t][i] = 0.f;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                uint32_t al[4], ah[4];
                const __nv_bfloat162 sl = g == 0 ? half_of<0>(fl) : (g == 1 ? half_of<1>(fl) : (g == 2 ? half_of<2>(fl) : half_of<3>(fl)));
                const __nv_bfloat162 sh = g == 0 ? half_of<0>(fh) : (g == 1 ? half_of<1>(fh) : (g == 2 ? half_of<2>(fh) : half_of<3>(fh)));
                decode_word(wl[g], *reinterpret_cast<const uint32_t*>(&sl), al);
                decode_word(wh[g], *reinterpret_cast<const uint32_t*>(&sh), ah);
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    mma_bf16(d[t], al[0], ah[0], al[1], ah[1], o.x[t][g].x, o.x[t][g].y);
                    mma_bf16(d[t], al[2], ah[2], al[3], ah[3], o.x[t][g].z, o.x[t][g].w);
                }
            }
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[r][t][i] += d[t][i];
        }
        return;
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const uint32_t wl[4] = {o.lo[r].x, o.lo[r].y, o.lo[r].z, o.lo[r].w}, wh[4] = {o.hi[r].x, o.hi[r].y, o.hi[r].z, o.hi[r].w};
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            uint32_t al[4], ah[4];
            const uint32_t b_lo = o.s_lo[r] >> (8 * g) & 255u, b_hi = o.s_hi[r] >> (8 * g) & 255u;
            const uint32_t c_lo = min(max(b_lo, 64u), 127u), c_hi = min(max(b_hi, 64u), 127u);
            decode_word(wl[g], (c_lo + 126u) * 0x00800080u, al);       // 2^126 * 2^(c - 127), both halves
            decode_word(wh[g], (c_hi + 126u) * 0x00800080u, ah);
            const float f_lo = scale_rest(b_lo, c_lo), f_hi = scale_rest(b_hi, c_hi);
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                float d[4] = {0.f, 0.f, 0.f, 0.f};
                mma_bf16(d, al[0], ah[0], al[1], ah[1], o.x[t][g].x, o.x[t][g].y);
                mma_bf16(d, al[2], ah[2], al[3], ah[3], o.x[t][g].z, o.x[t][g].w);
                acc[r][t][0] = fmaf(f_lo, d[0], acc[r][t][0]);
                acc[r][t][1] = fmaf(f_lo, d[1], acc[r][t][1]);
                acc[r][t][2] = fmaf(f_hi, d[2], acc[r][t][2]);
                acc[r][t][3] = fmaf(f_hi, d[3], acc[r][t][3]);
            }
        }
    }
}

}  // namespace
}  // namespace mxfp8
