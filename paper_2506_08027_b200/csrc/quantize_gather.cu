// mxfp8_moe_dispatch_quantize: the conversion of rows gathered by an index (tokens in the order of their experts, App. A.4),
// optionally weighted.  The arithmetic of a 32-row slab is that of the fast path (quantize_tma_kernel.cuh); what differs is
// how a slab arrives and who waits for whom:
//   loads  : a warp fetches its own slab with 16-byte asynchronous copies, two rows per instruction, straight from the
//            tokens' rows (a gathering tensor copy was tried first: its issue runs through the lanes one by one, some 2000
//            cycles of one warp per tile with the other three waiting: 88 us for the row-blocked copy of 53248 x 2048
//            rows against 55 us).  Rows without a slot and columns behind the tensor are zero-filled by the copies.
//   weights: one FP32 product and one rounding per element, in place in the slab, before the conversion
//   order  : slots of the tile after next are asked for under the current slab, its copies go out as soon as the slab
//            is done; the CTA meets once per tile, for the scale bytes
#include "quantize_tma_kernel.cuh"

namespace mxfp8 {
namespace {

constexpr int SLAB_BYTES = 32 * T_BYTES;

// Gathered rows in place, same ownership as act_slab: row j times the weight that lane j holds.
template <bool BF>
__device__ __forceinline__ void weigh_slab(uint8_t* mine, float weight)
{
#pragma unroll 8
    for (int j = 0; j < 32; ++j) {
        const float f = __shfl_sync(0xFFFFFFFFu, weight, j);
        uint2 w = *reinterpret_cast<const uint2*>(mine + j * T_BYTES);
        if constexpr (BF) {
            const __nv_bfloat162 lo = __floats2bfloat162_rn(__uint_as_float(w.x << 16) * f, __uint_as_float(w.x & 0xFFFF0000u) * f);
            const __nv_bfloat162 hi = __floats2bfloat162_rn(__uint_as_float(w.y << 16) * f, __uint_as_float(w.y & 0xFFFF0000u) * f);
            w.x = *reinterpret_cast<const uint32_t*>(&lo);
            w.y = *reinterpret_cast<const uint32_t*>(&hi);
        } else {
            w.x = __float_as_uint(__uint_as_float(w.x) * f);
            w.y = __float_as_uint(__uint_as_float(w.y) * f);
        }
        *reinterpret_cast<uint2*>(mine + j * T_BYTES) = w;
    }
}

template <int DTYPE, int ELEM, bool DO_ROW, bool DO_COL>
__global__ void __launch_bounds__(QT_THREADS, QT_CTAS_PER_SM)
quantize_gather_kernel(const __grid_constant__ QBatch batch)
{
    constexpr bool BF = (DTYPE == MXFP8_BF16);
    constexpr int VEC = BF ? 4 : 2;                 // elements per lane per row
    constexpr int ESZ = BF ? 2 : 4;
    constexpr int T_COLS = T_BYTES / ESZ;           // 128 or 64
    constexpr int LPB = 32 / VEC;                   // lanes per row block: 8 or 16

    extern __shared__ __align__(128) uint8_t smem[];
    uint8_t* sm_scales = smem + RING * IN_BYTES;    // 2 x (row scales + column scales of one tile, 512 bytes each)
    __shared__ int queue[4];                        // tiles of the next iterations

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;   // warp = 32-row slab of the tile
    const QParams& p = batch.t[0];
    const uint32_t rule_offset = (p.rule == MXFP8_RULE_PAPER) ? paper_offset<ELEM>() : 0u;
    uint8_t* my_slabs = smem + warp * SLAB_BYTES;   // + IN_BYTES for the ring's second slot

    // rows in use: whole 128-row tiles by construction of the sort; anything else is reported and nothing is stored
    const int used = *batch.used_rows;
    int num_tiles = 0;
    if (used < 0 || used > p.rows || used % T_ROWS) {
        if (tid == 0 && blockIdx.x == 0) atomicExch(batch.args_status, (int)MXFP8_ERR_DEVICE_ARGS);
    } else num_tiles = (used / T_ROWS) * p.tiles_x;

    // slot of this lane's row of tile t (-1: none), and that row's weight
    auto slot_in = [&](int t) {
        int lx, ly;
        divmod((uint32_t)t, (uint32_t)p.tiles_x, p.tiles_x_magic, ly, lx);
        return batch.slot_of[(int64_t)ly * T_ROWS + warp * 32 + lane];
    };
    auto checked = [&](int slot) {
        if ((uint32_t)slot < batch.slots) return slot;
        if (slot != -1) atomicExch(batch.args_status, (int)MXFP8_ERR_DEVICE_ARGS);
        return -1;
    };
    // this warp's slab of tile t -> ring slot buf: 16 copies of two rows; lane l carries 16 bytes of row l / 16 of each pair
    auto issue = [&](int t, int slot, int buf) {
        int lx, ly, token, rest;
        divmod((uint32_t)t, (uint32_t)p.tiles_x, p.tiles_x_magic, ly, lx);
        divmod(slot < 0 ? 0u : (uint32_t)slot, batch.top_k, batch.top_k_magic, token, rest);
        const int64_t col = (int64_t)lx * T_COLS + (lane & 15) * (16 / ESZ);
        const bool col_ok = col < p.cols;
        const uint8_t* src = static_cast<const uint8_t*>(batch.gather_src) + (col_ok ? col : 0) * ESZ;
        const uint32_t to = smem_addr(my_slabs + buf * IN_BYTES + (lane >> 4) * T_BYTES + (lane & 15) * 16);
        if (slot < 0) token = -1;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int tk = __shfl_sync(0xFFFFFFFFu, token, 2 * i + (lane >> 4));
            const uint32_t bytes = (tk >= 0 && col_ok) ? 16u : 0u;               // 0: the 16 bytes are filled with zeros
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;"
                         ::"r"(to + i * 2 * T_BYTES), "l"(src + (int64_t)max(tk, 0) * p.cols * ESZ), "r"(bytes) : "memory");
        }
    };
    auto commit = [] { asm volatile("cp.async.commit_group;" ::: "memory"); };
    auto next_tile = [&](int it) {                  // one thread: the tile of iteration `it` (handed out in order, or by CTA index)
        return batch.sched ? (int)atomicAdd(batch.sched, 1u) : (int)blockIdx.x + it * (int)gridDim.x;
    };

    if (tid == 0)
        for (int k = 0; k < 3; ++k) queue[k] = next_tile(k);
    __syncthreads();
    int slot[RING];                                 // of this lane's row in the slabs of iterations it, it + 1
    float weight[RING];
#pragma unroll
    for (int k = 0; k < RING; ++k) {
        slot[k] = -1;
        weight[k] = 0.f;
        if (queue[k] < num_tiles) {
            slot[k] = checked(slot_in(queue[k]));
            issue(queue[k], slot[k], k);
            if (batch.slot_weights != nullptr && slot[k] >= 0) weight[k] = batch.slot_weights[slot[k]];
        }
        commit();
    }
    for (int it = 0;; ++it) {
        const int tile = queue[it & 3];
        if (tile >= num_tiles) break;
        const int buf = it & 1;
        const int after = queue[(it + 2) & 3];      // the tile that will refill this slab
        int handed = 0;
        if (tid == 0) handed = next_tile(it + 3);   // asked for now, needed at the barrier (the counter's round trip hides under the slab)
        int raw = -1;
        if (after < num_tiles) raw = slot_in(after);
        uint8_t* sm_row = sm_scales + (it & 1) * 1024;          // 128 rows x 4 blocks, at stage_offset(row)
        uint8_t* sm_col = sm_row + 512;                         // T_COLS columns x 4 blocks, at stage_offset(column)
        int tile_x, tile_y;
        divmod((uint32_t)tile, (uint32_t)p.tiles_x, p.tiles_x_magic, tile_y, tile_x);
        const int64_t gcol0 = (int64_t)tile_x * T_COLS, grow0 = (int64_t)tile_y * T_ROWS;

        asm volatile("cp.async.wait_group 1;" ::: "memory");
        __syncwarp();
        uint8_t* my_in = my_slabs + buf * IN_BYTES + lane * 8;
        if (batch.slot_weights != nullptr) {
            weigh_slab<BF>(my_in, buf ? weight[1] : weight[0]);
            // a row without a slot holds zeros, which a weight of its own (0) leaves alone
        }
        const int64_t my_col = gcol0 + lane * VEC;
        const bool col_ok = my_col < p.cols;                                         // cols % 16 == 0: a lane's bytes are all in or all out
        uint8_t* my_qrow = p.q_row + ((grow0 + warp * 32) * p.cols + my_col);
        uint8_t* my_qcol = p.q_col + ((grow0 + warp * 32) * p.cols + my_col);
        const uint32_t pitch = (uint32_t)p.cols;
        uint8_t* my_sm_row = sm_row + warp * 4 + lane / LPB;                   // row 32 warp + j: + j * STAGE_PITCH
        uint8_t* my_sm_col = sm_col + stage_offset(lane * VEC) + warp;         // column lane * VEC + i: + i * STAGE_PITCH
        bool special = !__all_sync(0xFFFFFFFFu, col_ok);
        if (!special)
            special = slab_fast<DTYPE, ELEM, DO_ROW, DO_COL, false>(my_in, my_qrow, my_qcol, pitch, my_sm_row, my_sm_col, lane, rule_offset);
        if (special)
            slab_careful<DTYPE, ELEM, DO_ROW, DO_COL, false>(my_in, my_qrow, my_qcol, pitch, my_sm_row, my_sm_col, lane, rule_offset, 32, col_ok);
        __syncwarp();
        if (after < num_tiles) {
            raw = checked(raw);
            issue(after, raw, buf);
            const float w = (batch.slot_weights != nullptr && raw >= 0) ? batch.slot_weights[raw] : 0.f;
            if (buf) weight[1] = w;
            else weight[0] = w;
        }
        commit();
        if (tid == 0) queue[(it + 3) & 3] = handed;
        __syncthreads();                            // the tile's scale bytes are complete
        store_scales<BF, DO_ROW, DO_COL, false>(p, tile_x, tile_y, sm_row, sm_col, tid, lane, warp);
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    if (tid == 0 && batch.sched != nullptr) {       // the last CTA out zeroes the words for the next launch
        __threadfence();
        if (atomicAdd(batch.sched + 1, 1u) == gridDim.x - 1) {
            batch.sched[0] = 0u;
            batch.sched[1] = 0u;
        }
    }
}

template <int DTYPE, int ELEM, bool R, bool C>
cudaError_t launch_gather(const QBatch& p, cudaStream_t stream)
{
    constexpr int SMEM = RING * IN_BYTES + 2048;
    auto kernel = quantize_gather_kernel<DTYPE, ELEM, R, C>;
    static unsigned long long smem_set = 0;
    cudaError_t err = ensure_dynamic_smem(kernel, SMEM, smem_set);
    if (err != cudaSuccess) return err;
    const int sms = qt_sm_count();
    if (sms <= 0) return cudaErrorInvalidDevice;
    const int tiles = p.tile_start[1], most = sms * QT_CTAS_PER_SM;
    kernel<<<tiles < most ? tiles : most, QT_THREADS, SMEM, stream>>>(p);
    count_launch(1);
    return cudaGetLastError();
}
template <int DTYPE, int ELEM>
cudaError_t launch_gather_o(int orientation, const QBatch& p, cudaStream_t st)
{
    if (orientation == MXFP8_ROW) return launch_gather<DTYPE, ELEM, true, false>(p, st);
    if (orientation == MXFP8_COL) return launch_gather<DTYPE, ELEM, false, true>(p, st);
    return launch_gather<DTYPE, ELEM, true, true>(p, st);
}

}  // namespace

cudaError_t quantize_launch_gather(int elem, bool bf16_src, int orientation, const void* batch, cudaStream_t st)
{
    const QBatch& p = *static_cast<const QBatch*>(batch);
#define MXFP8_GATHER_CASE(E) \
    case E: return bf16_src ? launch_gather_o<MXFP8_BF16, E>(orientation, p, st) : launch_gather_o<MXFP8_FP32, E>(orientation, p, st);
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
    if (tokens > 0x7F000000LL || tokens * top_k > 0x7F000000LL) return MXFP8_ERR_UNSUPPORTED;
    if (!quantize_tma_eligible(src_dtype, rows, cols)) return MXFP8_ERR_UNSUPPORTED;   // needs cols % 16 == 0
    const QuantizeItem item{src, rows, cols, q_row, s_row, q_col, s_col};
    const GatherArgs gather{tokens, slot_of, weights, group_offsets + num_groups, top_k};
    return quantize_tma_batch(&item, 1, src_dtype, orientation, scale_rule, elem, sf_layout, static_cast<cudaStream_t>(stream), false, MXFP8_ACT_NONE,
                              nullptr, nullptr, false, nullptr, nullptr, nullptr, &gather);
}
