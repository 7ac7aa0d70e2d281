// The kernels of mxfp8_moe_dispatch_quantize: the conversion of rows that the tile loads gather by an index
// (quantize_tma_kernel.cuh, PRO_GATHER), all five element types, and its entry point.
#include "quantize_tma_kernel.cuh"

namespace mxfp8 {

cudaError_t quantize_tma_launch_gather(int elem, bool bf16_src, int orientation, const void* maps, const void* batch, cudaStream_t st)
{
    const QMaps& ms = *static_cast<const QMaps*>(maps);
    const QBatch& p = *static_cast<const QBatch*>(batch);
#define MXFP8_GATHER_CASE(E)                                                                                  \
    case E:                                                                                                   \
        return bf16_src ? launch_o<MXFP8_BF16, E, false, PRO_GATHER>(orientation, ms, p, st)                  \
                        : launch_o<MXFP8_FP32, E, false, PRO_GATHER>(orientation, ms, p, st);
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
