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
constexpr int MOE_MAX_ROWS = MOE_MAX_TOKENS * MOE_MAX_TOP_K, MOE_MAX_ENTRIES = MOE_MAX_EXPERTS + MOE_MAX_ROWS / 8;

struct MoeArgs {
    const __nv_bfloat16* x;          // [tokens, cols]
    const float* logits;             // [tokens, experts]
    const uint8_t *gate_up, *down;   // packed
    void* y;                         // [tokens, cols]
    bool bf16_out;
    int32_t* ids;
    float* weights;
    __nv_bfloat16 *m_hi, *m_lo;      // [rows, inner]: m = m_hi + m_lo; rows: the chosen (token, expert) pairs by expert, then token
    int tokens, experts, top_k, act, renormalize;
    int cols, inner;
    int col_tiles, inner_tiles;      // column tiles of gate_up and of down
    uint32_t pairs_magic;            // of inner / 16
};

// What a CTA knows of the choice: rows of m by expert, and entries, each the rows (a few at most) of one expert.
struct Choice {
    uint32_t who[MOE_MAX_EXPERTS][2];                     // one bit per token that chose the expert
    float share[MOE_MAX_ROWS];                            // by slot, later (weight) by row
    float weight[MOE_MAX_ROWS];
    short expert[MOE_MAX_ROWS];                           // by slot; -1: none
    short first[MOE_MAX_EXPERTS];                         // first row of an expert
    uint8_t token[MOE_MAX_ROWS];                          // by row
    short entry_expert[MOE_MAX_ENTRIES], entry_row[MOE_MAX_ENTRIES];
    uint8_t entry_rows[MOE_MAX_ENTRIES];
    int entries, scan[MOE_MAX_EXPERTS / 32];
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

// Chooses for all tokens, a warp for each in turn: top_k rounds of the largest remaining logit (the lowest expert among equals).  Then
// orders the pairs by expert and cuts every expert's rows into entries of at most `most`.  Ends with a barrier.
__device__ __forceinline__ void choose(const MoeArgs& a, Choice& choice, int most)
{
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = blockDim.x >> 5;
    constexpr int I = MOE_MAX_EXPERTS / 32;
    for (int e = tid; e < MOE_MAX_EXPERTS; e += blockDim.x) choice.who[e][0] = choice.who[e][1] = 0u;
    __syncthreads();
    for (int t = warp; t < a.tokens; t += warps) {
        uint32_t left[I];
#pragma unroll
        for (int i = 0; i < I; ++i) left[i] = lane + 32 * i < a.experts ? order_of(a.logits[t * a.experts + lane + 32 * i]) : 0u;
        float all = 0.f;
        uint32_t mine = 0u, top = 0u;                // lane j: choice j
        int expert = -1;
        for (int j = 0; j < a.top_k; ++j) {
            uint32_t best = 0u;
            int at = 0;
#pragma unroll
            for (int i = 0; i < I; ++i)
                if (32 * i < a.experts && left[i] > best) { best = left[i]; at = lane + 32 * i; }
            const uint32_t peak = __reduce_max_sync(0xFFFFFFFFu, best);
            if (peak == 0u) break;                   // none is left
            const int e = (int)__reduce_min_sync(0xFFFFFFFFu, best == peak ? (uint32_t)at : 0xFFFFu);
            if (j == 0) {
                top = peak;
                if (!a.renormalize)
#pragma unroll
                    for (int i = 0; i < I; ++i)
                        if (left[i] != 0u) all += share_of(left[i], top);
            }
            if (lane == j) {
                mine = peak;
                expert = e;
            }
#pragma unroll
            for (int i = 0; i < I; ++i)
                if (32 * i < a.experts && lane + 32 * i == e) left[i] = 0u;
        }
        const float share = expert >= 0 ? share_of(mine, top) : 0.f;
        float total = a.renormalize ? share : all;
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) total += __shfl_xor_sync(0xFFFFFFFFu, total, off);
        if (lane < a.top_k) {
            choice.expert[t * a.top_k + lane] = (short)expert;
            choice.share[t * a.top_k + lane] = share > 0.f ? share / total : 0.f;
            if (expert >= 0) atomicOr(&choice.who[expert][t >> 5], 1u << (t & 31));
        }
    }
    __syncthreads();
    // first rows and entries: a thread per expert, both sums in one number
    static_assert(MOE_MAX_ROWS < 65536 && MOE_MAX_EXPERTS == 256, "eight warps scan the experts");
    int n = 0, cut = 0, before = 0;
    if (warp < I) {
        n = __popc(choice.who[tid][0]) + __popc(choice.who[tid][1]);
        cut = (n + most - 1) / most;
        before = n | cut << 16;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const int v = __shfl_up_sync(0xFFFFFFFFu, before, off);
            if (lane >= off) before += v;
        }
        if (lane == 31) choice.scan[warp] = before;
        before -= n | cut << 16;
    }
    __syncthreads();
    if (warp < I) {
        int all = 0;
#pragma unroll
        for (int w = 0; w < I; ++w) {
            const int v = choice.scan[w];
            if (w < warp) before += v;
            all += v;
        }
        if (tid == 0) choice.entries = all >> 16;
        int row = before & 0xFFFF;
        choice.first[tid] = (short)row;
        for (int v = before >> 16; cut > 0; --cut, ++v, row += most, n -= most) {
            choice.entry_expert[v] = (short)tid;
            choice.entry_row[v] = (short)row;
            choice.entry_rows[v] = (uint8_t)min(most, n);
        }
    }
    __syncthreads();
    for (int s = tid; s < a.tokens * a.top_k; s += blockDim.x) {
        const int e = choice.expert[s], t = s / a.top_k;
        if (e < 0) continue;
        const uint32_t below = (1u << (t & 31)) - 1u;
        const int row = choice.first[e] + (t < 32 ? __popc(choice.who[e][0] & below) : __popc(choice.who[e][0]) + __popc(choice.who[e][1] & below));
        choice.token[row] = (uint8_t)t;
        choice.weight[row] = choice.share[s];
    }
    __syncthreads();
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

// A warp's ring of weight tiles in shared memory: R tiles (one column tile of R row tiles) to a stage, copied asynchronously by the warp's own
// lanes STAGES - 1 steps ahead.  Nothing but the warp's own copies and __syncwarp guards them.
__device__ __forceinline__ void copy_tile(uint32_t to, const uint8_t* from, int lane)          // both at the lane's 16 bytes
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" :: "r"(to), "l"(from) : "memory");
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" :: "r"(to + 512), "l"(from + 512) : "memory");
    if (lane < 4) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" :: "r"(to + 1024), "l"(from + 1024) : "memory");
}
__device__ __forceinline__ void copies_issued() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT>
__device__ __forceinline__ void copies_done() { asm volatile("cp.async.wait_group %0;" :: "n"(LEFT) : "memory"); }

template <int R, int NT>
__device__ __forceinline__ void read_tiles(Operands<R, NT>& o, const uint8_t* stage, int lane)
{
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const uint8_t* tile = stage + r * TILE_BYTES;
        o.lo[r] = *reinterpret_cast<const uint4*>(tile + lane * 16);
        o.hi[r] = *reinterpret_cast<const uint4*>(tile + lane * 16 + 512);
        o.s_lo[r] = *reinterpret_cast<const uint32_t*>(tile + TILE_CODES + (lane >> 2) * 4);
        o.s_hi[r] = *reinterpret_cast<const uint32_t*>(tile + TILE_CODES + (lane >> 2) * 4 + 32);
    }
}

// Activations under column tile kt of the rows `from` (a lane without a row reads another one: its columns of the products are not used).
// Columns behind the matrix are zeros.
template <int NT>
__device__ __forceinline__ void read_rows(uint4 (&x)[NT][4], const __nv_bfloat16* const (&from)[NT], int kt, int cols)
{
    const int k = kt * TILE_COLS;
    if (k + TILE_COLS <= cols) {
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int g = 0; g < 4; ++g) x[t][g] = *reinterpret_cast<const uint4*>(from[t] + k + g * 32);
    } else {
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                x[t][g] = k + g * 32 < cols ? *reinterpret_cast<const uint4*>(from[t] + k + g * 32) : make_uint4(0u, 0u, 0u, 0u);
    }
}

template <int R, int NT>
__device__ __forceinline__ void clear(float (&acc)[R][NT][4])
{
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[r][t][i] = 0.f;
}

// A warp's next `last - first` tiles of its ring: column tiles first .. last - 1 of R row tiles, NX blocks of eight rows wide.
template <int R, int NX, int STAGES, typename Fetch>
__device__ __forceinline__ void run_tiles(const __nv_bfloat16* const (&from)[NX], int first, int last, int cols, const uint8_t* ring, int& stage, Fetch& fetch,
                                          float (&acc)[R][NX][4])
{
    const int lane = threadIdx.x & 31;
#pragma unroll 1
    for (int kt = first; kt < last; ++kt) {
        Operands<R, NX> o;
        read_rows<NX>(o.x, from, kt, cols);
        copies_done<STAGES - 2>();
        __syncwarp();
        fetch();
        read_tiles(o, ring + stage * (R * TILE_BYTES), lane);
        stage = stage + 1 == STAGES ? 0 : stage + 1;
        product<R, NX>(o, acc);
    }
}

// m of one (row of an entry, row of the matrix)
__device__ __forceinline__ void put_m(const MoeArgs& a, int64_t row, int n, float gate, float up)
{
    const float m = activate(gate, a.act) * up;
    const __nv_bfloat16 hi = __float2bfloat16_rn(m);
    a.m_hi[row * a.inner + n] = hi;
    a.m_lo[row * a.inner + n] = __float2bfloat16_rn(m - __bfloat162float(hi));
}

// ---- first launch: units of 16 gate rows and the 16 up rows that belong to them, for the rows of one entry.  The CTAs take the units in
// turn.  A CTA's warps take a unit each while there is one for every warp; the column tiles of the units that are left are split evenly
// over all warps (less than a unit each, so parts of two at most), whose sums meet in shared memory.
template <int NT, int WARPS, int STAGES>
__global__ void __launch_bounds__(32 * WARPS, 1) moe_gate_up_kernel(const MoeArgs a)
{
    extern __shared__ __align__(16) uint8_t dynamic[];
    __shared__ Choice choice;
    constexpr int P = 8 * NT + 1, UNIT_SUMS = 2 * TILE_ROWS * P, STAGE = 2 * TILE_BYTES;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");       // the second launch may choose, and fetch weights, beside this one
    asm volatile("griddepcontrol.wait;" ::: "memory");                    // all that was launched before this call is done
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    uint8_t* ring = dynamic + warp * STAGES * STAGE;
    const uint32_t ring_at = (uint32_t)__cvta_generic_to_shared(ring) + lane * 16;
    float* sums = reinterpret_cast<float*>(dynamic + WARPS * STAGES * STAGE);        // [warp][first, second unit]
    choose(a, choice, 8 * NT);
    if (blockIdx.x == 0)
        for (int s = tid; s < a.tokens * a.top_k; s += 32 * WARPS) {
            if (a.ids) a.ids[s] = choice.expert[s];
            if (a.weights) a.weights[s] = choice.share[s];
        }
    const int pairs = a.inner / TILE_ROWS, units = choice.entries * pairs, ctas = gridDim.x, tiles = a.col_tiles;
    const int mine = units > (int)blockIdx.x ? (units - blockIdx.x + ctas - 1) / ctas : 0;       // unit i of this CTA is blockIdx.x + i * ctas
    const int whole = mine / WARPS, rest = mine % WARPS;
    const int s0 = rest * tiles * warp / WARPS, s1 = rest * tiles * (warp + 1) / WARPS;          // this warp's share of the rest
    const int r0 = s0 / tiles, k0 = s0 - r0 * tiles;
    const int64_t to_up = (int64_t)pairs * tiles * TILE_BYTES;
    // piece q of this warp: a whole unit, or one of the parts of the rest; its unit, first tile and number of tiles (0: there is none)
    struct Part { int unit, first, count; };
    auto part = [&](int q) {
        Part p{0, 0, 0};
        if (q < whole) return Part{(int)blockIdx.x + (q * WARPS + warp) * ctas, 0, tiles};
        if (q > whole + 1) return p;
        p.first = q == whole ? k0 : 0;
        p.count = q == whole ? min(s1 - s0, tiles - k0) : s1 - s0 - min(s1 - s0, tiles - k0);
        p.unit = blockIdx.x + (whole * WARPS + r0 + (q - whole)) * ctas;
        return p;
    };
    int f_q = -1, f_left = 0, f_stage = 0;
    const uint8_t* f_tile = nullptr;
    auto fetch = [&]() {
        if (f_left == 0 && f_q < whole + 1) {
            const Part p = part(++f_q);
            if (p.count > 0) {
                int v, i;
                divmod((uint32_t)p.unit, (uint32_t)pairs, a.pairs_magic, v, i);
                f_tile = a.gate_up + (((int64_t)choice.entry_expert[v] * 2 * pairs + i) * tiles + p.first) * TILE_BYTES + lane * 16;
                f_left = p.count;
            }
        }
        if (f_left > 0) {
            copy_tile(ring_at + f_stage * STAGE, f_tile, lane);
            copy_tile(ring_at + f_stage * STAGE + TILE_BYTES, f_tile + to_up, lane);
            f_tile += TILE_BYTES;
            --f_left;
        }
        copies_issued();
        f_stage = f_stage + 1 == STAGES ? 0 : f_stage + 1;
    };
#pragma unroll 1
    for (int s = 0; s < STAGES - 1; ++s) fetch();
    int stage = 0;
#pragma unroll 1
    for (int q = 0; q < whole + 2; ++q) {
        const Part p = part(q);
        if (p.count == 0) continue;
        int v, pair;
        divmod((uint32_t)p.unit, (uint32_t)pairs, a.pairs_magic, v, pair);
        const int row0 = choice.entry_row[v], rows = choice.entry_rows[v];
        const __nv_bfloat16* from[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int i = 8 * t + (lane >> 2);
            from[t] = a.x + (int64_t)choice.token[row0 + (i < rows ? i : 0)] * a.cols + (lane & 3) * 8;
        }
        float acc[2][NT][4];
        clear(acc);
        run_tiles<2, NT, STAGES>(from, p.first, p.first + p.count, a.cols, ring, stage, fetch, acc);
        float* to = sums + (2 * warp + (q - whole)) * UNIT_SUMS;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int n = (lane >> 2) + 8 * (i >> 1), s = 8 * t + 2 * (lane & 3) + (i & 1);
                if (q < whole) {
                    if (s < rows) put_m(a, row0 + s, pair * TILE_ROWS + n, acc[0][t][i], acc[1][t][i]);
                } else {
                    to[n * P + s] = acc[0][t][i];
                    to[(TILE_ROWS + n) * P + s] = acc[1][t][i];
                }
            }
    }
    copies_done<0>();
    if (rest == 0) return;
    __syncthreads();
    for (int r = warp; r < rest; r += WARPS) {
        int v, pair;
        divmod((uint32_t)(blockIdx.x + (whole * WARPS + r) * ctas), (uint32_t)pairs, a.pairs_magic, v, pair);
        const int row0 = choice.entry_row[v], rows = choice.entry_rows[v];
        // the warps with a part of unit r: those whose shares meet tiles r * tiles .. (r + 1) * tiles - 1
        for (int i = lane; i < rows * TILE_ROWS; i += 32) {
            const int n = i & (TILE_ROWS - 1), s = i >> 4;
            float g = 0.f, u = 0.f;
            for (int w = 0; w < WARPS; ++w) {
                const int b0 = rest * tiles * w / WARPS, b1 = rest * tiles * (w + 1) / WARPS;
                if (b1 <= b0 || b1 <= r * tiles || b0 >= (r + 1) * tiles) continue;
                const float* from = sums + (2 * w + (b0 < r * tiles)) * UNIT_SUMS + n * P + s;
                g += from[0];
                u += from[TILE_ROWS * P];
            }
            put_m(a, row0 + s, pair * TILE_ROWS + n, g, u);
        }
    }
}

// ---- second launch: a CTA takes 16 rows of all entries' down projections at a time.  Its warps take the entries' column tiles in turn; each
// holds the weighted sums of its share for all tokens, and they are added at the end.
template <int NT, int WARPS, int STAGES>
__global__ void __launch_bounds__(32 * WARPS, 1) moe_down_kernel(const MoeArgs a)
{
    extern __shared__ __align__(16) uint8_t dynamic[];
    __shared__ Choice choice;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    uint8_t* ring = dynamic + warp * STAGES * TILE_BYTES;
    const uint32_t ring_at = (uint32_t)__cvta_generic_to_shared(ring) + lane * 16;
    float* total = reinterpret_cast<float*>(dynamic + WARPS * STAGES * TILE_BYTES);      // [warp][token][row], rows padded to 17
    choose(a, choice, 8 * NT);
    const int row_tiles = a.cols / TILE_ROWS, entries = choice.entries;
    float* mine = total + warp * a.tokens * 17;
    // this warp's tiles of every row tile: a range of all entries' column tiles, one entry after the other
    const int tiles = entries * a.inner_tiles, w0 = (int)((int64_t)tiles * warp / WARPS), w1 = (int)((int64_t)tiles * (warp + 1) / WARPS);
    const int v0 = w0 / a.inner_tiles, k0 = w0 - v0 * a.inner_tiles;
    int f_rt = blockIdx.x - gridDim.x, f_v = 0, f_left = 0, f_here = 0, f_stage = 0;          // tiles left of the row tile, of the entry
    const uint8_t* f_tile = nullptr;
    auto fetch = [&]() {
        if (f_here == 0) {                                                  // on to the next entry, or to the next row tile
            if (f_left == 0 && w1 > w0 && f_rt + (int)gridDim.x < row_tiles) {
                f_rt += gridDim.x;
                f_v = v0 - 1;
                f_left = w1 - w0;
            }
            if (f_left > 0) {
                const bool begin = f_left == w1 - w0;
                ++f_v;
                f_tile = a.down + ((int64_t)choice.entry_expert[f_v] * row_tiles + f_rt) * a.inner_tiles * TILE_BYTES + (begin ? k0 * TILE_BYTES : 0) + lane * 16;
                f_here = min(f_left, a.inner_tiles - (begin ? k0 : 0));
                f_left -= f_here;
            }
        }
        if (f_here > 0) {
            copy_tile(ring_at + f_stage * TILE_BYTES, f_tile, lane);
            f_tile += TILE_BYTES;
            --f_here;
        }
        copies_issued();
        f_stage = f_stage + 1 == STAGES ? 0 : f_stage + 1;
    };
#pragma unroll 1
    for (int s = 0; s < STAGES - 1; ++s) fetch();
    asm volatile("griddepcontrol.wait;" ::: "memory");                     // the first launch's m is there
    int stage = 0;
    for (int rt = blockIdx.x; rt < row_tiles; rt += gridDim.x) {
        for (int i = lane; i < a.tokens * 17; i += 32) mine[i] = 0.f;
        __syncwarp();
        for (int v = v0, kt = k0, left = w1 - w0; left > 0; ++v, kt = 0) {
            const int row0 = choice.entry_row[v], rows = choice.entry_rows[v], here = min(left, a.inner_tiles - kt);
            left -= here;
            const __nv_bfloat16* from[2 * NT];
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const int i = 8 * t + (lane >> 2);
                const int64_t at = (int64_t)(row0 + (i < rows ? i : 0)) * a.inner + (lane & 3) * 8;
                from[t] = a.m_hi + at;
                from[NT + t] = a.m_lo + at;
            }
            float acc[1][2 * NT][4];
            clear(acc);
            run_tiles<1, 2 * NT, STAGES>(from, kt, kt + here, a.inner, ring, stage, fetch, acc);
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int s = 8 * t + 2 * (lane & 3) + (i & 1);
                    if (s < rows) {
                        float* to = mine + choice.token[row0 + s] * 17 + (lane >> 2) + 8 * (i >> 1);
                        *to = fmaf(choice.weight[row0 + s], acc[0][t][i] + acc[0][NT + t][i], *to);
                    }
                }
            __syncwarp();
        }
        __syncthreads();
        for (int i = tid; i < a.tokens * TILE_ROWS; i += 32 * WARPS) {
            const int n = i & (TILE_ROWS - 1), t = i >> 4;
            float s = 0.f;
            for (int w = 0; w < WARPS; ++w) s += total[(w * a.tokens + t) * 17 + n];
            const int64_t at = (int64_t)t * a.cols + rt * TILE_ROWS + n;
            if (a.bf16_out) static_cast<__nv_bfloat16*>(a.y)[at] = __float2bfloat16_rn(s);
            else static_cast<float*>(a.y)[at] = s;
        }
        __syncthreads();
    }
    copies_done<0>();
}

int multiprocessors()
{
    static PerDeviceCache<int> cache;
    int n = 0;
    return cache.get(n, [](int dev, int& v) { return cudaDeviceGetAttribute(&v, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess; }) ? n : 148;
}

// Launched before the launches ahead of it have ended; the kernel waits for them itself.
template <typename Kernel>
cudaError_t launch_early(Kernel kernel, int ctas, int threads, int smem, int most_smem, unsigned long long& set, const MoeArgs& a, cudaStream_t st)
{
    const cudaError_t err = ensure_dynamic_smem(kernel, most_smem, set);
    if (err != cudaSuccess) return err;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)ctas);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = (size_t)smem;
    cfg.stream = st;
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    const cudaError_t rc = cudaLaunchKernelEx(&cfg, kernel, a);
    if (rc == cudaSuccess) count_launch(1);
    return rc;
}

template <int NT, int WARPS, int STAGES>
cudaError_t launch_gate_up(const MoeArgs& a, cudaStream_t st)
{
    constexpr int SMEM = WARPS * (STAGES * 2 * TILE_BYTES + 2 * 2 * TILE_ROWS * (8 * NT + 1) * (int)sizeof(float));
    static unsigned long long set = 0;
    return launch_early(moe_gate_up_kernel<NT, WARPS, STAGES>, multiprocessors(), 32 * WARPS, SMEM, SMEM, set, a, st);
}

template <int NT, int WARPS, int STAGES>
cudaError_t launch_down(const MoeArgs& a, cudaStream_t st)
{
    constexpr int RING = WARPS * STAGES * TILE_BYTES, PER_TOKEN = WARPS * 17 * (int)sizeof(float);
    static unsigned long long set = 0;
    const int row_tiles = a.cols / TILE_ROWS, sms = multiprocessors();
    return launch_early(moe_down_kernel<NT, WARPS, STAGES>, row_tiles < sms ? row_tiles : sms, 32 * WARPS, RING + a.tokens * PER_TOKEN,
                        RING + MOE_MAX_TOKENS * PER_TOKEN, set, a, st);
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
    a.pairs_magic = div_magic((uint32_t)(a.inner / TILE_ROWS));
    // eight rows of an expert together, or sixteen where that many are expected of most
    const bool few = a.tokens <= 8 || a.tokens * a.top_k <= 4 * num_experts;
    cudaError_t err = few ? launch_gate_up<1, 16, 4>(a, st) : launch_gate_up<2, 16, 3>(a, st);
    if (err == cudaSuccess) err = few ? launch_down<1, 16, 8>(a, st) : launch_down<2, 16, 7>(a, st);
    return err == cudaSuccess ? MXFP8_OK : MXFP8_ERR_CUDA;
}
