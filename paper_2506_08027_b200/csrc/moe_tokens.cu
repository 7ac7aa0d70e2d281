// A mixture-of-experts layer for a few tokens with packed E2M1 matrices (mxfp8_e2m1_moe), in two launches:
//   1. the choice of the experts from the router's logits, their gate / up products, m = act(gate) * up
//   2. the down products of the chosen experts and their weighted sum, straight into y
// Every CTA of both launches chooses for itself (a few hundred logits, cheaper than a launch in between).  Bound by the
// weights of the experts that are used, 17/32 byte each, and by the instructions that decode them (210 per tile of 16 x 128 in launch 1).  Both are done once
// for every entry of an expert: ceil(slots / 8 or 16) times in launch 1, ceil(slots / 4 or 8) times in launch 2.
// One token with 8 of 64 experts of 2048 x 1408: 23 us; 16 tokens with 6: 68 to 73 us; 32 tokens with 2 of 8 experts of 4096 x 14336: 269 to
// 317 us from run to run with BF16 outputs, 35 us more with FP32 ones.
#include <type_traits>

#include "e2m1_tiles.cuh"
#include "mxfp8_host.h"

namespace mxfp8 {
namespace {

constexpr int MOE_MAX_TOKENS = 64, MOE_MAX_EXPERTS = 256, MOE_MAX_TOP_K = 16;
constexpr int MOE_MAX_ROWS = MOE_MAX_TOKENS * MOE_MAX_TOP_K;
// Entries of at most `most` = 4, 8 or 16 slots: an expert with n slots has ceil(n / most) of them.  With tokens <= 64 the sum over all experts is largest
// where every expert is used: 256 + 1024 / 4 entries, and entries * most places stay below 256 * 16 + 1024.
constexpr int MOE_MAX_ENTRIES = MOE_MAX_EXPERTS + MOE_MAX_ROWS / 4, MOE_MAX_LISTED = MOE_MAX_EXPERTS * 16 + MOE_MAX_ROWS;

struct MoeArgs {
    const __nv_bfloat16* x;          // [tokens, cols]
    const float* logits;             // [tokens, experts]
    const uint8_t *gate_up, *down;   // packed
    void* y;                         // [tokens, cols]
    bool bf16_out;
    int32_t* ids;
    float* weights;
    __nv_bfloat16 *m_hi, *m_lo, *m_rest;      // [slots, inner]: m = m_hi + m_lo (+ m_rest; null for BF16 outputs)
    int tokens, experts, top_k, act, renormalize;
    int cols, inner;
    int col_tiles, inner_tiles;      // column tiles of gate_up and of down
    uint32_t units_magic, top_k_magic, experts_magic;      // of the units of an entry, top_k and experts
};

// What a CTA knows of the choice.  An entry is one expert with a few of the slots (token, choice) that chose it; experts and, within one, tokens ascend.
struct Choice {
    uint32_t who[MOE_MAX_EXPERTS][2];                     // one bit per token that chose the expert
    uint32_t used[MOE_MAX_EXPERTS / 32];                  // one bit per expert that was chosen
    uint32_t large[MOE_MAX_EXPERTS / 32];                 // and per expert with more than one entry
    float weight[MOE_MAX_ROWS];                           // by slot (weigh fills it in)
    short expert[MOE_MAX_ROWS];                           // by slot; -1: none
    uint8_t token[MOE_MAX_ROWS];                          // by slot
    short slot[MOE_MAX_LISTED];                           // `most` places per entry
    short entry_expert[MOE_MAX_ENTRIES];
    uint8_t entry_rows[MOE_MAX_ENTRIES];
    int entries;
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

// Chooses for all tokens and makes the entries.  `keys`: shared memory for tokens * experts numbers.  An expert's place is the number of experts before
// it: larger logits, and equal ones of a lower number.  That is tokens * experts^2 comparisons, all threads side by side; where they are many,
// a warp per token takes the largest top_k times instead (one token of 64 experts: 4.4 thousand cycles for everything here, 7.0 the other way;
// 16 tokens: 8.4 and 6.3).  Ends with a barrier.
constexpr int MOE_COMPARISONS = 128 * 128;
__device__ __forceinline__ void choose(const MoeArgs& a, Choice& choice, uint32_t* keys, int most)
{
    const int tid = threadIdx.x, lane = tid & 31, threads = blockDim.x, pairs = a.tokens * a.experts, slots = a.tokens * a.top_k;
#pragma unroll 1
    for (int i = tid; i < pairs; i += threads) keys[i] = order_of(a.logits[i]);
#pragma unroll 1
    for (int e = tid; e < MOE_MAX_EXPERTS; e += threads) {
        choice.who[e][0] = choice.who[e][1] = 0u;
        if (e < MOE_MAX_EXPERTS / 32) choice.used[e] = choice.large[e] = 0u;
    }
#pragma unroll 1
    for (int s = tid; s < slots; s += threads) {
        int t, j;
        divmod((uint32_t)s, (uint32_t)a.top_k, a.top_k_magic, t, j);
        choice.expert[s] = -1;
        choice.token[s] = (uint8_t)t;
    }
    __syncthreads();
    auto take = [&](int t, int e, int place) {
        choice.expert[t * a.top_k + place] = (short)e;
        atomicOr(&choice.who[e][t >> 5], 1u << (t & 31));
        atomicOr(&choice.used[e >> 5], 1u << (e & 31));
    };
    if (pairs * a.experts <= MOE_COMPARISONS) {
#pragma unroll 1
        for (int i = tid; i < pairs; i += threads) {
            int t, e;
            divmod((uint32_t)i, (uint32_t)a.experts, a.experts_magic, t, e);
            const uint32_t key = keys[i], *row = keys + t * a.experts;
            int place = 0;
#pragma unroll 4
            for (int o = 0; o < a.experts; ++o) {
                const uint32_t other = row[o];
                place += other > key || (other == key && o < e);
            }
            if (key != 0u && place < a.top_k) take(t, e, place);
        }
    } else {
#pragma unroll 1
        for (int t = tid >> 5; t < a.tokens; t += threads >> 5) {
            uint32_t* row = keys + t * a.experts;
#pragma unroll 1
            for (int j = 0; j < a.top_k; ++j) {
                uint32_t best = 0u;
                int at = 0;
#pragma unroll 4
                for (int e = lane; e < a.experts; e += 32)
                    if (row[e] > best) { best = row[e]; at = e; }
                const uint32_t peak = __reduce_max_sync(0xFFFFFFFFu, best);
                if (peak == 0u) break;                   // none is left
                const int e = (int)__reduce_min_sync(0xFFFFFFFFu, best == peak ? (uint32_t)at : 0xFFFFu);
                if ((e & 31) == lane) {
                    take(t, e, j);
                    row[e] = 0u;                         // read again by this lane alone
                }
            }
        }
    }
    __syncthreads();
    if (a.tokens > most) {                               // experts with more than one entry
#pragma unroll 1
        for (int e = tid; e < a.experts; e += threads)
            if (__popc(choice.who[e][0]) + __popc(choice.who[e][1]) > most) atomicOr(&choice.large[e >> 5], 1u << (e & 31));
        __syncthreads();
    }
    // entries of the experts before e
    auto entries_before = [&](int e) {
        int v = 0;
#pragma unroll 1
        for (int w = 0; 32 * w < e; ++w) {
            const uint32_t below = e - 32 * w < 32 ? (1u << (e - 32 * w)) - 1u : 0xFFFFFFFFu;
            v += __popc(choice.used[w] & below);
            for (uint32_t more = choice.large[w] & below; more != 0u; more &= more - 1u) {
                const int l = 32 * w + __ffs(more) - 1;
                v += (__popc(choice.who[l][0]) + __popc(choice.who[l][1]) - 1) / most;
            }
        }
        return v;
    };
    // every slot's place in its expert's entries
#pragma unroll 1
    for (int s = tid; s < slots; s += threads) {
        const int e = choice.expert[s], t = choice.token[s];
        if (e < 0) continue;
        const uint32_t low = choice.who[e][0], high = choice.who[e][1], below = (1u << (t & 31)) - 1u;
        const int rank = t < 32 ? __popc(low & below) : __popc(low) + __popc(high & below), n = __popc(low) + __popc(high);
        const int v = entries_before(e);
        const int piece = rank / most;
        choice.slot[(v + piece) * most + rank - piece * most] = (short)s;
        if (rank == piece * most) {
            choice.entry_expert[v + piece] = (short)e;
            choice.entry_rows[v + piece] = (uint8_t)min(most, n - rank);
        }
    }
    if (tid == threads - 1) choice.entries = entries_before(MOE_MAX_EXPERTS);
    __syncthreads();
}

// The slots' weights, a warp per token.  The logits are read once more.
__device__ __forceinline__ void weigh(const MoeArgs& a, Choice& choice)
{
    const int lane = threadIdx.x & 31;
#pragma unroll 1
    for (int t = threadIdx.x >> 5; t < a.tokens; t += blockDim.x >> 5) {
        const float* row = a.logits + t * a.experts;
        const int e = lane < a.top_k ? choice.expert[t * a.top_k + lane] : -1;
        const int first = __shfl_sync(0xFFFFFFFFu, e, 0);
        if (first < 0) {
            if (lane < a.top_k) choice.weight[t * a.top_k + lane] = 0.f;
            continue;
        }
        const uint32_t top = order_of(row[first]);
        const float share = e >= 0 ? share_of(order_of(row[e]), top) : 0.f;
        float total = share;
        if (!a.renormalize) {
            total = 0.f;
#pragma unroll 1
            for (int o = lane; o < a.experts; o += 32) {
                const uint32_t key = order_of(row[o]);
                if (key != 0u) total += share_of(key, top);
            }
        }
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) total += __shfl_xor_sync(0xFFFFFFFFu, total, off);
        if (lane < a.top_k) choice.weight[t * a.top_k + lane] = share / total;
    }
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

// A warp's ring of weight tiles in shared memory: one column tile of R row tiles to a stage, copied asynchronously by the warp's own
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

// Two row tiles of a stage
template <int NX>
__device__ __forceinline__ void read_tiles(Operands<2, NX>& o, const uint8_t* stage, int lane)
{
#pragma unroll
    for (int r = 0; r < 2; ++r) {
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

// A warp's next `last - first` stages of its ring, column tiles first .. last - 1: their products with NX blocks of eight rows.  The rows come from
// L2; the other warps cover their latency (asking for them a tile ahead costs registers, and so warps: 12 of them with it took longer).
template <int NX, int STAGES, typename Fetch>
__device__ __forceinline__ void run_tiles(const __nv_bfloat16* const (&from)[NX], int first, int last, int cols, const uint8_t* ring, int& stage, Fetch& fetch,
                                          float (&acc)[2][NX][4])
{
    const int lane = threadIdx.x & 31;
#pragma unroll 1
    for (int kt = first; kt < last; ++kt) {
        Operands<2, NX> o;
        read_rows<NX>(o.x, from, kt, cols);
        copies_done<STAGES - 2>();
        __syncwarp();
        fetch();
        read_tiles<NX>(o, ring + stage * (2 * TILE_BYTES), lane);
        stage = stage + 1 == STAGES ? 0 : stage + 1;
        product<2, NX>(o, acc);
    }
}

// m of one (slot, row of the matrix) as BF16 numbers, which the tensor instructions of the second launch take.  FP32 outputs get three, which hold all of its 24
// bits (with two, y was 2.3e-6 from 64 bits where FP32 throughout is 2e-7 from it); BF16 outputs get two, 2^-16 of m beside
// their own rounding of 2^-8.  A finite m whose first part would round to infinity takes the largest BF16 number; the other parts
// of an infinity are zero, not infinity less infinity.
__device__ __forceinline__ void put_m(const MoeArgs& a, int64_t row, int n, float gate, float up)
{
    const float m = activate(gate, a.act) * up;
    __nv_bfloat16 hi = __float2bfloat16_rn(m);
    if (isinf(__bfloat162float(hi))) hi = __float2bfloat16_rz(m);
    a.m_hi[row * a.inner + n] = hi;
    const float rest = m - __bfloat162float(hi);
    const __nv_bfloat16 lo = __float2bfloat16_rn(isinf(m) ? 0.f : rest);
    a.m_lo[row * a.inner + n] = lo;
    if (a.m_rest) a.m_rest[row * a.inner + n] = __float2bfloat16_rn(isinf(m) ? 0.f : rest - __bfloat162float(lo));
}

// ---- first launch.  A unit is 16 gate rows and the 16 up rows that belong to them, for the slots of one entry.  The CTAs take the units in
// turn.  A CTA's warps take a unit each while there is one for every warp; the column tiles of the units that are left are split evenly
// over all warps (less than a unit each, so parts of two at most), whose sums meet in shared memory.
template <int NT, int WARPS, int STAGES>
__global__ void __launch_bounds__(32 * WARPS, 1) moe_gate_up_kernel(const MoeArgs a)
{
    extern __shared__ __align__(16) uint8_t dynamic[];
    __shared__ Choice choice;
    constexpr int P = 8 * NT + 1, UNIT_SUMS = 2 * TILE_ROWS * P, STAGE = 2 * TILE_BYTES;
    asm volatile("griddepcontrol.wait;" ::: "memory");                    // all that was launched before this call is done
    // only now: the second launch chooses and fetches weights beside this one, from inputs that those launches may have written
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    uint8_t* ring = dynamic + warp * STAGES * STAGE;
    const uint32_t ring_at = (uint32_t)__cvta_generic_to_shared(ring) + lane * 16;
    float* sums = reinterpret_cast<float*>(dynamic + WARPS * STAGES * STAGE);        // [warp][first, second unit]
    choose(a, choice, reinterpret_cast<uint32_t*>(dynamic), 8 * NT);
    const int per_entry = a.inner / TILE_ROWS, units = choice.entries * per_entry, ctas = gridDim.x, tiles = a.col_tiles;
    const int mine = units > (int)blockIdx.x ? (units - blockIdx.x + ctas - 1) / ctas : 0;       // unit i of this CTA is blockIdx.x + i * ctas
    const int whole = mine / WARPS, rest = mine % WARPS;
    const int s0 = rest * tiles * warp / WARPS, s1 = rest * tiles * (warp + 1) / WARPS;          // this warp's share of the rest
    const int r0 = s0 / tiles, k0 = s0 - r0 * tiles;
    const int64_t to_up = (int64_t)per_entry * tiles * TILE_BYTES;
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
                divmod((uint32_t)p.unit, (uint32_t)per_entry, a.units_magic, v, i);
                f_tile = a.gate_up + (((int64_t)choice.entry_expert[v] * 2 * per_entry + i) * tiles + p.first) * TILE_BYTES + lane * 16;
                f_left = p.count;
            }
        }
        if (f_left > 0) {
            const uint32_t to = ring_at + f_stage * STAGE;
            copy_tile(to, f_tile, lane);
            copy_tile(to + TILE_BYTES, f_tile + to_up, lane);
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
        int v, unit;
        divmod((uint32_t)p.unit, (uint32_t)per_entry, a.units_magic, v, unit);
        const short* slot = choice.slot + v * 8 * NT;
        const int rows = choice.entry_rows[v];
        const __nv_bfloat16* from[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int i = 8 * t + (lane >> 2);
            from[t] = a.x + (int64_t)choice.token[slot[i < rows ? i : 0]] * a.cols + (lane & 3) * 8;
        }
        float acc[2][NT][4];
        clear(acc);
        run_tiles<NT, STAGES>(from, p.first, p.first + p.count, a.cols, ring, stage, fetch, acc);
        float* to = sums + (2 * warp + (q - whole)) * UNIT_SUMS;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int n = (lane >> 2) + 8 * (i >> 1), s = 8 * t + 2 * (lane & 3) + (i & 1);
                if (q < whole) {
                    if (s < rows) put_m(a, slot[s], unit * TILE_ROWS + n, acc[0][t][i], acc[1][t][i]);
                } else {
                    to[n * P + s] = acc[0][t][i];
                    to[(TILE_ROWS + n) * P + s] = acc[1][t][i];
                }
            }
    }
    copies_done<0>();
    if (rest > 0) {
        __syncthreads();
        for (int r = warp; r < rest; r += WARPS) {
            int v, unit;
            divmod((uint32_t)(blockIdx.x + (whole * WARPS + r) * ctas), (uint32_t)per_entry, a.units_magic, v, unit);
            const short* slot = choice.slot + v * 8 * NT;
            const int rows = choice.entry_rows[v];
            // the warps with a part of unit r: those whose shares meet tiles r * tiles .. (r + 1) * tiles - 1
            for (int i = lane; i < rows * TILE_ROWS; i += 32) {
                const int n = i % TILE_ROWS, s = i / TILE_ROWS;
                float g = 0.f, u = 0.f;
#pragma unroll 4
                for (int w = 0; w < WARPS; ++w) {
                    const int b0 = rest * tiles * w / WARPS, b1 = rest * tiles * (w + 1) / WARPS;
                    if (b1 <= b0 || b1 <= r * tiles || b0 >= (r + 1) * tiles) continue;
                    const float* from = sums + (2 * w + (b0 < r * tiles)) * UNIT_SUMS + n * P + s;
                    g += from[0];
                    u += from[TILE_ROWS * P];
                }
                put_m(a, slot[s], unit * TILE_ROWS + n, g, u);
            }
        }
    }
    if (blockIdx.x == gridDim.x - 1 && (a.ids || a.weights)) {              // the CTA with the fewest units
        __syncthreads();
        if (a.weights) weigh(a, choice);
        __syncthreads();
        for (int s = tid; s < a.tokens * a.top_k; s += 32 * WARPS) {
            if (a.ids) a.ids[s] = choice.expert[s];
            if (a.weights) a.weights[s] = choice.weight[s];
        }
    }
}

// ---- second launch.  A cluster of two CTAs takes two row tiles of all entries' down projections at a time, and its warps split the entries'
// column tiles evenly: m, read from L2 by everybody, serves 32 rows (each CTA reads half of it).  A warp holds the weighted sums of
// its share for all tokens; at the end they are gathered through the cluster's shared memory, half of the outputs by each CTA.
// A block of eight columns of the tensor instructions takes the first two parts of m of four slots: entries have 4 NB slots at most.  Their third parts, where
// there are any, fill the columns of further blocks, eight slots to each.
constexpr int DOWN_ROWS = 2 * TILE_ROWS, DOWN_PITCH = DOWN_ROWS + 1;
template <int NB, int PARTS, int WARPS, int STAGES>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(32 * WARPS, 1) moe_down_kernel(const MoeArgs a)
{
    extern __shared__ __align__(16) uint8_t dynamic[];
    __shared__ Choice choice;
    constexpr int STAGE = 2 * TILE_BYTES, P = DOWN_PITCH, NX = PARTS == 2 ? NB : NB + (NB + 1) / 2;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rank = blockIdx.x & 1, cluster = blockIdx.x >> 1, clusters = gridDim.x >> 1;
    uint8_t* ring = dynamic + warp * STAGES * STAGE;
    const uint32_t ring_at = (uint32_t)__cvta_generic_to_shared(ring) + lane * 16;
    float* total = reinterpret_cast<float*>(dynamic + WARPS * STAGES * STAGE);           // [warp][token][row], rows padded
    choose(a, choice, reinterpret_cast<uint32_t*>(dynamic), 4 * NB);
    const int row_tiles = a.cols / TILE_ROWS, groups = row_tiles / 2;                    // cols is a multiple of 32
    float* mine = total + warp * a.tokens * P;
    // this warp's tiles of every group: a range of all entries' column tiles, one entry after the other
    const int tiles = choice.entries * a.inner_tiles, share = rank * WARPS + warp;
    const int w0 = (int)((int64_t)tiles * share / (2 * WARPS)), w1 = (int)((int64_t)tiles * (share + 1) / (2 * WARPS));
    const int v0 = w0 / a.inner_tiles, k0 = w0 - v0 * a.inner_tiles;
    const int64_t row_tile = (int64_t)a.inner_tiles * TILE_BYTES, matrix = row_tiles * row_tile;
    int f_group = cluster - clusters, f_v = 0, f_left = 0, f_here = 0, f_stage = 0;                  // tiles left of the group, of the entry
    const uint8_t* f_tile = nullptr;
    auto fetch = [&]() {
        if (f_here == 0) {                                                  // on to the next entry, or to the next group
            if (f_left == 0 && w1 > w0 && f_group + clusters < groups) {
                f_group += clusters;
                f_v = v0 - 1;
                f_left = w1 - w0;
            }
            if (f_left > 0) {
                const int begin = f_left == w1 - w0 ? k0 : 0;
                ++f_v;
                f_tile = a.down + choice.entry_expert[f_v] * matrix + 2 * f_group * row_tile + begin * TILE_BYTES + lane * 16;
                f_here = min(f_left, a.inner_tiles - begin);
                f_left -= f_here;
            }
        }
        if (f_here > 0) {
            const uint32_t to = ring_at + f_stage * STAGE;
            copy_tile(to, f_tile, lane);
            copy_tile(to + TILE_BYTES, f_tile + row_tile, lane);
            f_tile += TILE_BYTES;
            --f_here;
        }
        copies_issued();
        f_stage = f_stage + 1 == STAGES ? 0 : f_stage + 1;
    };
#pragma unroll 1
    for (int s = 0; s < STAGES - 1; ++s) fetch();
    weigh(a, choice);
    __syncthreads();
    asm volatile("griddepcontrol.wait;" ::: "memory");                     // the first launch's m is there
    int stage = 0;
    for (int group = cluster; group < groups; group += clusters) {
        for (int i = lane; i < a.tokens * P; i += 32) mine[i] = 0.f;
        __syncwarp();
#pragma unroll 1
        for (int v = v0, kt = k0, left = w1 - w0; left > 0; ++v, kt = 0) {
            const short* slot = choice.slot + v * 4 * NB;
            const int rows = choice.entry_rows[v], here = min(left, a.inner_tiles - kt);
            left -= here;
            const __nv_bfloat16* from[NX];
#pragma unroll
            for (int t = 0; t < NX; ++t) {               // columns 0 .. 3: the first parts of four slots, 4 .. 7: their second parts
                const int i = t < NB ? 4 * t + ((lane >> 2) & 3) : 8 * (t - NB) + (lane >> 2);
                from[t] = (t < NB ? (lane & 16 ? a.m_lo : a.m_hi) : a.m_rest) + (int64_t)slot[i < rows ? i : 0] * a.inner + (lane & 3) * 8;
            }
            float acc[2][NX][4];
            clear(acc);
            run_tiles<NX, STAGES>(from, kt, kt + here, a.inner, ring, stage, fetch, acc);
#pragma unroll
            for (int t = 0; t < NB; ++t)
#pragma unroll
                for (int c = 0; c < 2; ++c) {            // the lane's two columns
                    const int s = 4 * t + 2 * (lane & 3) + c;
                    const bool in = (lane & 2) == 0 && s < rows;
                    const int of = slot[in ? s : 0];
                    float* to = mine + choice.token[of] * P + (lane >> 2);
                    const float weight = choice.weight[of];
#pragma unroll
                    for (int r = 0; r < 2; ++r)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            // the third part lies in this lane for even blocks, in the lane of the second part for odd ones; the smaller two are added first
                            const float part = acc[r][t][2 * h + c], third = PARTS == 2 ? 0.f : acc[r][PARTS == 2 ? t : NB + t / 2][2 * h + c];
                            const float other = __shfl_xor_sync(0xFFFFFFFFu, t % 2 ? part + third : part, 2);
                            const float all = part + (t % 2 ? other : other + third);
                            if (in) to[r * TILE_ROWS + 8 * h] = fmaf(weight, all, to[r * TILE_ROWS + 8 * h]);
                        }
                }
            __syncwarp();
        }
        __syncwarp();
        asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
        // a thread per output: the sums of the warps of both CTAs
        const int half = a.tokens * (DOWN_ROWS / 2);
        for (int i = tid; i < half; i += 32 * WARPS) {
            const int o = rank * half + i, t = o / DOWN_ROWS, n = o % DOWN_ROWS;
            const uint32_t at = (uint32_t)__cvta_generic_to_shared(total + t * P + n);
            float part[2][WARPS];
#pragma unroll
            for (uint32_t c = 0; c < 2; ++c) {
                uint32_t there;
                asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(at), "r"(c));
#pragma unroll
                for (int w = 0; w < WARPS; ++w)
                    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(part[c][w]) : "r"(there + w * a.tokens * P * (int)sizeof(float)) : "memory");
            }
            float s = 0.f;
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int w = 0; w < WARPS; ++w) s += part[c][w];
            const int64_t to = (int64_t)t * a.cols + group * DOWN_ROWS + n;
            if (a.bf16_out) static_cast<__nv_bfloat16*>(a.y)[to] = __float2bfloat16_rn(s);
            else static_cast<float*>(a.y)[to] = s;
        }
        __syncwarp();
        asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
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
constexpr int MOE_DYNAMIC_SMEM = 227 * 1024 - (int)sizeof(Choice) - 64;
template <typename Kernel>
cudaError_t launch_early(Kernel kernel, int ctas, int threads, int smem, unsigned long long& set, const MoeArgs& a, cudaStream_t st)
{
    const cudaError_t err = ensure_dynamic_smem(kernel, MOE_DYNAMIC_SMEM, set);
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
    static_assert(SMEM <= MOE_DYNAMIC_SMEM, "ring and sums fit");
    static unsigned long long set = 0;
    return launch_early(moe_gate_up_kernel<NT, WARPS, STAGES>, multiprocessors(), 32 * WARPS, SMEM, set, a, st);
}

template <int NB, int PARTS, int WARPS, int STAGES, int TOKENS>
cudaError_t launch_down(const MoeArgs& a, cudaStream_t st)
{
    constexpr int RING = WARPS * STAGES * 2 * TILE_BYTES, PER_TOKEN = WARPS * DOWN_PITCH * (int)sizeof(float);
    static_assert(RING + TOKENS * PER_TOKEN <= MOE_DYNAMIC_SMEM, "ring and sums fit");
    static unsigned long long set = 0;
    const int groups = a.cols / DOWN_ROWS, most = multiprocessors() / 2;
    return launch_early(moe_down_kernel<NB, PARTS, WARPS, STAGES>, 2 * (groups < most ? groups : most), 32 * WARPS, RING + a.tokens * PER_TOKEN, set, a, st);
}

}  // namespace
}  // namespace mxfp8

using namespace mxfp8;

extern "C" size_t mxfp8_e2m1_moe_ws_bytes(int64_t tokens, int top_k, int64_t inner)
{
    if (tokens <= 0 || top_k <= 0 || inner <= 0 || tokens > MOE_MAX_TOKENS || top_k > MOE_MAX_TOP_K) return 0;
    return (size_t)tokens * top_k * (size_t)inner * 3 * sizeof(__nv_bfloat16);
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
    a.m_rest = a.bf16_out ? nullptr : a.m_lo + tokens * top_k * inner;
    a.tokens = (int)tokens; a.experts = num_experts; a.top_k = top_k; a.act = act; a.renormalize = renormalize != 0;
    a.cols = (int)cols; a.inner = (int)inner;
    a.col_tiles = (int)((cols + TILE_COLS - 1) / TILE_COLS); a.inner_tiles = (int)((inner + TILE_COLS - 1) / TILE_COLS);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    a.units_magic = div_magic((uint32_t)(a.inner / TILE_ROWS)); a.top_k_magic = div_magic((uint32_t)a.top_k); a.experts_magic = div_magic((uint32_t)a.experts);
    // Slots of an expert that are worked on together: by how many are expected of one (all of an expert's tiles are copied and decoded again for the next entry).
    // First launch, 8 or 16: 24 tokens with 2 of 8 experts of 4096 x 4096 93.1 us, 95.6 with 16; 32 tokens 107.8 and 105.2; 64 with 6 of 64 of 2048 x 1408 147.9 and 149.2.
    // Second launch, 4 or 8: 8 tokens with 2 of 8 66.5 us, 68.2 with 8; 12 tokens 74.0 and 73.3; 16 with 6 of 64 69.6 and 71.7, 32 97.9 and 96.3;
    // with FP32 outputs 70.5 and 72.3, 78.8 and 77.6, 73.4 and 77.6, 103.6 and 104.5.
    const int slots = a.tokens * a.top_k;
    cudaError_t err = a.tokens <= 8 || slots <= 6 * num_experts ? launch_gate_up<1, 16, 4>(a, st) : launch_gate_up<2, 16, 3>(a, st);
    if (err == cudaSuccess) {
        auto down = [&](auto nb) {
            constexpr int NB = decltype(nb)::value;
            // three blocks of activations need the registers of 12 warps (32 tokens with 2 of 8 experts of 4096 x 14336 363 us with 16, 315 with 12)
            if (a.m_rest) return NB == 1 && a.tokens <= 32 ? launch_down<NB, 3, NB == 1 ? 16 : 12, 3, 32>(a, st) : launch_down<NB, 3, 12, 3, 64>(a, st);
            return a.tokens <= 32 ? launch_down<NB, 2, 16, 3, 32>(a, st) : launch_down<NB, 2, 12, 3, 64>(a, st);
        };
        err = a.tokens <= 4 || slots <= 2 * num_experts ? down(std::integral_constant<int, 1>{}) : down(std::integral_constant<int, 2>{});
    }
    return err == cudaSuccess ? MXFP8_OK : MXFP8_ERR_CUDA;
}
