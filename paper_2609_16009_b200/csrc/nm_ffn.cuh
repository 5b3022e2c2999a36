// Feed-forward operators (nm_ffn.cu, nm_ffn_stream.cu): arguments shared by the kernels, activations, the plan of rows by expert.
#pragma once

#include "nm_async.cuh"

namespace nm {

// ---- activations, fp32 -------------------------------------------------------------------------------------------------------
// Of n values at once: one branch.  __expf is within 2 + |1.2 x| steps of exp(x) and the quotient within 2, which the 16 bits that are kept do not see.
// x / (1 + exp(-2 s)), s half of the exponent (of x itself, or of the tanh form's polynomial).  From h = exp(-|s|): the quotient is x / (1 + h h) for s >= 0 and
// x h h / (1 + h h) below, so the denominator stays in [1, 2] and h is a normal number as long as the result is one.  (exp(-2 s) itself leaves fp32 at -89, and
// __fdividef gives 0 from a denominator of 2^126 on: silu(-87.5) = -8.7e-37 is a normal number in fp32 and in bf16.)  Below 2^-126 the result is within steps of 2^-149.
__device__ __forceinline__ float gated_by_exp(float x, float s)
{
    const float h = __expf(-fabsf(s));
    return __fdividef(s < 0.f ? x * h * h : x, fmaf(h, h, 1.f));
}
template <int n>
__device__ __forceinline__ void activate(int act, float (&v)[n])
{
    switch (act) {
    case NM_ACT_RELU:
#pragma unroll
        for (int i = 0; i < n; ++i) v[i] = v[i] < 0.f ? 0.f : v[i];                       // a NaN stays one
        break;
    case NM_ACT_SILU:
#pragma unroll
        for (int i = 0; i < n; ++i) v[i] = gated_by_exp(v[i], 0.5f * v[i]);
        break;
    case NM_ACT_GELU:
#pragma unroll
        for (int i = 0; i < n; ++i) v[i] = 0.5f * v[i] * erfcf(-0.70710678f * v[i]);       // erfc: no cancellation for negative values
        break;
    case NM_ACT_GELU_TANH:                                                              // 0.5 (1 + tanh z) = 1 / (1 + exp(-2 z))
#pragma unroll
        for (int i = 0; i < n; ++i) v[i] = gated_by_exp(v[i], 0.79788456f * (v[i] + 0.044715f * v[i] * v[i] * v[i]));
        break;
    default: break;
    }
}

// A value of either 16-bit type, and rounding to it.
__device__ __forceinline__ float widen16(uint16_t v, bool f16) { return f16 ? __half2float(__ushort_as_half(v)) : __uint_as_float((uint32_t)v << 16); }
__device__ __forceinline__ uint16_t round16(float v, bool f16) { return f16 ? __half_as_ushort(__float2half_rn(v)) : __bfloat16_as_ushort(__float2bfloat16_rn(v)); }

// Rows of the experts.  Pair p = (token p / top_k, choice p % top_k) belongs to expert experts[p] - first where that is one of the E held
// here.  Rows are the pairs sorted by expert, each expert's in rising order: `order` has their tokens, `place` the row of each pair; a tile is up to R of one
// expert's rows.
struct RowTile { int expert, row0, rows, unused; };

// How the items of a product (a row tile x a column tile, kb steps of 64 k each) are dealt out: the first `whole` as they are, each of the others in
// `parts` chunks of kc steps (the last one shorter).  Chunk c < whole is item c; behind them part (c - whole) % parts of item whole + (c - whole) / parts.
struct Schedule { int whole, parts, kc, chunks; };

struct RowPlan {
    const RowTile *tiles;
    const Schedule *schedule;          // of this product
    const int *order;                  // [sorted row] -> token
    // Few pairs (up to kOwnPairs, in gathered tiles): every CTA makes the plan itself, in shared memory, and no kernel has to come first.  0: it is there.
    int own_pairs;
    const int32_t *experts; int first, E, top_k;
    int *place;                        // [pair] -> sorted row, for the weighted sum
};
constexpr int kOwnPairs = 128;

// Words of the counter area: a ticket for each product of a call (the chunks dealt out beyond one for each CTA), CTAs that are done, and the chunks there
// are of an item that is cut.
constexpr int kTicketUp = 0, kTicketDown = 1, kDone = 2, kItemCounters = 32, kMaxCut = 2 * kSMs, kCounterWords = kItemCounters + kMaxCut;

// The cut with the least modelled time.  Rounds in which all CTAs work take a step in busy_us (HBM: 148 x 32 KB at 6.9 TB/s, 0.70 us).  In the last one, with what
// is left, a CTA takes in 96 GB/s at most (0.25 us a step of 16 KB at least), or its part of HBM's rate; near each other the two add up to more than the
// larger, taken as a norm (72 CTAs: 0.48 us a step of 32 KB where either bound says 0.35).  The sums of a chunk take a CTA chunk_us - the store, a fence, a counter, each
// behind the copies' traffic - which has to fit beside the next chunk's copies; and at the end all of an item's come back to one CTA, sums_us each (35 GB/s), behind
// 2.5 us for the last counter and the first of them.
// All items but the last one to two rounds stay whole: sums in the workspace cost as much as the rows do, and only the end has to be even.
struct CutModel { int kb, column_tiles, most_chunks, forced; float alone_us, busy_us, sums_us, chunk_us; };
__host__ __device__ inline float cut_cost(const CutModel &m, int rest, int parts)
{
    if (m.forced) return parts <= m.forced ? (float)(m.forced - parts) : 1e9f;        // the nearest that may be
    const int kc = (m.kb + parts - 1) / parts, p = (m.kb + kc - 1) / kc, chunks = rest * p, rounds = chunks / kSMs, left = chunks - rounds * kSMs;
    const float share = m.busy_us * left / kSMs, step = left ? cbrtf(share * share * share + m.alone_us * m.alone_us * m.alone_us) : 0.f;
    const float body = kc * (rounds * m.busy_us + step), between = m.chunk_us * (rounds - (left ? 0 : 1));
    return p > 1 ? (body > between ? body : between) + 2.5f + (1 + p) * m.sums_us : body;
}
__host__ __device__ inline int whole_items(int items) { return items >= 2 * kSMs ? (items / kSMs - 1) * kSMs : 0; }
__host__ __device__ inline Schedule schedule_of(int items, int kb, int parts)
{
    const int whole = whole_items(items), kc = (kb + parts - 1) / parts, p = (kb + kc - 1) / kc;
    return p > 1 ? Schedule{whole, p, kc, whole + (items - whole) * p} : Schedule{items, 1, kb, items};
}

// The best schedule for `tiles` row tiles: by a warp, a lane for each number of parts.
__device__ __forceinline__ Schedule best_schedule(const CutModel &m, int tiles, int lane)
{
    const int items = tiles * m.column_tiles, rest = items - whole_items(items), parts = lane + 1;
    const bool may = parts == 1 || (parts <= m.kb && (long)rest * parts <= m.most_chunks);
    const float cost = may ? cut_cost(m, rest, parts) : INFINITY;
    const unsigned least = __reduce_min_sync(0xffffffffu, __float_as_uint(cost));                // (costs are not negative: their bits order as they do)
    return schedule_of(items, m.kb, __ffs((int)__ballot_sync(0xffffffffu, __float_as_uint(cost) == least)));
}

// One product of the streaming kernel (nm_ffn_stream.cu): rows of a token operand against weights of their expert.
enum { kOutAct = 0, kOutHidden = 1, kOutDown = 2 };
struct ProductArgs {
    int rows;                          // token rows there are (kOutAct), or pairs
    int N, K;                          // outputs (of one of the two parts, where gated), inner dimension
    int R;                             // rows of a tile, the accumulator's columns: 16, 32, 64 or 128
    float expected_rows;               // of a tile
    long row_tiles;                    // there may be
    int terms;                         // 16-bit terms that a token value is the sum of
    bool col, f16;
    bool gather;                       // token rows by the plan's order (one term)
    bool planned;                      // row tiles from the plan; else tile i is rows i * R ..
    bool early_weights;                // weights (and the plan) may be read ahead of the programmatic wait
    bool programmatic;                 // launched so
    int act;
    RowPlan plan;
    const void *W; long w_expert;      // weights, elements between experts; parts of a gated product behind each other (NM_COL_MAJOR: rows, NM_ROW_MAJOR: columns)
    int E;
    const void *x; long ldx; long x_rows; long x_term;  // token operand: row pitch, rows, elements between terms
    // outputs
    const void *bias, *residual; long ld_residual;
    void *out; long ldo;               // kOutAct: 16-bit C; kOutHidden: 16-bit terms [2][rows][ldo] (bf16) or fp32 [rows][ldo] (fp16); kOutDown: fp32 [rows][ldo]
    const float *row_scale;            // kOutDown: factor of each row, or NULL
    float *partial; unsigned *counters; int ticket;
};
// The widest row tile for `rows` rows a group on average (at most `most`), the 128-wide slabs of weights that an item of N outputs has, and the workspace for
// sums of chunks.
int stream_tile_rows(double average, int most);
int stream_slabs(int N, bool gated);
size_t stream_partial_bytes(int R, int N, int K, bool gated, long row_tiles);
CutModel stream_cut_model(int R, float rows, int N, int K, bool gated, int terms, long row_tiles);
cudaError_t launch_product(int mode, bool gated, const ProductArgs &p, cudaStream_t s, const char **what);

}  // namespace nm
