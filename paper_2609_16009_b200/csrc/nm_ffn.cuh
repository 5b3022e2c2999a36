// Feed-forward operators (nm_ffn.cu, nm_ffn_stream.cu): arguments shared by the kernels, activations, the plan of rows by expert.
#pragma once

#include "nm_async.cuh"

namespace nm {

// ---- activations, fp32 -------------------------------------------------------------------------------------------------------
__device__ __forceinline__ float activate(int act, float x)
{
    switch (act) {
    case NM_ACT_RELU: return x < 0.f ? 0.f : x;                                        // a NaN stays one
    case NM_ACT_SILU: return x / (1.f + expf(-x));
    case NM_ACT_GELU: return 0.5f * x * erfcf(-0.70710678f * x);                        // erfc: no cancellation for negative x
    case NM_ACT_GELU_TANH: return x / (1.f + expf(-1.59576912f * (x + 0.044715f * x * x * x)));   // 0.5 (1 + tanh z) = 1 / (1 + exp(-2 z))
    default: return x;
    }
}

// A value of either 16-bit type, and rounding to it.
__device__ __forceinline__ float widen16(uint16_t v, bool f16) { return f16 ? __half2float(__ushort_as_half(v)) : __uint_as_float((uint32_t)v << 16); }
__device__ __forceinline__ uint16_t round16(float v, bool f16) { return f16 ? __half_as_ushort(__float2half_rn(v)) : __bfloat16_as_ushort(__float2bfloat16_rn(v)); }

// Rows of the experts.  Pair p = (token p / top_k, choice p % top_k) belongs to expert experts[p] - first where that is one of the E held
// here.  `order` lists the pairs by expert, each expert's in rising order; `place` is its inverse; a tile is up to R of one expert's rows.
struct RowTile { int expert, row0, rows, unused; };
struct RowPlan {
    const RowTile *tiles;
    const int *n_tiles;
    const int *order;                  // [sorted row] -> pair
    const int *place;                  // [pair] -> sorted row
    int top_k;
};

// One product of the streaming kernel (nm_ffn_stream.cu): rows of a token operand against weights of their expert.
enum { kOutAct = 0, kOutHidden = 1, kOutDown = 2 };
struct ProductArgs {
    int rows;                          // token rows there are (kOutAct), or pairs
    int N, K;                          // outputs (of one of the two parts, where gated), inner dimension
    int R;                             // rows of a tile, the accumulator's columns: 16, 32, 64 or 128
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
    float *partial; unsigned *counters;
};
size_t stream_partial_bytes(int R, int slabs);
// The widest row tile for `rows` rows a group on average (at most `most`), and the 128-wide slabs of weights an item has.
int stream_tile_rows(double average, int most);
int stream_slabs(int R, bool gated);
cudaError_t launch_product(int mode, bool gated, const ProductArgs &p, cudaStream_t s, const char **what);

}  // namespace nm
