// Feed-forward half of a decode layer: the products of the chosen experts (nm_moe_ffn) and a product with bias, activation, gate and
// residual in its epilogue (nm_matmul_act).
//
//     y[t] = residual[t] + sum_j w[t, j] * h[t, j] Wdown[e],   h[t, j] = act(x[t] Wgate[e]) o (x[t] Wup[e]),   e = experts[t, j] - first
//
// What bounds them: the weights of every expert that some token chose, read once from HBM.  The products are in nm_ffn_stream.cu; here is what stands around them - rows by
// expert, rows sorted, fp16 hidden values scaled into range, the weighted sum of a token's experts - the host side, and the products for operands that tensor
// maps cannot address (rows that do not start on 16 bytes): fp32 sums on CUDA cores, four times as long for one row of 2048 x 4004, 13 times for 100, a hundred
// and more for many (1024 tokens through 6 of 64 experts of 7168 x 1536 138 ms).
#include <algorithm>

#include "nm_ffn.cuh"

namespace nm {

namespace {

static_assert(kCounterWords * sizeof(unsigned) <= NM_WS_COUNTER_BYTES, "the counters have a place of their own");
constexpr int kMaxPairs = 1 << 22, kMaxDim = 1 << 20;  // (items and chunks are then counted in 32 bits)

// ---- products of operands of any alignment -----------------------------------------------------------------------------------
// A block of four warps computes 32 outputs of one row.  Column-major weights: a warp per output in turn, lanes along k.  Row-major: a lane
// per output, the warps along k, their sums joined in shared memory.  What is read is read element by element.  One row a block: the row stays in L1, and the weights are
// read again for every row, from L2 as far as they fit (100 rows of 2048 x 4004: 328 us, 70 for one).  It is there to be right for operands that are laid out so, not for many rows.
constexpr int kSimpleN = 32, kSimpleThreads = 128;

struct SimpleArgs {
    const void *x; long ldx; bool x_f32;       // token rows, 16-bit or fp32
    const int32_t *experts; int first, E, top_k;  // NULL: one set of weights, rows as they are
    bool x_by_pair;                             // row p of the operand belongs to pair p (else to token p / top_k)
    const uint16_t *W; long w_expert; bool col, gated, f16;
    const uint16_t *bias, *residual; long ld_residual;
    void *out; long ldo; bool out_f32;
    long rows;
    int N, K, act;
    Span in_x, in_W, in_bias, in_residual, in_out, in_experts;
    unsigned *status;
};

__global__ void __launch_bounds__(kSimpleThreads) simple_product_kernel(const SimpleArgs a)
{
    __shared__ float s_part[2][4][kSimpleN];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int ntiles = ceil_div(a.N, kSimpleN);
    const long total = a.rows * ntiles;
    pdl_launch_dependents();
    pdl_wait_prior_grids();
    for (long item = blockIdx.x; item < total; item += gridDim.x) {
        const long r = item / ntiles;
        const int n0 = (int)(item % ntiles) * kSimpleN;
        long e = 0, xr = r;
        if (a.experts) {
            e = (long)NM_LD(a.experts + r, a.in_experts, a.status) - a.first;
            if (e < 0 || e >= a.E) continue;                     // the same for the whole block
            xr = a.x_by_pair ? r : r / a.top_k;
        }
        const uint16_t *W = a.W + e * a.w_expert;
        const int parts = a.gated ? 2 : 1;
        const long wide = (long)a.N * parts;
        auto token = [&](int k) {
            return a.x_f32 ? NM_LD(static_cast<const float *>(a.x) + xr * a.ldx + k, a.in_x, a.status)
                           : widen16(NM_LD(static_cast<const uint16_t *>(a.x) + xr * a.ldx + k, a.in_x, a.status), a.f16);
        };
        __syncthreads();                                          // the sums of the item before have been read
        if (a.col) {
            for (int i = warp; i < kSimpleN * parts; i += 4) {
                const int n = n0 + i % kSimpleN, part = i / kSimpleN;
                float sum = 0.f;
                if (n < a.N) {
                    const uint16_t *w = W + ((long)part * a.N + n) * a.K;
                    for (int k = lane; k < a.K; k += 32) sum = fmaf(token(k), widen16(NM_LD(w + k, a.in_W, a.status), a.f16), sum);
                }
#pragma unroll
                for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
                if (lane == 0) s_part[part][0][i % kSimpleN] = sum;
            }
        } else {
            const int n = n0 + lane;
            for (int part = 0; part < parts; ++part) {
                float sum = 0.f;
                if (n < a.N)
                    for (int k = warp; k < a.K; k += 4) sum = fmaf(token(k), widen16(NM_LD(W + k * wide + (long)part * a.N + n, a.in_W, a.status), a.f16), sum);
                s_part[part][warp][lane] = sum;
            }
        }
        __syncthreads();
        const int n = n0 + lane;
        if (warp == 0 && n < a.N) {
            float z[2] = {0.f, 0.f};
            for (int part = 0; part < parts; ++part) {
                z[part] = s_part[part][0][lane];
                if (!a.col) z[part] = (z[part] + s_part[part][1][lane]) + (s_part[part][2][lane] + s_part[part][3][lane]);
                if (a.bias) z[part] += widen16(NM_LD(a.bias + (long)part * a.N + n, a.in_bias, a.status), a.f16);
            }
            float one[1] = {z[0]};
            activate(a.act, one);
            float v = one[0];
            if (a.gated) v *= z[1];
            if (a.residual) v += widen16(NM_LD(a.residual + r * a.ld_residual + n, a.in_residual, a.status), a.f16);
            if (a.out_f32) NM_ST(static_cast<float *>(a.out) + r * a.ldo + n, v, a.in_out, a.status);
            else NM_ST(static_cast<uint16_t *>(a.out) + r * a.ldo + n, round16(v, a.f16), a.in_out, a.status);
        }
    }
}

// ---- the weighted sum of a token's experts -----------------------------------------------------------------------------------
struct CombineArgs {
    const float *y;                             // [rows][d]
    const int *place;                           // pair -> row of y; NULL: the pair itself
    const int32_t *experts; int first, E, top_k;
    const float *weights;                       // NULL: all one
    const uint16_t *residual; long ld_residual;
    uint16_t *out; long ldo;
    int T, d;
    bool f16;
    Span in_y, in_place, in_experts, in_weights, in_residual, in_out;
    unsigned *status;
};

// A block takes kV * 256 columns of one token: the token's rows and weights once, then the choices in their order, eight rows of y asked for at a
// time; fp32 sum, one rounding.  kV = 4: 16-byte loads (d, pitches and pointers allow them); kV = 1: any.
constexpr int kCombineChoices = 64;             // choices whose rows a block keeps at a time
template <int kV>
__global__ void __launch_bounds__(256) combine_kernel(const CombineArgs a)
{
    __shared__ int s_row[kCombineChoices];
    __shared__ float s_weight[kCombineChoices];
    pdl_launch_dependents();
    const int chunks = ceil_div(a.d, 256 * kV);
    const long total = (long)a.T * chunks;
    pdl_wait_prior_grids();
    for (long item = blockIdx.x; item < total; item += gridDim.x) {
        const long t = item / chunks;
        const int n = ((int)(item % chunks) * 256 + (int)threadIdx.x) * kV;
        float sum[kV], skip[kV];
#pragma unroll
        for (int i = 0; i < kV; ++i) { sum[i] = 0.f; skip[i] = 0.f; }
        if (a.residual && n < a.d) {
            const uint16_t *r = a.residual + t * a.ld_residual + n;
            if constexpr (kV == 4) {
                const uint2 v = NM_LD(reinterpret_cast<const uint2 *>(r), a.in_residual, a.status);
                skip[0] = widen16((uint16_t)v.x, a.f16); skip[1] = widen16((uint16_t)(v.x >> 16), a.f16);
                skip[2] = widen16((uint16_t)v.y, a.f16); skip[3] = widen16((uint16_t)(v.y >> 16), a.f16);
            } else {
                skip[0] = widen16(NM_LD(r, a.in_residual, a.status), a.f16);
            }
        }
        for (int j0 = 0; j0 < a.top_k; j0 += kCombineChoices) {
            const int here = min(kCombineChoices, a.top_k - j0);
            __syncthreads();
            if ((int)threadIdx.x < here) {
                const long p = t * a.top_k + j0 + threadIdx.x;
                const long e = (long)NM_LD(a.experts + p, a.in_experts, a.status) - a.first;
                const bool held = e >= 0 && e < a.E;
                s_row[threadIdx.x] = !held ? -1 : a.place ? NM_LD(a.place + p, a.in_place, a.status) : (int)p;
                s_weight[threadIdx.x] = held && a.weights ? NM_LD(a.weights + p, a.in_weights, a.status) : 1.f;
            }
            __syncthreads();
            if (n < a.d)
                for (int j = 0; j < here; j += 8) {
                    float v[8][kV];
#pragma unroll
                    for (int q = 0; q < 8; ++q) {
                        // (some row where there is none: a load under a condition would wait for the one before it)
                        const float *y = a.y + (long)max(s_row[min(j + q, here - 1)], 0) * a.d + n;
                        if constexpr (kV == 4) {
                            const float4 f = NM_LD(reinterpret_cast<const float4 *>(y), a.in_y, a.status);
                            v[q][0] = f.x; v[q][1] = f.y; v[q][2] = f.z; v[q][3] = f.w;
                        } else {
                            v[q][0] = NM_LD(y, a.in_y, a.status);
                        }
                    }
#pragma unroll
                    for (int q = 0; q < 8; ++q)
                        if (j + q < here && s_row[j + q] >= 0)
#pragma unroll
                            for (int i = 0; i < kV; ++i) sum[i] = fmaf(s_weight[j + q], v[q][i], sum[i]);
                }
        }
        if (n < a.d) {
            uint16_t *o = a.out + t * a.ldo + n;
            if constexpr (kV == 4) {
                uint32_t w[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = round16(sum[i] + skip[i], a.f16);
                NM_ST(reinterpret_cast<uint2 *>(o), make_uint2(w[0] | w[1] << 16, w[2] | w[3] << 16), a.in_out, a.status);
            } else {
                NM_ST(o, round16(sum[0] + skip[0], a.f16), a.in_out, a.status);
            }
        }
    }
}

// ---- rows by expert ------------------------------------------------------------------------------------------------------------
// A CTA an expert: all count how many pairs each expert has (shared-memory counters), so each knows where its own rows begin, and then puts its
// pairs there in their order: a warp takes a run of pairs, counts its own among them, and writes them behind those of the warps before.  Nothing is passed
// between CTAs and the order is always the same.  The experts of up to 8192 pairs are read once and kept (16 bits each).
constexpr int kPlanThreads = 512, kPlanWarps = kPlanThreads / 32, kPlanKept = 8192;
struct PlanArgs {
    const int32_t *experts; int first, E;
    int pairs, R, top_k;
    RowTile *tiles; int *order; int *place;
    int *n_rows;                                // rows there are in all
    Schedule *schedules;                        // of the two products
    CutModel model[2];
    Span in_experts, in_tiles, in_order, in_place;
    unsigned *status;
};

__device__ __forceinline__ int2 block_sum(int2 v, int2 *s_warp)     // the same for all threads
{
    v.x = __reduce_add_sync(0xffffffffu, v.x);
    v.y = __reduce_add_sync(0xffffffffu, v.y);
    if ((threadIdx.x & 31) == 0) s_warp[threadIdx.x >> 5] = v;
    __syncthreads();
    int2 sum = make_int2(0, 0);
#pragma unroll
    for (int i = 0; i < kPlanWarps; ++i) { sum.x += s_warp[i].x; sum.y += s_warp[i].y; }
    return sum;
}

__global__ void __launch_bounds__(kPlanThreads) plan_kernel(const PlanArgs a)
{
    __shared__ int s_count[NM_MAX_EXPERTS], s_before[kPlanWarps];
    __shared__ int2 s_warp[kPlanWarps];
    __shared__ uint16_t s_expert[kPlanKept];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, mine = blockIdx.x;
    const bool kept = a.pairs <= kPlanKept;
    for (int i = tid; i < a.E; i += kPlanThreads) s_count[i] = 0;
    pdl_launch_dependents();
    pdl_wait_prior_grids();
    __syncthreads();
    constexpr uint16_t kNone = 0xffffu;
    auto expert_of = [&](int p) {
        const long e = (long)NM_LD(a.experts + p, a.in_experts, a.status) - a.first;
        return e >= 0 && e < a.E ? (uint16_t)e : kNone;
    };
#pragma unroll 4
    for (int p = tid; p < a.pairs; p += kPlanThreads) {
        const uint16_t e = expert_of(p);
        if (kept) s_expert[p] = e;
        if (e != kNone) atomicAdd(&s_count[e], 1);
    }
    __syncthreads();
    int2 before = make_int2(0, 0);
    for (int i = tid; i < mine; i += kPlanThreads) { before.x += s_count[i]; before.y += ceil_div(s_count[i], a.R); }
    before = block_sum(before, s_warp);
    const int row0 = before.x, tile0 = before.y, count = s_count[mine], own = ceil_div(count, a.R);
    if (mine == a.E - 1) {
        if (tid == 0) *a.n_rows = row0 + count;
        if (warp < 2) {                                           // a warp a product: a lane for each number of parts
            const Schedule best = best_schedule(a.model[warp], tile0 + own, lane);
            if (lane == 0) a.schedules[warp] = best;
        }
    }
    for (int i = tid; i < own; i += kPlanThreads) NM_ST(a.tiles + tile0 + i, (RowTile{mine, row0 + i * a.R, min(a.R, count - i * a.R), 0}), a.in_tiles, a.status);
    if (count == 0) return;
    // Warp w: pairs [w, w + 1) of sixteen equal runs, 32 at a time.
    const int run = ceil_div(ceil_div(a.pairs, 32), kPlanWarps) * 32, p0 = min(a.pairs, warp * run), p1 = min(a.pairs, p0 + run);
    auto votes_at = [&](int p) { return __ballot_sync(0xffffffffu, p < p1 && (kept ? s_expert[p] : expert_of(p)) == mine); };
    int n = 0;
    for (int p = p0; p < p1; p += 32) n += __popc(votes_at(p + lane));
    if (lane == 0) s_before[warp] = n;
    __syncthreads();
    int row = row0;
    for (int i = 0; i < warp; ++i) row += s_before[i];
    for (int p = p0; p < p1; p += 32) {
        const unsigned votes = votes_at(p + lane);
        if (votes >> lane & 1u) {
            const int at = row + __popc(votes & ((1u << lane) - 1u));
            NM_ST(a.order + at, (p + lane) / a.top_k, a.in_order, a.status);
            NM_ST(a.place + p + lane, at, a.in_place, a.status);
        }
        row += __popc(votes);
    }
}

// ---- rows in the order of their experts ------------------------------------------------------------------------------------------
// For tiles of many rows (see nm_ffn_stream.cu): a block a row, 16 bytes a thread.
__global__ void __launch_bounds__(256) sort_rows_kernel(const uint16_t *x, long ldx, const int *order, const int *n_rows, int d, uint16_t *to, unsigned *status, Span in_x,
                                                        Span in_order, Span in_to)
{
    pdl_launch_dependents();
    pdl_wait_prior_grids();
    const int rows = *n_rows;
    for (int r = blockIdx.x; r < rows; r += gridDim.x) {
        const uint16_t *from = x + (long)NM_LD(order + r, in_order, status) * ldx;
        for (int i = 8 * threadIdx.x; i < d; i += 2048)
            NM_ST(reinterpret_cast<uint4 *>(to + (size_t)r * d + i), NM_LD(reinterpret_cast<const uint4 *>(from + i), in_x, status), in_to, status);
    }
}

// ---- fp16: hidden values beyond the type's range ---------------------------------------------------------------------------------
// act(g) * u may leave fp16 at either end, so a row is scaled by a power of two that brings its largest value to 2^14 .. 2^15, and the product's
// row is scaled back (fp32, exact).  Two terms: 22 bits, down to 2^-40 of the row's largest.  All pairs' rows are walked over, those of choices held elsewhere too, although nobody
// wrote them: what comes of these is not read (the number of rows there are would be one more load before the first).
__global__ void __launch_bounds__(256) hidden_terms_kernel(const float *h, uint16_t *terms, float *row_scale, int rows, int n, unsigned *status, Span in_h, Span in_terms, Span in_scale)
{
    __shared__ float s_max[8];
    pdl_launch_dependents();
    pdl_wait_prior_grids();
    constexpr int kKept = 8;                                       // values a thread keeps (rows of up to 2048); the others are read again
    for (int r = blockIdx.x; r < rows; r += gridDim.x) {
        const float *x = h + (size_t)r * n;
        float kept[kKept];
        float m = 0.f;
#pragma unroll
        for (int i = 0; i < kKept; ++i) {
            const int at = i * 256 + threadIdx.x;
            kept[i] = at < n ? NM_LD(x + at, in_h, status) : 0.f;
        }
#pragma unroll
        for (int i = 0; i < kKept; ++i)
            if (fabsf(kept[i]) < INFINITY) m = fmaxf(m, fabsf(kept[i]));
        for (int at = kKept * 256 + threadIdx.x; at < n; at += 256) {
            const float v = fabsf(NM_LD(x + at, in_h, status));
            if (v < INFINITY) m = fmaxf(m, v);
        }
        m = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(m)));      // (not negative: the bits order as the values)
        __syncthreads();
        if ((threadIdx.x & 31) == 0) s_max[threadIdx.x >> 5] = m;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 8; ++i) m = fmaxf(m, s_max[i]);
        int e = 0;
        if (m > 0.f) { frexpf(m, &e); e = max(e - 15, -100); }   // (not below 2^-100: the factor back has to be a normal number)
        auto put = [&](int at, float value) {
            const float v = scalbnf(value, -e);
            const __half hi = __float2half_rn(v);
            const float rest = v - __half2float(hi);
            uint16_t *to = terms + (size_t)r * n + at;
            NM_ST(to, __half_as_ushort(hi), in_terms, status);
            NM_ST(to + (size_t)rows * n, fabsf(v) < INFINITY ? __half_as_ushort(__float2half_rn(rest)) : (uint16_t)0, in_terms, status);
        };
#pragma unroll
        for (int i = 0; i < kKept; ++i)
            if (i * 256 + (int)threadIdx.x < n) put(i * 256 + threadIdx.x, kept[i]);
        for (int at = kKept * 256 + threadIdx.x; at < n; at += 256) put(at, NM_LD(x + at, in_h, status));
        if (threadIdx.x == 0) NM_ST(row_scale + r, scalbnf(1.f, e), in_scale, status);
    }
}

template <typename... P, typename... Args>
cudaError_t launch(void (*kern)(P...), long grid, unsigned threads, bool programmatic, cudaStream_t s, const Args &...args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)std::min<long>(grid, 1 << 20));
    cfg.blockDim = dim3(threads);
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = programmatic ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kern, args...);
}

size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }

bool ffn_dtype_ok(nm_dtype t) { return t == NM_BF16 || t == NM_F16; }
bool ffn_layout_ok(nm_layout l) { return l == NM_ROW_MAJOR || l == NM_COL_MAJOR; }
bool act_ok(nm_act act) { return act >= NM_ACT_NONE && act <= NM_ACT_GELU_TANH; }

// Whether tensor maps can address rows of `pitch` 16-bit elements at p: both on 16 bytes, and no stride of 2^40 bytes.
bool stride_ok(long elements) { return elements < (1l << 39); }
bool rows_on_16(const void *p, long pitch) { return !((uintptr_t)p & 15u) && pitch % 8 == 0 && stride_ok(pitch); }

struct MoeLayout { size_t tiles, n_rows, schedules, order, place, partial, h, terms, scale, y, total; };
MoeLayout moe_layout(long pairs, int d, int inter, int E, bool f16)
{
    const int R = stream_tile_rows((double)pairs / E, (int)std::min<long>(pairs, 128));
    MoeLayout l{};
    size_t at = NM_WS_COUNTER_BYTES;
    l.n_rows = at; at += 256;
    l.schedules = at; at += 256;
    l.tiles = at; at += align256((E + pairs / 16) * sizeof(RowTile));
    l.order = at; at += align256(4 * (size_t)pairs);
    l.place = at; at += align256(4 * (size_t)pairs);
    l.scale = at; at += align256(4 * (size_t)pairs);
    const long tiles = E + pairs / R;
    l.partial = at;
    at += align256(std::max(stream_partial_bytes(R, inter, d, true, tiles), std::max(stream_partial_bytes(R, inter, d, false, tiles), stream_partial_bytes(R, d, inter, false, tiles))));
    l.h = at; at += align256(4 * (size_t)pairs * inter);
    l.terms = f16 ? at : l.h;
    if (f16) at += align256(4 * (size_t)pairs * inter);
    l.y = at; at += align256(4 * (size_t)pairs * d);
    l.total = at;
    return l;
}

}  // namespace

}  // namespace nm

using namespace nm;

extern "C" {
#pragma GCC visibility push(default)

size_t nm_matmul_act_workspace_bytes(int M, int N, int K, int gated, nm_dtype dtype)
{
    if (M < 1 || M > NM_MAX_FFN_ROWS || N < 1 || N > kMaxDim || K < 1 || K > kMaxDim || !ffn_dtype_ok(dtype)) return 0;
    const int R = stream_tile_rows(M, M);
    return NM_WS_COUNTER_BYTES + stream_partial_bytes(R, N, K, gated != 0, ceil_div(M, R));
}

int nm_matmul_act(const void *A, long lda, const void *B, const void *bias, const void *residual, long ld_residual, void *C, long ldc, int M,
                  int N, int K, nm_act act, int gated, nm_dtype dtype, nm_layout layout_B, void *workspace, size_t workspace_bytes,
                  nm_stream stream)
{
    if (!A || !B || !C || M < 1 || M > NM_MAX_FFN_ROWS || N < 1 || N > kMaxDim || K < 1 || K > kMaxDim || lda < K || ldc < N || (residual && ld_residual < N)) return NM_ERR_INVALID_ARG;
    if (!ffn_dtype_ok(dtype) || !ffn_layout_ok(layout_B) || !act_ok(act)) return NM_ERR_UNSUPPORTED;
    if (((uintptr_t)A & 1u) || ((uintptr_t)B & 1u) || ((uintptr_t)C & 1u) || ((uintptr_t)bias & 1u) || ((uintptr_t)residual & 1u)) return NM_ERR_ALIGNMENT;
    if (!workspace || workspace_bytes < nm_matmul_act_workspace_bytes(M, N, K, gated, dtype)) return NM_ERR_WORKSPACE;
    if ((uintptr_t)workspace & 15u) return NM_ERR_ALIGNMENT;
    const int parts = gated ? 2 : 1;
    cudaStream_t s = (cudaStream_t)stream;
    const bool col = layout_B == NM_COL_MAJOR, programmatic = programmatic_launch_enabled();
    if (M == 1) lda = (K + 7l) / 8 * 8;                             // (one row: its pitch is any)
    if (rows_on_16(A, lda) && rows_on_16(B, col ? K : N) && stride_ok((long)M * lda)) {
        ProductArgs p{};
        p.rows = M; p.N = N; p.K = K; p.R = stream_tile_rows(M, M); p.expected_rows = (float)std::min(M, p.R); p.row_tiles = ceil_div(M, p.R); p.terms = 1;
        p.col = col; p.f16 = dtype == NM_F16; p.early_weights = p.programmatic = programmatic;
        p.act = act;
        p.W = B; p.w_expert = (long)parts * N * K; p.E = 1;
        p.x = A; p.ldx = lda; p.x_rows = M; p.x_term = (long)M * lda;
        p.bias = bias; p.residual = residual; p.ld_residual = ld_residual;
        p.out = C; p.ldo = ldc;
        p.counters = static_cast<unsigned *>(workspace);
        p.partial = reinterpret_cast<float *>(static_cast<unsigned char *>(workspace) + NM_WS_COUNTER_BYTES);
        const char *what = "";
        const cudaError_t e = launch_product(kOutAct, gated != 0, p, s, &what);
        return e == cudaSuccess ? NM_OK : record_cuda_error(e, what);
    }
    SimpleArgs a{};
    a.x = A; a.ldx = lda;
    a.W = static_cast<const uint16_t *>(B); a.col = layout_B == NM_COL_MAJOR; a.gated = gated != 0; a.f16 = dtype == NM_F16;
    a.bias = static_cast<const uint16_t *>(bias); a.residual = static_cast<const uint16_t *>(residual); a.ld_residual = ld_residual;
    a.out = C; a.ldo = ldc;
    a.rows = M; a.N = N; a.K = K; a.act = act;
    a.in_x = make_span(A, 2 * ((size_t)(M - 1) * lda + K));
    a.in_W = make_span(B, 2 * (size_t)parts * N * K);
    a.in_bias = make_span(bias, bias ? 2 * (size_t)parts * N : 0);
    a.in_residual = make_span(residual, residual ? 2 * ((size_t)(M - 1) * ld_residual + N) : 0);
    a.in_out = make_span(C, 2 * ((size_t)(M - 1) * ldc + N));
    a.status = bounds_status_ptr();
    const cudaError_t e = launch(simple_product_kernel, (long)M * ceil_div(N, kSimpleN), kSimpleThreads, programmatic, s, a);
    return e == cudaSuccess ? NM_OK : record_cuda_error(e, "product with epilogue launch");
}

size_t nm_moe_ffn_workspace_bytes(int T, int d, int inter, int E, int top_k, nm_dtype dtype)
{
    if (T < 1 || d < 1 || d > kMaxDim || inter < 1 || inter > kMaxDim || E < 1 || E > NM_MAX_EXPERTS || top_k < 1 || (long)T * top_k > kMaxPairs || !ffn_dtype_ok(dtype)) return 0;
    return moe_layout((long)T * top_k, d, inter, E, dtype == NM_F16).total;
}

int nm_moe_ffn(const void *x, long ldx, const int32_t *experts, const float *weights, const void *W_up, const void *W_down,
               const void *residual, long ld_residual, void *out, long ldo, int T, int d, int inter, int E, int top_k, int first_expert,
               nm_act act, int gated, nm_dtype dtype, nm_layout layout, void *workspace, size_t workspace_bytes, nm_stream stream)
{
    if (!x || !experts || !W_up || !W_down || !out || T < 1 || d < 1 || d > kMaxDim || inter < 1 || inter > kMaxDim || E < 1 || top_k < 1 ||
        first_expert < 0 || ldx < d || ldo < d || (residual && ld_residual < d))
        return NM_ERR_INVALID_ARG;
    if (!ffn_dtype_ok(dtype) || !ffn_layout_ok(layout) || !act_ok(act) || E > NM_MAX_EXPERTS || (long)T * top_k > kMaxPairs) return NM_ERR_UNSUPPORTED;
    if (((uintptr_t)x & 1u) || ((uintptr_t)W_up & 1u) || ((uintptr_t)W_down & 1u) || ((uintptr_t)residual & 1u) || ((uintptr_t)out & 1u) ||
        ((uintptr_t)experts & 3u) || ((uintptr_t)weights & 3u))
        return NM_ERR_ALIGNMENT;
    if (!workspace || workspace_bytes < nm_moe_ffn_workspace_bytes(T, d, inter, E, top_k, dtype)) return NM_ERR_WORKSPACE;
    if ((uintptr_t)workspace & 15u) return NM_ERR_ALIGNMENT;
    cudaStream_t s = (cudaStream_t)stream;
    const long pairs = (long)T * top_k;
    const bool col = layout == NM_COL_MAJOR, f16 = dtype == NM_F16, programmatic = programmatic_launch_enabled();
    if (T == 1) ldx = (d + 7l) / 8 * 8;                             // (one row: its pitch is any)
    const MoeLayout lay = moe_layout(pairs, d, inter, E, f16);
    unsigned char *ws = static_cast<unsigned char *>(workspace);
    float *h = reinterpret_cast<float *>(ws + lay.h), *y = reinterpret_cast<float *>(ws + lay.y);
    const int *place = nullptr;
    const int parts = gated ? 2 : 1;
    const Span in_experts = make_span(experts, 4 * (size_t)pairs);
    unsigned *const status = bounds_status_ptr();
    const char *what = "experts' products launch";
    cudaError_t e;
    if (rows_on_16(x, ldx) && rows_on_16(W_up, col ? d : inter) && rows_on_16(W_down, col ? inter : d) && inter % 8 == 0 &&
        stride_ok((long)parts * inter * d) && stride_ok(pairs * inter) && stride_ok(pairs * d)) {
        PlanArgs pl{};
        pl.experts = experts; pl.first = first_expert; pl.E = E; pl.pairs = (int)pairs; pl.top_k = top_k;
        pl.R = stream_tile_rows((double)pairs / E, (int)std::min<long>(pairs, 128));
        pl.tiles = reinterpret_cast<RowTile *>(ws + lay.tiles); pl.n_rows = reinterpret_cast<int *>(ws + lay.n_rows);
        pl.schedules = reinterpret_cast<Schedule *>(ws + lay.schedules);
        const float rows = (float)std::min<double>(pl.R, std::max(1.0, (double)pairs / E));
        pl.model[0] = stream_cut_model(pl.R, rows, inter, d, gated != 0, 1, E + pairs / pl.R);
        pl.model[1] = stream_cut_model(pl.R, rows, d, inter, false, 2, E + pairs / pl.R);
        pl.order = reinterpret_cast<int *>(ws + lay.order); pl.place = reinterpret_cast<int *>(ws + lay.place);
        pl.in_experts = in_experts; pl.in_tiles = make_span(pl.tiles, sizeof(RowTile) * (E + (size_t)pairs / pl.R));
        pl.in_order = make_span(pl.order, 4 * (size_t)pairs); pl.in_place = make_span(pl.place, 4 * (size_t)pairs);
        pl.status = status;
        place = pl.place;
        const bool own_plan = pl.R <= 16 && pairs <= kOwnPairs;
        e = own_plan ? cudaSuccess : launch(plan_kernel, E, kPlanThreads, programmatic, s, pl);

        ProductArgs p{};
        p.rows = (int)pairs; p.N = inter; p.K = d; p.R = pl.R; p.expected_rows = rows; p.row_tiles = E + pairs / pl.R; p.terms = 1;
        p.col = col; p.f16 = f16; p.planned = true; p.programmatic = own_plan ? programmatic : true;
        p.act = act;
        p.plan = RowPlan{pl.tiles, pl.schedules, pl.order, own_plan ? (int)pairs : 0, experts, first_expert, E, top_k, pl.place};
        p.W = W_up; p.w_expert = (long)parts * inter * d; p.E = E;
        p.gather = pl.R <= 16;
        if (p.gather) {
            p.x = x; p.ldx = ldx; p.x_rows = T;
        } else {                                                  // the sorted rows lie where y will be
            uint16_t *sorted = reinterpret_cast<uint16_t *>(y);
            if (e == cudaSuccess)
                e = launch(sort_rows_kernel, pairs, 256, true, s, static_cast<const uint16_t *>(x), ldx, static_cast<const int *>(pl.order), static_cast<const int *>(pl.n_rows), d,
                           sorted, status, make_span(x, 2 * ((size_t)(T - 1) * ldx + d)), pl.in_order, make_span(sorted, 2 * (size_t)pairs * d));
            p.x = sorted; p.ldx = d; p.x_rows = pairs; p.x_term = pairs * d;
        }
        p.out = h; p.ldo = inter;
        p.counters = reinterpret_cast<unsigned *>(ws); p.ticket = kTicketUp; p.partial = reinterpret_cast<float *>(ws + lay.partial);
        if (e == cudaSuccess) e = launch_product(kOutHidden, gated != 0, p, s, &what);

        float *row_scale = reinterpret_cast<float *>(ws + lay.scale);
        uint16_t *terms = reinterpret_cast<uint16_t *>(ws + lay.terms);
        if (e == cudaSuccess && f16)
            e = launch(hidden_terms_kernel, pairs, 256, true, s, static_cast<const float *>(h), terms, row_scale, (int)pairs, inter, status, make_span(h, 4 * (size_t)pairs * inter),
                       make_span(terms, 4 * (size_t)pairs * inter), make_span(row_scale, 4 * (size_t)pairs));

        ProductArgs q = p;
        q.N = d; q.K = inter; q.terms = 2; q.gather = false; q.early_weights = true; q.act = NM_ACT_NONE;
        q.programmatic = true; q.plan.schedule = pl.schedules + 1; q.ticket = kTicketDown;
        q.W = W_down; q.w_expert = (long)inter * d;
        q.x = terms; q.ldx = inter; q.x_rows = pairs; q.x_term = pairs * inter;
        q.row_scale = f16 ? row_scale : nullptr;
        q.out = y; q.ldo = d;
        if (e == cudaSuccess) e = launch_product(kOutDown, false, q, s, &what);
    } else {
        SimpleArgs a{};
        a.x = x; a.ldx = ldx;
        a.experts = experts; a.first = first_expert; a.E = E; a.top_k = top_k;
        a.W = static_cast<const uint16_t *>(W_up); a.w_expert = (long)parts * inter * d; a.col = col; a.gated = gated != 0; a.f16 = f16;
        a.out = h; a.ldo = inter; a.out_f32 = true;
        a.rows = pairs; a.N = inter; a.K = d; a.act = act;
        a.in_x = make_span(x, 2 * ((size_t)(T - 1) * ldx + d));
        a.in_W = make_span(W_up, 2 * (size_t)E * a.w_expert);
        a.in_experts = in_experts;
        a.in_out = make_span(h, 4 * (size_t)pairs * inter);
        a.status = status;
        e = launch(simple_product_kernel, pairs * ceil_div(inter, kSimpleN), kSimpleThreads, programmatic, s, a);

        SimpleArgs b = a;
        b.x = h; b.ldx = inter; b.x_f32 = true; b.x_by_pair = true;
        b.W = static_cast<const uint16_t *>(W_down); b.w_expert = (long)inter * d; b.gated = false;
        b.out = y; b.ldo = d;
        b.N = d; b.K = inter; b.act = NM_ACT_NONE;
        b.in_x = a.in_out;
        b.in_W = make_span(W_down, 2 * (size_t)E * b.w_expert);
        b.in_out = make_span(y, 4 * (size_t)pairs * d);
        if (e == cudaSuccess) e = launch(simple_product_kernel, pairs * ceil_div(d, kSimpleN), kSimpleThreads, true, s, b);
    }

    CombineArgs c{};
    c.y = y; c.place = place; c.experts = experts; c.first = first_expert; c.E = E; c.top_k = top_k; c.weights = weights;
    c.residual = static_cast<const uint16_t *>(residual); c.ld_residual = ld_residual;
    c.out = static_cast<uint16_t *>(out); c.ldo = ldo; c.T = T; c.d = d; c.f16 = f16;
    c.in_y = make_span(y, 4 * (size_t)pairs * d); c.in_experts = in_experts; c.in_place = make_span(place, place ? 4 * (size_t)pairs : 0);
    c.in_weights = make_span(weights, weights ? 4 * (size_t)pairs : 0);
    c.in_residual = make_span(residual, residual ? 2 * ((size_t)(T - 1) * ld_residual + d) : 0);
    c.in_out = make_span(out, 2 * ((size_t)(T - 1) * ldo + d));
    c.status = status;
    const bool wide = d % 4 == 0 && ldo % 4 == 0 && !((uintptr_t)out & 7u) && (!residual || (ld_residual % 4 == 0 && !((uintptr_t)residual & 7u)));
    if (e == cudaSuccess) e = wide ? launch(combine_kernel<4>, (long)T * ceil_div(d, 1024), 256, true, s, c) : launch(combine_kernel<1>, (long)T * ceil_div(d, 256), 256, true, s, c);
    return e == cudaSuccess ? NM_OK : record_cuda_error(e, what);
}

#pragma GCC visibility pop
}  // extern "C"
