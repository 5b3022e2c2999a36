// Routing of tokens to experts: scores, a bias for balance, groups, the top k, their weights.
//
// Per token, over its E logits x:
//     s = softmax(x)  or  sigmoid(x),   key = s + bias
//     groups of E / G experts count as their best key (or the sum of their two best); the `keep` best groups stay
//     the k largest keys among them, ties to the lowest index, in falling order;  weight = s [/ sum of the chosen s] * scale
//
// One warp a token, expert 32 i + lane in register i of a lane.  Which expert is chosen is a matter of comparisons, so scores and keys are
// fp64: two keys that differ are told apart whatever the order their sums were taken in, and 64-bit arithmetic is a small part of what
// bounds the kernel (latency for few tokens).  A key becomes an unsigned word that orders as
// the key does, and a round of the selection is a maximum over a lane's own keys followed by three warp reductions of 32 bits: high half,
// low half, index.
#include "nm_async.cuh"

namespace nm {

namespace {

constexpr int kRouteWarps = 4;
constexpr int kMaxGroups = 32, kMaxTopK = 32, kMaxE = NM_MAX_EXPERTS;
constexpr unsigned kAll = 0xffffffffu;

struct RouteArgs {
    const void *logits;
    long ld;
    const float *bias;
    int32_t *experts;
    float *weights;
    int T, E, k, groups, group_size, keep, best, sigmoid, renormalise;
    float scale;
    Span in_logits, in_bias, in_experts, in_weights;
    unsigned *status;
};

template <typename T> struct Logit;
template <> struct Logit<float> { __device__ static float get(const float *p, const RouteArgs &a) { return NM_LD(p, a.in_logits, a.status); } };
template <> struct Logit<bf16_t> { __device__ static float get(const bf16_t *p, const RouteArgs &a) { return Elem<bf16_t>::widen(NM_LD(p, a.in_logits, a.status)); } };
template <> struct Logit<f16_t> { __device__ static float get(const f16_t *p, const RouteArgs &a) { return Elem<f16_t>::widen(NM_LD(p, a.in_logits, a.status)); } };

// Unsigned order of fp64 keys; a NaN counts as minus infinity, -0 as 0.  0 is below every key: what may not be chosen (any more).
__device__ __forceinline__ unsigned long long ordered(double key)
{
    if (key != key) key = -__longlong_as_double(0x7ff0000000000000ll);
    const unsigned long long b = (unsigned long long)__double_as_longlong(key + 0.0);
    return b & 0x8000000000000000ull ? ~b : b | 0x8000000000000000ull;
}

__device__ __forceinline__ double warp_sum(double v)
{
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(kAll, v, o);
    return v;
}

// exp(x - m), with m the largest logit: its limits where m is infinite (only the infinite logits share the weight; none, if all are -inf).
__device__ __forceinline__ double numerator(float x, float m)
{
    if (m == INFINITY) return x == INFINITY ? 1.0 : 0.0;
    return x == -INFINITY ? 0.0 : exp((double)x - (double)m);
}
__device__ __forceinline__ double sigmoid64(float x) { return 1.0 / (1.0 + exp(-(double)x)); }

// The lane and value of the largest word over the warp; ties to the lowest `index`.
__device__ __forceinline__ int warp_best(unsigned long long v, int index)
{
    const unsigned hi = __reduce_max_sync(kAll, (unsigned)(v >> 32));
    const bool top = (unsigned)(v >> 32) == hi;
    const unsigned lo = __reduce_max_sync(kAll, top ? (unsigned)v : 0u);
    return (int)__reduce_min_sync(kAll, top && (unsigned)v == lo ? (unsigned)index : kAll);
}

template <typename TL, int kPer>
__global__ void __launch_bounds__(kRouteWarps * 32) route_kernel(const RouteArgs a)
{
    extern __shared__ double s_keys[];                          // [warp][E], where there are groups
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const long t = (long)blockIdx.x * kRouteWarps + warp;
    pdl_launch_dependents();
    pdl_wait_prior_grids();
    if (t >= a.T) return;
    const TL *row = static_cast<const TL *>(a.logits) + t * a.ld;
    auto logit = [&](int e) {
        const float x = Logit<TL>::get(row + e, a);
        return x == x ? x : -INFINITY;                          // a NaN logit counts as minus infinity
    };
    float x[kPer];
    float m = -INFINITY;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int e = 32 * i + lane;
        x[i] = e < a.E ? logit(e) : -INFINITY;
        m = fmaxf(m, x[i]);
    }
    double sum = 1.0;
    double s[kPer];
    if (a.sigmoid) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) s[i] = sigmoid64(x[i]);
    } else {
#pragma unroll
        for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(kAll, m, o));
        sum = 0.0;
#pragma unroll
        for (int i = 0; i < kPer; ++i) { s[i] = numerator(x[i], m); sum += s[i]; }
        sum = warp_sum(sum);
        if (sum == 0.0) sum = 1.0;
#pragma unroll
        for (int i = 0; i < kPer; ++i) s[i] /= sum;
    }
    unsigned long long key[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int e = 32 * i + lane;
        if (e < a.E && a.bias) s[i] += (double)NM_LD(a.bias + e, a.in_bias, a.status);
        key[i] = e < a.E ? ordered(s[i]) : 0ull;
    }

    if (a.groups > 1) {
        double *mine = s_keys + (size_t)warp * a.E;
#pragma unroll
        for (int i = 0; i < kPer; ++i)
            if (32 * i + lane < a.E) mine[32 * i + lane] = s[i] == s[i] ? s[i] : -INFINITY;
        __syncwarp();
        unsigned long long of_group = 0ull;                      // lane g: group g
        if (lane < a.groups) {
            double first = -INFINITY, second = -INFINITY;
            for (int j = 0; j < a.group_size; ++j) {
                const double v = mine[lane * a.group_size + j];
                if (v > first) { second = first; first = v; }
                else if (v > second) second = v;
            }
            of_group = ordered(a.best == 2 ? first + second : first);
        }
        unsigned kept = 0u;
        for (int j = 0; j < a.keep; ++j) {
            const int g = warp_best(of_group, lane);
            kept |= 1u << g;
            if (lane == g) of_group = 0ull;
        }
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int e = 32 * i + lane;
            if (e < a.E && !(kept >> (e / a.group_size) & 1u)) key[i] = 0ull;
        }
    }

    int chosen = 0;                                              // lane j: the j-th choice
    unsigned long long best = 0ull;
    int at = 0;
    auto local_best = [&] {
        best = key[0]; at = lane;
#pragma unroll
        for (int i = 1; i < kPer; ++i)
            if (key[i] > best) { best = key[i]; at = 32 * i + lane; }
    };
    local_best();
    for (int j = 0; j < a.k; ++j) {
        const int e = warp_best(best, at);
        if (lane == j) chosen = e;
        if (at == e) {
#pragma unroll
            for (int i = 0; i < kPer; ++i)
                if (32 * i + lane == e) key[i] = 0ull;
            local_best();
        }
    }

    double w = 0.0;
    if (lane < a.k) w = a.sigmoid ? sigmoid64(logit(chosen)) : numerator(logit(chosen), m) / sum;
    if (a.renormalise) {
        const double total = warp_sum(w);
        w = total > 0.0 ? w / total : 0.0;
    }
    if (lane < a.k) {
        NM_ST(a.experts + t * a.k + lane, chosen, a.in_experts, a.status);
        NM_ST(a.weights + t * a.k + lane, (float)(w * (double)a.scale), a.in_weights, a.status);
    }
}

template <typename TL, int kPer>
cudaError_t launch_route(const RouteArgs &a, cudaStream_t stream)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ceil_div(a.T, kRouteWarps));
    cfg.blockDim = dim3(kRouteWarps * 32);
    cfg.dynamicSmemBytes = a.groups > 1 ? (size_t)kRouteWarps * a.E * sizeof(double) : 0;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = programmatic_launch_enabled() ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, route_kernel<TL, kPer>, a);
}

template <typename TL>
cudaError_t launch_by_width(const RouteArgs &a, cudaStream_t s)
{
    if (a.E <= 64) return launch_route<TL, 2>(a, s);
    if (a.E <= 128) return launch_route<TL, 4>(a, s);
    if (a.E <= 256) return launch_route<TL, 8>(a, s);
    if (a.E <= 512) return launch_route<TL, 16>(a, s);
    return launch_route<TL, 32>(a, s);
}

}  // namespace

}  // namespace nm

using namespace nm;

extern "C" {
#pragma GCC visibility push(default)

int nm_moe_route(const void *logits, long ld_logits, const float *bias, int32_t *experts, float *weights, int T, int E, int top_k,
                 nm_dtype dtype, nm_score score, int groups, int keep_groups, int group_best, int renormalise, float scale,
                 nm_stream stream)
{
    if (!logits || !experts || !weights || T < 1 || T > (1 << 24) || E < 1 || ld_logits < E || top_k < 1 || top_k > E || groups < 1 || E % groups ||
        keep_groups < 1 || keep_groups > groups || (long)keep_groups * (E / groups) < top_k || group_best < 1 || group_best > 2 ||
        group_best > E / groups || (score != NM_SCORE_SOFTMAX && score != NM_SCORE_SIGMOID))
        return NM_ERR_INVALID_ARG;
    if (E > kMaxE || top_k > kMaxTopK || groups > kMaxGroups || (dtype != NM_F32 && dtype != NM_BF16 && dtype != NM_F16)) return NM_ERR_UNSUPPORTED;
    const size_t size = dtype == NM_F32 ? 4 : 2;
    if (((uintptr_t)logits & (size - 1)) || ((uintptr_t)bias & 3u) || ((uintptr_t)experts & 3u) || ((uintptr_t)weights & 3u)) return NM_ERR_ALIGNMENT;
    RouteArgs a{};
    a.logits = logits; a.ld = ld_logits; a.bias = bias; a.experts = experts; a.weights = weights;
    a.T = T; a.E = E; a.k = top_k; a.groups = keep_groups == groups ? 1 : groups; a.group_size = E / groups; a.keep = keep_groups; a.best = group_best;
    a.sigmoid = score == NM_SCORE_SIGMOID; a.renormalise = renormalise != 0; a.scale = scale;
    a.in_logits = make_span(logits, size * ((size_t)(T - 1) * ld_logits + E));
    a.in_bias = make_span(bias, bias ? 4 * (size_t)E : 0);
    a.in_experts = make_span(experts, 4 * (size_t)T * top_k);
    a.in_weights = make_span(weights, 4 * (size_t)T * top_k);
    a.status = bounds_status_ptr();
    cudaStream_t s = (cudaStream_t)stream;
    const cudaError_t e = dtype == NM_F32 ? launch_by_width<float>(a, s) : dtype == NM_BF16 ? launch_by_width<bf16_t>(a, s) : launch_by_width<f16_t>(a, s);
    return e == cudaSuccess ? NM_OK : record_cuda_error(e, "expert routing launch");
}

#pragma GCC visibility pop
}  // extern "C"
