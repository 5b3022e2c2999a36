// Routing of tokens to experts: scores, a bias for balance, groups, the top k, their weights.
//
// Per token, over its E logits x:
//     s = softmax(x)  or  sigmoid(x),   key = s + bias
//     groups of E / G experts count as their best key (or the sum of their two best); the `keep` best groups stay
//     the k largest keys among them, ties to the lowest index, in falling order;  weight = s [/ sum of the chosen s] * scale
//
// One warp a token, expert 32 i + lane in register i of a lane.  Which expert is chosen is a matter of comparisons, and what it says is decided in 64 bits:
//   - keys in fp32 come first.  Without a bias that is the logit itself, which orders as the score does (while the score in 64 bits tells neighbouring logits
//     apart); with one it is the score in fp32 plus the bias, off by no more than a bound that goes with it.
//   - where two keys whose order matters (neighbours among the chosen, the last chosen and the best that is left, the last group kept and the best that is
//     not) are nearer than that, the token is done again with fp64 keys.  Equal logits without a bias are equal keys, and no doubt.
// A key becomes an unsigned word that orders as it does; a round of the selection is a warp reduction and a vote (in 64 bits three reductions: high half,
// low half, index).  The chosen scores, and the sum of all where the weights are not renormalised, are always fp64.
// Bound by latency: a token is two selections of k dependent rounds each, and at 64 registers a thread 41% of the warps are there to cover them; 53% of the issue slots are
// used.  8192 tokens over 320 experts in groups take 26 to 27 us, all of them in fp64 52.
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
    int group_shift;                            // lanes a group: 2^group_shift
    unsigned group_mul;                         // e / group_size = e * group_mul >> 20, for e < 1024 (a division takes three conversions in the unit that is the bound)
    float scale;
    Span in_logits, in_bias, in_experts, in_weights;
    unsigned *status;
};

template <typename T> struct Logit;
template <> struct Logit<float> { __device__ static float get(const float *p, const RouteArgs &a) { return NM_LD(p, a.in_logits, a.status); } };
template <> struct Logit<bf16_t> { __device__ static float get(const bf16_t *p, const RouteArgs &a) { return Elem<bf16_t>::widen(NM_LD(p, a.in_logits, a.status)); } };
template <> struct Logit<f16_t> { __device__ static float get(const f16_t *p, const RouteArgs &a) { return Elem<f16_t>::widen(NM_LD(p, a.in_logits, a.status)); } };

// A NaN logit counts as minus infinity.
template <typename TL>
__device__ __forceinline__ float logit_of(const TL *row, int e, const RouteArgs &a)
{
    const float x = Logit<TL>::get(row + e, a);
    return x == x ? x : -INFINITY;
}

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

// Where the groups' best keys lie: the lanes of a group of lanes share a group of experts, `take(v)` of them merged by `merge`.
struct GroupLanes { int shift, each, group, sub; };              // lanes a group (a power of two), this lane's group and place
__device__ __forceinline__ GroupLanes group_lanes(const RouteArgs &a, int lane)
{
    return GroupLanes{a.group_shift, 1 << a.group_shift, lane >> a.group_shift, lane & ((1 << a.group_shift) - 1)};
}

// The two largest of a group's keys, over the lanes that share it.
template <typename K>
__device__ __forceinline__ void best_two(const K *keys, const RouteArgs &a, const GroupLanes &g, K lowest, K &first, K &second)
{
    first = lowest; second = lowest;
    if (g.group < a.groups)
#pragma unroll 4
        for (int j = g.sub; j < a.group_size; j += g.each) {
            const K v = keys[g.group * a.group_size + j];
            if (v > first) { second = first; first = v; }
            else if (v > second) second = v;
        }
    for (int o = 1; o < g.each; o <<= 1) {
        const K f = __shfl_xor_sync(kAll, first, o), s = __shfl_xor_sync(kAll, second, o);
        second = f > first ? (first > s ? first : s) : (second > f ? second : f);
        first = f > first ? f : first;
    }
}

// The chosen experts with fp64 keys: lane j returns the j-th.  `m` is the largest logit.
template <typename TL, int kPer>
__device__ __noinline__ int choose64(const RouteArgs &a, const TL *row, float m, double *mine, int lane)
{
    unsigned long long key[kPer];
    double sum = 1.0;
    if (!a.sigmoid) {
        sum = 0.0;
#pragma unroll
        for (int i = 0; i < kPer; ++i)
            if (32 * i + lane < a.E) sum += numerator(logit_of(row, 32 * i + lane, a), m);
        sum = warp_sum(sum);
        if (sum == 0.0) sum = 1.0;
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int e = 32 * i + lane;
        key[i] = 0ull;
        if (e < a.E) {
            const float x = logit_of(row, e, a);
            double s = a.sigmoid ? sigmoid64(x) : numerator(x, m) / sum;
            if (a.bias) s += (double)NM_LD(a.bias + e, a.in_bias, a.status);
            key[i] = ordered(s);
            if (a.groups > 1) mine[e] = s == s ? s : -INFINITY;
        }
    }
    if (a.groups > 1) {
        __syncwarp();
        const GroupLanes g = group_lanes(a, lane);
        double first, second;
        best_two<double>(mine, a, g, -INFINITY, first, second);
        unsigned long long of_group = g.group < a.groups && g.sub == 0 ? ordered(a.best == 2 ? first + second : first) : 0ull;
        unsigned kept = 0u;
        for (int j = 0; j < a.keep; ++j) {
            const int at = warp_best(of_group, lane);
            kept |= 1u << (at >> g.shift);
            if (lane == at) of_group = 0ull;
        }
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int e = 32 * i + lane;
            if (e < a.E && !(kept >> ((unsigned)e * a.group_mul >> 20) & 1u)) key[i] = 0ull;
        }
    }
    int chosen = 0, at = 0;
    unsigned long long best = 0ull;
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
    return chosen;
}

// fp32 keys as words that order as they do; 0 is below every key.
__device__ __forceinline__ unsigned ordered32(float key)
{
    const unsigned b = __float_as_uint(key + 0.f);                // (-0 as 0)
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float key_of(unsigned word) { return __uint_as_float(word & 0x80000000u ? word & 0x7fffffffu : ~word); }

template <typename TL, int kPer>
__global__ void __launch_bounds__(kRouteWarps * 32) route_kernel(const RouteArgs a)
{
    extern __shared__ double s_keys[];                          // [warp][E], where there are groups
    __shared__ unsigned s_cand[kRouteWarps][64];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const long t = (long)blockIdx.x * kRouteWarps + warp;
    pdl_launch_dependents();
    pdl_wait_prior_grids();
    if (t >= a.T) return;
    const TL *row = static_cast<const TL *>(a.logits) + t * a.ld;
    float x[kPer], bias[kPer];
    float m = -INFINITY;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int e = 32 * i + lane;
        x[i] = e < a.E ? logit_of(row, e, a) : -INFINITY;
        bias[i] = a.bias && e < a.E ? NM_LD(a.bias + e, a.in_bias, a.status) : 0.f;
        m = fmaxf(m, x[i]);
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(kAll, m, o));
    double sum = 1.0;
    if (!a.sigmoid && !a.renormalise) {
        sum = 0.0;
#pragma unroll
        for (int i = 0; i < kPer; ++i)
            if (32 * i + lane < a.E) sum += numerator(x[i], m);
        sum = warp_sum(sum);
        if (sum == 0.0) sum = 1.0;
    }

    // fp32 keys, and how far each may be from its fp64 key at most: `off` + 2^-23 |key|.
    //   sigmoid: exp within 2 + 1.2 |x| steps of itself (s' = s (1 - s) of that: below 2^-23), sum 2^-24 and quotient 2^-22 of s <= 1: below 2^-21; the bias adds
    //   half a step of the key
    //   softmax: exp(x - m) within 3 + 1.2 |x - m| steps (times exp(x - m): below 2^-21), a sum of up to 32 + 5 roundings, reciprocal and product: below 2^-18 of the
    //   largest score, 1 / sum
    //   the logit itself: exact, where fp64 scores tell what logits do: equal ones, and ones 2^-30 apart (s' is 3e-4 of that or more while a sigmoid's logits are
    //   up to 8; below, scores differ in proportion) that are not within reach of an underflow, 600 below 0 or the largest; what is beyond is `dubious`
    const bool plain = !a.bias && !(a.groups > 1 && a.best == 2);
    float off = 0.f;
    bool dubious = !(fabsf(m) < 1e30f);                           // infinities, the lowest values: in fp64
    unsigned key[kPer];
    if (plain) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) key[i] = 32 * i + lane < a.E ? ordered32(x[i]) : 0u;
        if (a.sigmoid) dubious = dubious || m > 8.f;
    } else {
        float total = 1.f;
        if (!a.sigmoid) {
            total = 0.f;
#pragma unroll
            for (int i = 0; i < kPer; ++i) { x[i] = 32 * i + lane < a.E ? __expf(x[i] - m) : 0.f; total += x[i]; }
#pragma unroll
            for (int o = 16; o; o >>= 1) total += __shfl_xor_sync(kAll, total, o);
        }
        const float share = 1.f / total;
        off = a.sigmoid ? 0x1p-21f : 0x1p-18f * share;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int e = 32 * i + lane;
            float s = a.sigmoid ? __fdividef(1.f, 1.f + __expf(-x[i])) : x[i] * share;
            s += bias[i];
            if (e < a.E && !(fabsf(s) < 1e30f)) dubious = true;
            key[i] = e < a.E ? ordered32(s) : 0u;
            x[i] = s;
        }
        dubious = __any_sync(kAll, dubious);
    }
    const float floor = a.sigmoid ? -600.f : m - 600.f;
    auto near = [&](float above, float below) {
        return plain ? !(above == below || above - below > 0x1p-30f) || !(above > floor) : !(above - below > 2.f * off + 0x1p-22f * (fabsf(above) + fabsf(below)));
    };

    if (a.groups > 1) {
        float *mine = reinterpret_cast<float *>(s_keys + (size_t)warp * a.E);
#pragma unroll
        for (int i = 0; i < kPer; ++i)
            if (32 * i + lane < a.E) mine[32 * i + lane] = x[i];
        __syncwarp();
        const GroupLanes g = group_lanes(a, lane);
        float first, second;
        best_two<float>(mine, a, g, -INFINITY, first, second);
        unsigned of_group = g.group < a.groups && g.sub == 0 ? ordered32(a.best == 2 ? first + second : first) : 0u;
        unsigned kept = 0u, last = 0u;
        for (int j = 0; j < a.keep; ++j) {
            last = __reduce_max_sync(kAll, of_group);
            const int at = __ffs((int)__ballot_sync(kAll, of_group == last)) - 1;
            kept |= 1u << (at >> g.shift);
            if (lane == at) of_group = 0u;
        }
        // the best group that is not kept; where equal keys are no doubt, the best that differs
        const unsigned next = __reduce_max_sync(kAll, plain && of_group == last ? 0u : of_group);
        // (a sum of two keys: twice the distance, and roundings of what was added; of every group, though two alone matter)
        if (a.best == 2) dubious = dubious || (g.group < a.groups && !(key_of(last) - key_of(next) > 4.f * off + 0x1p-21f * (fabsf(first) + fabsf(second))));
        else dubious = dubious || (next != 0u ? near(key_of(last), key_of(next)) : plain && !(key_of(last) > floor));
        dubious = __any_sync(kAll, dubious);
        __syncwarp();
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int e = 32 * i + lane;
            if (e < a.E && !(kept >> ((unsigned)e * a.group_mul >> 20) & 1u)) key[i] = 0u;
        }
    }

    // The k-th largest of the lanes' own largest keys bounds the k-th largest of all from below: what is not below it goes to a lane each, in the order of experts.  A
    // round then is a maximum and a vote, and the first of equals is the lowest lane.  The more choices, the lower the bound (for 32 it is the least of the maxima): of normal
    // logits over 256 experts 9 keys pass it for 8 choices, 21 for 16, 29 for 20, 40 for 24, 100 for 32.  Where more than 32 pass, the token is done again with fp64 keys: none up
    // to 14 choices, 1 of 3000 for 16, 16% for 20, 91% for 24, all for 28.  8192 tokens over 256 experts by softmax, us: 13 for 8 choices, 21 for 16, 34 for 20, 59 for 24, 67 for 32.
    int chosen = 0;                                               // lane j: the j-th choice
    if (!dubious) {
        unsigned v = key[0];
#pragma unroll
        for (int i = 1; i < kPer; ++i) v = max(v, key[i]);
        unsigned least = 0u;
        for (int j = 0; j < a.k; ++j) {
            least = __reduce_max_sync(kAll, v);
            if (lane == __ffs((int)__ballot_sync(kAll, v == least)) - 1) v = 0u;
        }
        least = max(least, 1u);
        unsigned *cand = s_cand[warp];
        int count = 0;
        unsigned under = 0u;                                      // the best key that is no candidate
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const bool is = key[i] >= least;
            const unsigned votes = __ballot_sync(kAll, is);
            const int at = count + __popc(votes & ((1u << lane) - 1u));
            if (is && at < 32) { cand[at] = key[i]; cand[32 + at] = 32u * i + lane; }
            if (!is) under = max(under, key[i]);
            count += __popc(votes);
        }
        __syncwarp();
        if (count > 32) {
            dubious = true;                                       // (many choices, or many equal keys)
        } else {
            v = lane < count ? cand[lane] : 0u;
            const int e = lane < count ? (int)cand[32 + lane] : 0;
            unsigned mine = 0u;
            for (int j = 0; j < a.k; ++j) {
                const unsigned top = __reduce_max_sync(kAll, v);
                const int from = __ffs((int)__ballot_sync(kAll, v == top)) - 1, who = __shfl_sync(kAll, e, from);
                if (lane == j) { chosen = who; mine = top; }
                if (lane == from) v = 0u;
            }
            // neighbours among the chosen; the last one and the best that is left (where equal keys are no doubt, the best that differs)
            const unsigned last = __shfl_sync(kAll, mine, a.k - 1), left = __reduce_max_sync(kAll, max(under, plain && v == last ? 0u : v));
            const unsigned below = __shfl_down_sync(kAll, mine, 1);
            if (lane < a.k - 1) dubious = near(key_of(mine), key_of(below));
            if (lane == a.k - 1) dubious = left != 0u ? near(key_of(last), key_of(left)) : plain && !(key_of(last) > floor);
            dubious = __any_sync(kAll, dubious);
        }
    }
    if (dubious) chosen = choose64<TL, kPer>(a, row, m, s_keys + (size_t)warp * a.E, lane);

    double w = 0.0;
    if (lane < a.k) w = a.sigmoid ? sigmoid64(logit_of(row, chosen, a)) : numerator(logit_of(row, chosen, a), m) / sum;
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

// Experts a lane: the least of 2, 4, .. 16, 20, 24 and 32 that holds them all.  Two more than needed cost 4 to 13% (8192 tokens, sigmoid and bias, no groups, us: 64 experts
// with two or four 11.2, 11.9; 160 with six or eight 13.9, 15.0; 256 with eight or ten 16.8, 17.9; 320 with ten or twelve 20.2, 22.8; 448 with fourteen or
// sixteen 25.6, 27.3; 640 with twenty or twenty-four 38.9, 44.0, with thirty-two 51.8; 768 with twenty-four or thirty-two 50.6, 58.3).  Wider steps from sixteen on, where
// the kernel is at its registers' bound (sixteen: 72, twenty 91, twenty-four 101, thirty-two 128): twenty-eight is no faster than thirty-two (896 without a bias 38.8 and
// 36.6, 16 tokens 9.2 and 8.5).
template <typename TL, int kPer>
cudaError_t launch_by_width(const RouteArgs &a, cudaStream_t s)
{
    if constexpr (32 * kPer >= kMaxE) return launch_route<TL, kPer>(a, s);
    else return a.E <= 32 * kPer ? launch_route<TL, kPer>(a, s) : launch_by_width<TL, kPer + (kPer < 16 ? 2 : kPer < 24 ? 4 : 8)>(a, s);
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
    a.group_mul = ((1u << 20) + a.group_size - 1) / a.group_size;
    for (a.group_shift = 0; a.groups << (a.group_shift + 1) <= 32; ++a.group_shift) {}
    a.sigmoid = score == NM_SCORE_SIGMOID; a.renormalise = renormalise != 0; a.scale = scale;
    a.in_logits = make_span(logits, size * ((size_t)(T - 1) * ld_logits + E));
    a.in_bias = make_span(bias, bias ? 4 * (size_t)E : 0);
    a.in_experts = make_span(experts, 4 * (size_t)T * top_k);
    a.in_weights = make_span(weights, 4 * (size_t)T * top_k);
    a.status = bounds_status_ptr();
    cudaStream_t s = (cudaStream_t)stream;
    const cudaError_t e = dtype == NM_F32 ? launch_by_width<float, 2>(a, s) : dtype == NM_BF16 ? launch_by_width<bf16_t, 2>(a, s) : launch_by_width<f16_t, 2>(a, s);
    return e == cudaSuccess ? NM_OK : record_cuda_error(e, "expert routing launch");
}

#pragma GCC visibility pop
}  // extern "C"
