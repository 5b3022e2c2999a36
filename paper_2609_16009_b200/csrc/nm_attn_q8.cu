// Latent attention of a batch over the quantised cache (records: nm_mla_q8.cuh), with a prefix that all sequences share.
//
//   o[t,h] = sum_j p_j row_j[:512],  p = softmax_j(scale <Q[t,h], row_j>),  row_j = s_j (k_j | r_j),  j over the prefix rows, then t's own
//
// Three launches: the queries are split and laid out (one warp per head), the pass over the rows (tcgen05), the merge of its parts.
//
// The pass.  A work item is up to 128 rows of the query matrix [T * H] x a run of cache rows: over the prefix the heads of several
// sequences fill the 128 rows of the matrix unit, so its records are read once per 128 heads, not once per sequence; a sequence's own
// rows meet its H heads.  Two CTAs per item, one per half of the 512 output columns (O[128 x 256] fp32 is half of TMEM, see
// nm_attn_wide.cu; the scores are computed by both).  The stored bytes ARE the matrix operands - nothing is unpacked:
//   scores   q' = q 2^-a (a per head) is two e4m3 terms, hi = round(q'), lo = round(q' - hi): a bf16's eight bits exactly down to 2^-10
//            of the head's largest, and 2^-19 of that absolutely below.  S = hi k^T + lo k^T (kind::f8f6f4, K = 32) + the key part in bf16
//            (kind::f16), 36 MMAs M128 N96.  Each k block serves as K-major operand here and as MN-major operand of P * V.
//   P * V    the weight of row j is p_j s_j: with t_j = score_j + log2 s_j, w_j = 2^(t_j - m + 11), m the running maximum of t (moved, and O
//            rescaled, only when it grows by more than 4).  w goes to fp16 - eleven bits, 2^-24 to 2^15, so a row 2^-27 below the largest
//            still counts, which in e4m3 it would not: many small weights beside one large one are what long caches have - and
//            from there into three e5m2 terms (fp16's upper byte is e5m2): truncate, subtract exactly, again, round the last; nine bits and
//            more.  18 MMAs M128 N128 K32 a tile, P from TMEM, fp32 accumulation.  The sum of p_j = w_j / s_j stays fp32.
// What is resident: the lo terms, half of the hi terms and the key part of Q in 112 KB of shared memory, the other half of hi in 64 columns of
// TMEM; nine 12 KB slots of [96 rows x 128 bytes] for the records.  96 rows a tile: two score buffers of 96 columns fit TMEM beside O
// and Q, so the scores of the next tile run while this one's exponentials do.  The MMAs of a tile by themselves take 3040 clocks
// (1890 for the scores, bound by shared memory's 128 bytes a clock, 1150 for P * V).
//   walk     One CTA per SM.  The tiles of all units are cut into even shares for the 74 pairs of CTAs, and a CTA walks over the items of its
//            share - one mostly, nine short sequences behind a long prefix; the ring runs on across them.
// Measured: 16 x 128 heads, 32768 shared rows and about 500 own ones each: 204 to 220 us (148 GFLOP of scores and P * V in one pass: 700 TFLOP/s, 42 % of
// the bf16 rate, at two and three terms); 16 x 128, ragged 4096: 49 us; 1 x 128, 16384: 25 us; 1 x 16, 257: 13 us.  (In
// runs of many milliseconds the power cap, 1000 W, takes the clock from 1965 to 1695 MHz: 251 us for the first.)  A tile takes 4300 clocks:
// the matrix unit waits neither for copies nor for weights then, but its MMAs run slower beside the softmax warps than alone (3770 with
// their work taken out).  Made no difference: no copies at all, one polling lane per warp, waits ahead of the MMAs, descriptors as 32-bit
// words, loops instead of straight-line MMAs, fewer shared-memory reads in the softmax.  Made one: MMAs issued by an elected lane of a walking
// warp (7500 -> 4500 clocks a tile), two softmax threads per row (-10 %), even shares (-14 %).
#include <algorithm>

#include <cuda_fp8.h>

#include "nm_async.cuh"
#include "nm_mla_q8.cuh"
#include "nm_tcgen05.cuh"

namespace nm {

namespace {

constexpr int kKv = 512, kRope = 64, kRec = 656;
constexpr int kM = 128;                            // query rows of an item
constexpr int kR = 96;                             // cache rows of a tile
constexpr int kQRow = 2 * kKv + 2 * kRope;         // bytes of a prepared query: hi | lo | key part
constexpr int kQBlock = kM * 128, kSlotBytes = kR * 128, kSlots = 9;
constexpr int kQBytes = 7 * kQBlock;               // lo 0-3, hi of this half's two blocks, key part
constexpr int kTables = 4, kTableBytes = kTables * kR;
constexpr int kSmemBytes = 1024 + kQBytes + kSlots * kSlotBytes + kTableBytes + 256;
static_assert(kSmemBytes <= 232448, "shared memory");
constexpr int kSoftmax = 256, kThreads = 64 + kSoftmax;       // TMA, MMA, two softmax threads per query row
constexpr uint32_t kColO = 0, kColS = 256, kColQ = 448;
constexpr float kHeadroom = 11.f, kLazy = 4.f;     // log2: weights are at most 2^(11 + 4)
constexpr int kMaxT = NM_MAX_Q8_BATCH, kPairs = kSMs / 2;
constexpr int kMaxRows = 1 << 30;                  // of the prefix, of a sequence: row numbers a few tiles past the end stay 32-bit
constexpr int kMaxUnits = 2 * kMaxT;               // query tiles of the prefix (at most 64 * 128 / 128) and sequences
constexpr int kMaxItems = kMaxUnits + kPairs;      // every unit once, and one more where a pair's share ends inside a unit

struct Item {
    int q_row, n_q;                                // query rows
    int source;                                    // 0: the prefix, 1 + t: sequence t
    int row0, row1;                                // cache rows
    int out_row;                                   // where its partial results start
};
struct PassArgs {
    CUtensorMap q;                                 // [rows][1152] bytes, boxes of 128 x 128
    CUtensorMap k[1 + kMaxT];                      // records as bytes, boxes of 128 x 96
    const unsigned char *records[1 + kMaxT];
    const unsigned char *q_rows;
    const float *q_mult;
    float *ml, *O;
    unsigned *status;
    int total_q;
    short first[kPairs + 1];                       // items of each pair of CTAs
    Item items[kMaxItems];
#ifdef NM_BOUNDS_CHECK
    int pause_where, pause_warp;                   // see nm_debug_set_attention_q8_pause
    unsigned pause_ns;
    Span in_records[1 + kMaxT], in_q, in_mult, in_ml, in_O;       // extents of the operands
#endif
};
struct MergeArgs {
    const float *ml, *O;
    uint16_t *o_bf16;
    float *o_f32, *lse;
    int H, tile_rows;                              // query rows of a prefix item
    int prefix_row[kMaxT], own_row[kMaxT];         // first partial row of each query tile of the prefix, of each sequence
    short prefix_n[kMaxT], own_n[kMaxT];           // and their parts
    unsigned *status;                              // of the debug build's checks, as the rest
#ifdef NM_BOUNDS_CHECK
    Span in_ml, in_O, in_bf16, in_f32, in_lse;
#endif
};

__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// ---- queries ---------------------------------------------------------------------------------------------------------
__global__ void __launch_bounds__(128) q8_prepare_kernel(const uint16_t *__restrict__ Q, long q_stride, int T, int H, unsigned char *__restrict__ q_rows,
                                                         float *__restrict__ q_mult, float scale_log2, unsigned *status)
{
    const Span in_q = make_span(Q, 2 * ((T - 1) * (size_t)q_stride + H * (kKv + kRope))), in_rows = make_span(q_rows, (size_t)T * H * kQRow),
               in_mult = make_span(q_mult, 4 * (size_t)T * H);
    (void)in_q; (void)in_rows; (void)in_mult; (void)status;        // (the debug build's)
    pdl_launch_dependents();
    const int row = blockIdx.x * 4 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    if (row >= T * H) return;
    const int t = row / H, h = row - t * H;
    const uint16_t *q = Q + t * q_stride + (long)h * (kKv + kRope);
    const uint4 a = NM_LD(reinterpret_cast<const uint4 *>(q + 16 * lane), in_q, status), b = NM_LD(reinterpret_cast<const uint4 *>(q + 16 * lane + 8), in_q, status);
    const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    const uint32_t key = NM_LD(reinterpret_cast<const uint32_t *>(q + kKv + 2 * lane), in_q, status);
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) top = __vmaxu2(top, w[j] & 0x7fff7fffu);
    uint32_t top_key = key & 0x7fff7fffu;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        top = __vmaxu2(top, __shfl_xor_sync(0xffffffffu, top, o));
        top_key = __vmaxu2(top_key, __shfl_xor_sync(0xffffffffu, top_key, o));
    }
    const uint32_t most = max(top >> 16, top & 0xffffu), most_key = max(top_key >> 16, top_key & 0xffffu);       // the largest magnitudes' bits
    const bool odd = max(most, most_key) >= 0x7f80u;
    // least exponent with |q| <= 448 * 2^e, 448 = 1.75 * 2^8 (bf16: mantissa 0x60), kept where 2^-e is a normal number and the key part
    // times 2^-e stays in range
    int e = 0;
    if (most) e = max((int)(most >> 7) - 127 - 8 + ((most & 0x7fu) > 0x60u), -112);
    e = max(e, (int)(most_key >> 7) - 127 - 100);
    const float inv = __uint_as_float((uint32_t)(127 - e) << 23);
    unsigned char *out = q_rows + (long)row * kQRow;
    uint32_t hi[4], lo[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float x[4] = {__uint_as_float(w[2 * j] << 16) * inv, __uint_as_float(w[2 * j] & 0xffff0000u) * inv, __uint_as_float(w[2 * j + 1] << 16) * inv,
                      __uint_as_float(w[2 * j + 1] & 0xffff0000u) * inv};
        hi[j] = lo[j] = 0;
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            const uint32_t c = __nv_cvt_float2_to_fp8x2(make_float2(x[2 * p], x[2 * p + 1]), __NV_SATFINITE, __NV_E4M3);
            const __half2_raw r = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)c, __NV_E4M3);
            const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&r));
            hi[j] |= c << (16 * p);
            lo[j] |= (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(x[2 * p] - f.x, x[2 * p + 1] - f.y), __NV_SATFINITE, __NV_E4M3) << (16 * p);
        }
    }
    NM_ST(reinterpret_cast<uint4 *>(out + 16 * lane), make_uint4(hi[0], hi[1], hi[2], hi[3]), in_rows, status);
    NM_ST(reinterpret_cast<uint4 *>(out + kKv + 16 * lane), make_uint4(lo[0], lo[1], lo[2], lo[3]), in_rows, status);
    const float k0 = __uint_as_float(key << 16) * inv, k1 = __uint_as_float(key & 0xffff0000u) * inv;
    const uint32_t k01 = (uint32_t)__bfloat16_as_ushort(__float2bfloat16_rn(k0)) | ((uint32_t)__bfloat16_as_ushort(__float2bfloat16_rn(k1)) << 16);
    NM_ST(reinterpret_cast<uint32_t *>(out + 2 * kKv + 4 * lane), k01, in_rows, status);
    // an infinity or a NaN in a head makes its scores NaN (and nobody else's)
    if (lane == 0) NM_ST(&q_mult[row], odd ? __uint_as_float(0x7fc00000u) : __uint_as_float((uint32_t)(127 + e) << 23) * scale_log2, in_mult, status);
}

// ---- the pass ----------------------------------------------------------------------------------------------------------
// Instruction descriptor, kind::f8f6f4: a_format e4m3 (0) or e5m2 (1), B e4m3, fp32 accumulation.
__host__ __device__ constexpr uint32_t instr_desc_f8(int m, int n, int a_format, bool b_mn_major)
{
    return (1u << 4) | ((uint32_t)a_format << 7) | ((b_mn_major ? 1u : 0u) << 16) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}
__device__ __forceinline__ void tmem_st4(uint32_t addr, const uint32_t (&r)[4])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]) : "memory");
}
__device__ __forceinline__ bool elect_one()
{
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r != 0;
}
// Matrix descriptors as their lower words - address / 16 and, above it, the leading stride / 16; the upper word (8 rows 1024 bytes
// apart, version 1, 128-byte swizzle) is the same for all.  Put together inside the instruction's own assembly: as 64-bit arithmetic
// the compiler repeats two dozen uniform instructions per MMA, and the issuing warp, not the pipe, sets the pace.
constexpr uint32_t kDescHigh = (1024u >> 4) | (1u << 14) | (2u << 29);
__device__ __forceinline__ uint32_t desc_low(uint32_t addr, uint32_t lead_bytes) { return ((addr & 0x3ffffu) >> 4) | ((lead_bytes >> 4) << 16); }
#define NM_Q8_MMA(KIND, A)                                                                                                            \
    "{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\tsetp.ne.b32 p, %4, 0;\n\tmov.b64 a, {%1, %5};\n\tmov.b64 b, {%2, %5};\n\t"                 \
    "tcgen05.mma.cta_group::1.kind::" KIND " [%0], " A ", b, %3, p;\n\t}"
__device__ __forceinline__ void mma_f8_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, bool accumulate)
{
    asm volatile(NM_Q8_MMA("f8f6f4", "a") ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"((uint32_t)accumulate), "r"(kDescHigh) : "memory");
}
__device__ __forceinline__ void mma_f8_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, bool accumulate)
{
    asm volatile(NM_Q8_MMA("f8f6f4", "[%1]") ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"((uint32_t)accumulate), "r"(kDescHigh) : "memory");
}
__device__ __forceinline__ void mma_key_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, bool accumulate)
{
    asm volatile(NM_Q8_MMA("f16", "a") ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"((uint32_t)accumulate), "r"(kDescHigh) : "memory");
}
#undef NM_Q8_MMA

// The bounded wait of the issuing warp: no function call, and every decision is the warp's vote, so that its control flow stays uniform
// to the compiler and the operands of the MMAs around it stay in uniform registers.
__device__ __forceinline__ bool wait_uniform(uint32_t bar, uint32_t par, volatile int *abort_flag, unsigned *status)
{
    if (__all_sync(0xffffffffu, mbar_try_wait(bar, par))) return true;
    const uint64_t t0 = global_timer_ns();
#pragma unroll 1
    for (;;) {
        if (__all_sync(0xffffffffu, mbar_try_wait(bar, par))) return true;
        if (__any_sync(0xffffffffu, *abort_flag != 0)) return false;
        if (__any_sync(0xffffffffu, global_timer_ns() - t0 > kWaitLimitNs)) {
            *abort_flag = 1;
            if (status) atomicOr(status, kStatusWaitExpired);
            return false;
        }
    }
}
// A whole warp's wait: one lane polls (32 of them take shared memory's time from the matrix unit), the others meet it.
__device__ __forceinline__ void warp_wait(uint32_t bar, uint32_t par, int lane, volatile int *abort_flag, unsigned *status)
{
    if (lane == 0 && !mbar_try_wait(bar, par)) mbar_wait(bar, par, abort_flag, status);
    __syncwarp();
    tc_fence_after();
}

// How often a slot of the ring has been filled after so many blocks.
__host__ __device__ constexpr int times_armed(int blocks, int slot) { return (blocks + kSlots - 1 - slot) / kSlots; }
static_assert(times_armed(0, 0) == 0 && times_armed(1, 0) == 1 && times_armed(1, 1) == 0 && times_armed(kSlots, kSlots - 1) == 1 && times_armed(kSlots + 1, 0) == 2 &&
              times_armed(kSlots + 1, 1) == 1, "the ring's slots in turn");
constexpr uint64_t kDrainLimitNs = 100000000ull;
__device__ __noinline__ void drain(uint32_t bar, uint32_t par)
{
    const uint64_t t0 = global_timer_ns();
    while (!mbar_try_wait(bar, par) && global_timer_ns() - t0 < kDrainLimitNs) {}
}

// Debug build only: one warp of every CTA is held up at a named place, so that a test can show that the order of what the warps tell each
// other does not hang on their pace.  Bounded by the clock.
enum Pause {
    kPauseAfterMaxima = 1,                         // a softmax warp, behind the barrier of a tile, before it reads its rows' maxima
    kPauseAfterWeights,                            // a softmax warp that has handed in the weights of an item's last tile
    kPauseBeforeProduct,                           // the issuing warp, with all weights of a tile in and its P * V not issued
    kPauseBeforeCopy,                              // the copying thread, a slot free and its copy not begun
    kPausePlaces = kPauseBeforeCopy
};
#ifdef NM_BOUNDS_CHECK
__device__ __noinline__ void pause_here(unsigned ns)
{
    const uint64_t t0 = global_timer_ns();
    while (global_timer_ns() - t0 < ns) __nanosleep(100);
}
#define NM_PAUSE(where) do { if (a.pause_where == (where) && a.pause_warp == warp && !*static_cast<volatile int *>(&s_abort)) pause_here(a.pause_ns); } while (0)
#else
#define NM_PAUSE(where) do {} while (0)
#endif

__global__ void __launch_bounds__(kThreads, 1) attn_q8_kernel(const __grid_constant__ PassArgs a)
{
    extern __shared__ unsigned char smem_raw[];
    const uint32_t raw_addr = smem_u32(smem_raw), base = (raw_addr + 1023u) & ~1023u;      // swizzle atoms want 1024-byte alignment
    unsigned char *smem = smem_raw + (base - raw_addr);
    const uint32_t q_addr = base, ring = base + kQBytes;
    // [4][96]: the biased exponents of a tile's scales, 16 to a read - the matrix unit wants shared memory's bandwidth for itself
    unsigned char *s_table = smem + kQBytes + kSlots * kSlotBytes;
    uint64_t *bars = reinterpret_cast<uint64_t *>(smem + kQBytes + kSlots * kSlotBytes + kTableBytes);
    const uint32_t bar_full = smem_u32(bars), bar_empty = bar_full + 8 * kSlots, bar_q = bar_empty + 8 * kSlots, bar_qt = bar_q + 8,
                   bar_s = bar_qt + 8, bar_p = bar_s + 16, bar_pv = bar_p + 16,
                   bar_free = bar_pv + 16, bar_done = bar_free + 8;
    __shared__ uint32_t s_tmem;
    // What the two threads of a row tell each other, in turn for the tiles: a thread may be a whole tile ahead of the other one's read of
    // what it told last (the next tile's scores wait for nobody's softmax), and not two - the barrier of the next tile is in between.
    __shared__ float s_pair[2][2][kM];
    __shared__ int s_abort;
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31, half = blockIdx.x & 1;
    const int pair = blockIdx.x >> 1, item0 = a.first[pair], item1 = a.first[pair + 1];
    if (tid == 0) {
        s_abort = 0;
        for (int i = 0; i < kSlots; ++i) { mbar_init(bar_full + 8 * i, 1); mbar_init(bar_empty + 8 * i, 1); }
        mbar_init(bar_q, 1);
        mbar_init(bar_qt, 128);
        for (int i = 0; i < 2; ++i) { mbar_init(bar_s + 8 * i, 1); mbar_init(bar_p + 8 * i, kSoftmax / 32); mbar_init(bar_pv + 8 * i, 1); }
        mbar_init(bar_free, kSoftmax / 32);
        mbar_init(bar_done, 1);
        mbar_init_fence();
    }
    if (warp == 1) tmem_alloc(&s_tmem, 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = s_tmem;
    pdl_launch_dependents();

    // Barriers of tile g: scores bar_s, weights bar_p and P * V bar_pv, each the one of g's parity in its phase g / 2.  A wait is by one bit of the
    // phase, so it may meet two states only: the phase before through, or its own.  The one after its own is out of reach of all of them -
    // scores g + 2 are issued behind the wait for the weights of g, and P * V of g + 2 behind the waiting warp's own arrival for g + 2 - and
    // the one before is through: scores g seen say so of P * V g - 2, which was issued ahead of them.  (With one bar_pv for all tiles a
    // warp that has handed in its last weights might find two P * V outstanding, one or none: three states, and the wait for the last but one
    // takes both through for neither.)  The barriers of an item - bar_q its queries in place, bar_qt their part in TMEM, bar_free everything of it
    // read - go through one phase an item, and each is waited for once in it: queries i + 1 are asked for behind bar_free of i, which needs all
    // weights of i handed in, and those need the scores that the issuing warp gives behind its waits for i.  The ring's pair is the usual one: a slot is
    // filled behind its release and released behind the wait for its fill.

    // A tile's five blocks in ring order: the other half's two latent blocks, the key part, this half's two latent blocks (the last
    // ones to be given back: they are also V).  x: byte offset in the record.
    const int other = 2 * (half ^ 1), mine = 2 * half;
    auto block_x = [&](int j) { return j < 2 ? 128 * (other + j) : (j == 2 ? kKv : 128 * (mine + j - 3)); };

    // Copies of blocks and of queries begun by thread 0
    int blocks = 0, queries = 0;

    // The CTA takes its items one after another; the ring runs on from one to the next, so an item's records are on their way while the
    // one before it is being finished.
    if (warp == 0) {
        if (lane == 0) {
            tma_prefetch_descriptor(&a.q);
            const uint64_t keep = l2_policy_evict_last();
            int slot = 0, par = 1;                                 // (parity 1: a fresh barrier's phase before the first counts as complete)
            bool ok = true;
            auto load_queries = [&](int i) {                       // lo 0-3, hi of this half, key part
                if (i > item0 && !mbar_try_wait(bar_free, (i - item0 - 1) & 1)) ok = mbar_wait(bar_free, (i - item0 - 1) & 1, &s_abort, a.status);
                if (*static_cast<volatile int *>(&s_abort)) ok = false;        // (the item before was given up, not finished)
                if (!ok) return;
                ++queries;
                mbar_arrive_expect_tx(bar_q, kQBytes);
                for (int b = 0; b < 7; ++b)
                    tma_load_2d(q_addr + b * kQBlock, &a.q, b < 4 ? kKv + 128 * b : (b < 6 ? 128 * (mine + b - 4) : 2 * kKv), a.items[i].q_row, bar_q, keep);
            };
            for (int i = item0; i < item1 && ok; ++i) {
                const Item &it = a.items[i];
                const CUtensorMap *map_k = &a.k[it.source];
                tma_prefetch_descriptor(map_k);
                const int total = 5 * ceil_div(it.row1 - it.row0, kR);
                // An item's first tiles go ahead of its queries: these wait for the item before to be finished (the first item's for the
                // kernel that prepares them - the records were written before that began)
                const int ahead = min(total, 5);
                for (int b = 0, x = 0, row = it.row0; b < total && ok; ++b) {
                    if (b == ahead) {
                        if (i == item0) pdl_wait_prior_grids();
                        load_queries(i);
                        if (!ok) break;
                    }
                    if (!mbar_try_wait(bar_empty + 8 * slot, par) && !mbar_wait(bar_empty + 8 * slot, par, &s_abort, a.status)) { ok = false; break; }
                    NM_PAUSE(kPauseBeforeCopy);
                    ++blocks;
                    mbar_arrive_expect_tx(bar_full + 8 * slot, kSlotBytes);
                    tma_load_2d(ring + slot * kSlotBytes, map_k, block_x(x), row, bar_full + 8 * slot, keep);
                    if (++slot == kSlots) { slot = 0; par ^= 1; }
                    if (++x == 5) { x = 0; row += kR; }
                }
                if (ok && total <= ahead) {
                    if (i == item0) pdl_wait_prior_grids();
                    load_queries(i);
                }
            }
        }
    } else if (warp == 1) {
        // The whole warp walks, one elected lane issues: descriptors and addresses are then uniform values, which an MMA takes as they are.
        // (Computed by one lane in a branch of its own each MMA costs 100 to 170 clocks of issue; so, N = 96 from shared memory 57,
        // from TMEM 49, N = 128 from TMEM 65 - shared memory's and the pipe's own times.)
        constexpr uint32_t idesc_s = instr_desc_f8(kM, kR, 0, false), idesc_key = instr_desc(kM, kR, false, false), idesc_o = instr_desc_f8(kM, 128, 1, true);
        const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0), sm = __shfl_sync(0xffffffffu, base, 0);
        const bool leader = elect_one();
        bool alive = true;
        const uint32_t q_low = desc_low(sm, 16), q_other = q_low + other * (kQBlock >> 4), q_mine = q_low + mine * (kQBlock >> 4);
        // A block is waited for before the MMAs of the one before it are issued: the pipe queues only a few, and a wait between them
        // would let it run dry.
        // (After an expired wait the walk goes on, every operand in its place whatever it holds, so that the control flow stays uniform; the status
        // word disowns the result.  Only no slot is given back any more: one that is refilled has been waited for.  Of the ways to see to
        // that this one costs nothing; with `leader` taken away 16 x 128 heads behind 32768 rows took 247 us instead of 214, with the abort
        // flag looked at ahead of every copy 3 % more.)
        auto wait = [&](uint32_t bar, uint32_t par) {
            alive = wait_uniform(bar, par, &s_abort, a.status) && alive;
        };
        int wait_slot = 0, wait_par = 0, slot = 0, v_slot = 3;     // the ring's block waited for next, issued next, and the next tile's first V block
        int gs = 0, gp = 0;                                        // tiles of all items so far: scores issued, P * V issued
        for (int i = item0; i < item1; ++i) {
            const int ntiles = ceil_div(a.items[i].row1 - a.items[i].row0, kR), total = 5 * ntiles;
            int waited = 0;
            auto wait_block = [&]() {
                if (waited < total) {
                    wait(bar_full + 8 * wait_slot, wait_par);
                    if (++wait_slot == kSlots) { wait_slot = 0; wait_par ^= 1; }
                }
                ++waited;
            };
            wait(bar_q, (i - item0) & 1);
            wait(bar_qt, (i - item0) & 1);
            tc_fence_after();                                      // (for what other threads did to TMEM; copies into shared memory need none)
            wait_block();
            auto scores = [&]() {
                const uint32_t d = tm + kColS + kR * (gs & 1);
#pragma unroll
                for (int j = 0; j < 5; ++j) {
                    wait_block();                                  // (the one after this)
                    const uint32_t k = desc_low(sm + kQBytes, 16) + slot * (kSlotBytes >> 4);
                    if (leader) {
                        if (j == 2) {
                            const uint32_t q = q_low + 6 * (kQBlock >> 4);
#pragma unroll
                            for (int kk = 0; kk < 4; ++kk) mma_key_ss(d, q + 2 * kk, k + 2 * kk, idesc_key, true);
                        } else {
                            const uint32_t lo = (j < 2 ? q_other + j * (kQBlock >> 4) : q_mine + (j - 3) * (kQBlock >> 4));
                            const uint32_t hi = q_low + (j < 2 ? 0 : 4 + j - 3) * (kQBlock >> 4);
#pragma unroll
                            for (int kk = 0; kk < 4; ++kk) {       // 32 latent dimensions: 32 bytes in shared memory, 8 columns of TMEM
                                if (j < 2) mma_f8_ts(d, tm + kColQ + 32 * j + 8 * kk, k + 2 * kk, idesc_s, (j | kk) != 0);
                                else mma_f8_ss(d, hi + 2 * kk, k + 2 * kk, idesc_s, true);
                                mma_f8_ss(d, lo + 2 * kk, k + 2 * kk, idesc_s, true);
                            }
                        }
                        if (j < 3 && alive) mma_commit(bar_empty + 8 * slot);
                        if (j == 4) mma_commit(bar_s + 8 * (gs & 1));
                    }
                    __syncwarp();
                    if (++slot == kSlots) slot = 0;
                }
                ++gs;
            };
            scores();
            for (int t = 0; t < ntiles; ++t, ++gp) {
                if (t + 1 < ntiles) scores();
                wait(bar_p + 8 * (gp & 1), (gp >> 1) & 1);
                NM_PAUSE(kPauseBeforeProduct);
                tc_fence_after();
                const uint32_t p = tm + kColS + kR * (gp & 1);
                const int v_next = v_slot + 1 == kSlots ? 0 : v_slot + 1;
                const uint32_t v_low = desc_low(sm + kQBytes, 1024), b0 = v_low + v_slot * (kSlotBytes >> 4), b1 = v_low + v_next * (kSlotBytes >> 4);
                if (leader) {
#pragma unroll
                    for (int v = 0; v < 2; ++v) {
#pragma unroll
                        for (int kk = 0; kk < 3; ++kk)             // 32 rows: four groups of eight, 1024 bytes apart
#pragma unroll
                            for (int term = 0; term < 3; ++term)
                                mma_f8_ts(tm + kColO + 128 * v, p + 32 * kk + 8 * term, (v ? b1 : b0) + 256 * kk, idesc_o, t > 0 || (kk | term) != 0);
                        if (alive) mma_commit(bar_empty + 8 * (v ? v_next : v_slot));
                    }
                    mma_commit(bar_pv + 8 * (gp & 1));
                }
                __syncwarp();
                v_slot += 5;
                if (v_slot >= kSlots) v_slot -= kSlots;
            }
        }
    } else {
        // ---- softmax: two threads per query row, each with 48 of a tile's cache rows (one alone needs 4000 clocks a tile, more than
        //      the matrix unit's 3100); warp w may touch the TMEM lanes of quarter w % 4 ------------------------------------------
        const int set = (warp - 2) >> 2, quad = warp & 3, r = quad * 32 + lane;
        const uint32_t lanes = tmem + ((uint32_t)(quad * 32) << 16);
        int g = 0;                                                 // tiles of all items so far
        for (int item = item0; item < item1; ++item) {
        const Item &it = a.items[item];
        const int row0 = it.row0, row1 = it.row1, ntiles = ceil_div(row1 - row0, kR);
        const unsigned char *records = a.records[it.source];
        const int entry = set == 0 ? r : kR;                       // the row of a tile whose scale this thread fetches, if there is one
        auto row_entry = [&](float s) {                            // (a record of zeros is a row of zeros, and has its weight: 2^-60 will do for its s)
            return (unsigned char)(s == 0.f ? 127 - 60 : __float_as_uint(s) >> 23);
        };
        auto row_scale = [&](int t) {
            const int row = row0 + t * kR + entry;
            const float *s = reinterpret_cast<const float *>(records + (long)row * kRec + kKv + 2 * kRope);
            return entry < kR && row < row1 && NM_INSIDE(s, 4, a.in_records[it.source], a.status) ? __ldg(s) : 0.f;
        };
        const float s0 = row_scale(0), s1 = row_scale(1);
        float s_next = row_scale(2);
        if (item == item0) pdl_wait_prior_grids();
        if (set == 0) {
            // the hi terms of the other half's columns to TMEM, 256 bytes a row; rows past the last query are zeros
            const int q_row = it.q_row + r;
            const uint4 *src = reinterpret_cast<const uint4 *>(a.q_rows + (long)min(q_row, a.total_q - 1) * kQRow + 128 * other);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t v[16];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint4 u = q_row < a.total_q ? NM_LD(&src[4 * i + j], a.in_q, a.status) : make_uint4(0u, 0u, 0u, 0u);
                    v[4 * j] = u.x; v[4 * j + 1] = u.y; v[4 * j + 2] = u.z; v[4 * j + 3] = u.w;
                }
                tmem_st16(lanes + kColQ + 16 * i, v);
            }
            tmem_wait_st();
            tc_fence_before();
            mbar_arrive(bar_qt);
        }
        const float mult = r < it.n_q ? NM_LD(&a.q_mult[it.q_row + r], a.in_mult, a.status) : 0.f;
        if (entry < kR) { s_table[entry] = row_entry(s0); s_table[kR + entry] = row_entry(s1); }
        named_barrier_sync(1, kSoftmax);
        float m = -INFINITY, l = 0.f, l1 = 0.f;
        for (int t = 0; t < ntiles; ++t, ++g) {
            const uint32_t col = lanes + kColS + kR * (g & 1);
            // (after an expired wait every later wait returns at once: the loop runs on, so that the threads keep meeting at the
            // named barrier below, and ends with a result that the status word disowns)
            warp_wait(bar_s + 8 * (g & 1), (g >> 1) & 1, lane, &s_abort, a.status);
            uint32_t raw[3][16];                                   // three pieces of 16 cache rows
#pragma unroll
            for (int c = 0; c < 3; ++c) tmem_ld16(col + 48 * set + 16 * c, raw[c]);
            tmem_wait_ld();
            // s as a number is its exponent in place; log2 s: the exponent below 2^23's last binary place, less 2^23 and the bias
            uint32_t exps[12];
#pragma unroll
            for (int c = 0; c < 3; ++c) {
                const uint4 e = reinterpret_cast<const uint4 *>(s_table + kR * (t % kTables) + 48 * set)[c];
                exps[4 * c] = e.x; exps[4 * c + 1] = e.y; exps[4 * c + 2] = e.z; exps[4 * c + 3] = e.w;
            }
            float mx = -1e30f, mx1 = -1e30f;                       // (two chains; the start keeps a row without any finite score from becoming NaN)
#pragma unroll
            for (int c = 0; c < 3; ++c)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const uint32_t w = exps[4 * c + i / 4], e = __byte_perm(w, 0, 0x4440 + (i & 3));
                    const float x = fmaf(__uint_as_float(raw[c][i]), mult * __uint_as_float(e << 23), __uint_as_float(0x4b000000u | e) - 8388735.f);
                    raw[c][i] = __float_as_uint(x);
                }
            const int valid = row1 - (row0 + t * kR) - 48 * set;
            if (valid < 48) {                                      // (the last tile) rows past the end: no weight
#pragma unroll
                for (int c = 0; c < 3; ++c)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (16 * c + i >= valid) raw[c][i] = 0xff800000u;
            }
#pragma unroll
            for (int c = 0; c < 3; ++c)
#pragma unroll
                for (int i = 0; i < 16; i += 2) { mx = fmaxf(mx, __uint_as_float(raw[c][i])); mx1 = fmaxf(mx1, __uint_as_float(raw[c][i + 1])); }
            // One barrier a tile.  Before it: this tile's scores are in registers (P may overwrite them), its maxima are told, and the
            // table of the tile after next is written - into a buffer whose last readers passed the barrier before this one.
            s_pair[t & 1][set][r] = fmaxf(mx, mx1);
            if (entry < kR) s_table[kR * ((t + 2) % kTables) + entry] = row_entry(s_next);
            named_barrier_sync(1, kSoftmax);
            NM_PAUSE(kPauseAfterMaxima);
            s_next = row_scale(t + 3);
            mx = fmaxf(s_pair[t & 1][0][r], s_pair[t & 1][1][r]);
            const bool grow = t == 0 || mx > m + kLazy;
            if (t > 0 && __any_sync(0xffffffffu, grow)) {
                // the previous tile's P * V has to be through before O is touched; each of the row's threads takes half of the columns
                warp_wait(bar_pv + 8 * ((g - 1) & 1), ((g - 1) >> 1) & 1, lane, &s_abort, a.status);
                const float f = grow ? ex2(m - mx) : 1.f;
#pragma unroll 1
                for (int c = 128 * set; c < 128 * set + 128; c += 64) {
                    uint32_t o[2][32];
                    tmem_ld32(lanes + kColO + c, o[0]);
                    tmem_ld32(lanes + kColO + c + 32, o[1]);
                    tmem_wait_ld();
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        o[0][i] = __float_as_uint(__uint_as_float(o[0][i]) * f); o[1][i] = __float_as_uint(__uint_as_float(o[1][i]) * f);
                    }
                    tmem_st32(lanes + kColO + c, o[0]);
                    tmem_st32(lanes + kColO + c + 32, o[1]);
                }
                l *= f; l1 *= f;
            }
            if (grow) m = mx;
            const float ref = m - kHeadroom;
#pragma unroll
            for (int c = 0; c < 3; ++c) {
                uint32_t hi[4], mid[4], lo[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    uint32_t h[2], h1[2], h2[2];
                    const uint32_t w = exps[4 * c + q];
#pragma unroll
                    for (int p = 0; p < 2; ++p) {
                        const int i = 4 * q + 2 * p;
                        const float w0 = ex2(__uint_as_float(raw[c][i]) - ref), w1 = ex2(__uint_as_float(raw[c][i + 1]) - ref);
                        // 1 / s by its exponent (past the end, 0: 2^127, times no weight)
                        l = fmaf(w0, __uint_as_float(0x7f000000u - (__byte_perm(w, 0, 0x4440 + 2 * p) << 23)), l);
                        l1 = fmaf(w1, __uint_as_float(0x7f000000u - (__byte_perm(w, 0, 0x4441 + 2 * p) << 23)), l1);
                        const __half2 x = __floats2half2_rn(w0, w1);
                        h[p] = *reinterpret_cast<const uint32_t *>(&x);
                        const uint32_t top = h[p] & 0xff00ff00u;
                        const __half2 x1 = __hsub2(x, *reinterpret_cast<const __half2 *>(&top));
                        h1[p] = *reinterpret_cast<const uint32_t *>(&x1);
                        const uint32_t top1 = h1[p] & 0xff00ff00u;
                        const __half2 x2 = __hsub2(x1, *reinterpret_cast<const __half2 *>(&top1));
                        h2[p] = *reinterpret_cast<const uint32_t *>(&x2) + 0x00800080u;
                    }
                    hi[q] = __byte_perm(h[0], h[1], 0x7531); mid[q] = __byte_perm(h1[0], h1[1], 0x7531); lo[q] = __byte_perm(h2[0], h2[1], 0x7531);
                }
                // 32 cache rows have 8 columns of each term, 16 rows half of them, over the columns of their scores
                const int piece = 3 * set + c;
                const uint32_t to = col + 32 * (piece >> 1) + 4 * (piece & 1);
                tmem_st4(to, hi);
                tmem_st4(to + 8, mid);
                tmem_st4(to + 16, lo);
            }
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar_p + 8 * (g & 1));
        }
        // both of the last two: the scores of the last tile say that P * V of the last but two is through
        NM_PAUSE(kPauseAfterWeights);
        if (ntiles > 1) warp_wait(bar_pv + 8 * (g & 1), ((g - 2) >> 1) & 1, lane, &s_abort, a.status);
        warp_wait(bar_pv + 8 * ((g - 1) & 1), ((g - 1) >> 1) & 1, lane, &s_abort, a.status);
        // ---- out: the warp's 32 rows and its set's 128 columns, 64 at a time through its own corner of the queries' place (the last
        //      scores are through), so that the stores run along the rows ----------------------------------------------------------------------
        named_barrier_sync(1, kSoftmax);
        s_pair[0][set][r] = l + l1;                                // (the next item's maxima come behind its first barrier, which every reader meets)
        named_barrier_sync(1, kSoftmax);
        if (half == 0 && set == 0 && r < it.n_q)
            NM_ST(reinterpret_cast<float2 *>(a.ml + 2 * (long)(it.out_row + r)), make_float2(m, s_pair[0][0][r] + s_pair[0][1][r]), a.in_ml, a.status);
        float4 *corner = reinterpret_cast<float4 *>(smem + (4 * set + quad) * 8192);        // [32 rows][16 float4], the index XOR-ed with row & 15
        for (int c0 = 128 * set; c0 < 128 * set + 128; c0 += 64) {
            uint32_t o[2][32];
            tmem_ld32(lanes + kColO + c0, o[0]);
            tmem_ld32(lanes + kColO + c0 + 32, o[1]);
            tmem_wait_ld();
            __syncwarp();
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const uint32_t *v = &o[i >> 3][4 * (i & 7)];
                corner[lane * 16 + (i ^ (lane & 15))] = make_float4(__uint_as_float(v[0]), __uint_as_float(v[1]), __uint_as_float(v[2]), __uint_as_float(v[3]));
            }
            __syncwarp();
#pragma unroll 4
            for (int i = lane; i < 32 * 16; i += 32) {
                const int rr = i >> 4, f = i & 15, q = quad * 32 + rr;
                if (q < it.n_q)
                    NM_ST(reinterpret_cast<float4 *>(a.O + (long)(it.out_row + q) * kKv + 256 * half + c0 + 4 * f), corner[rr * 16 + (f ^ (rr & 15))], a.in_O, a.status);
            }
        }
        // the next item's queries may come: into the place just used, and (from this warp's threads) into TMEM
        fence_proxy_async();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_free);
        }
    }
    tc_fence_before();
    __syncthreads();
    if (s_abort) {
        // A wait expired: what is still under way, copies into this CTA's shared memory and products on its TMEM, gets a bounded chance to end
        // before either is given back.  Of a barrier armed n times phase n - 2 is through: it is armed again only behind what waited for that.
        if (tid == 0) {
            for (int i = 0; i < kSlots; ++i) {
                const int armed = times_armed(blocks, i);
                if (armed > 0) drain(bar_full + 8 * i, (armed - 1) & 1);
            }
            if (queries > 0) drain(bar_q, (queries - 1) & 1);
        }
        if (warp == 1) {
            if (elect_one()) mma_commit(bar_done);                 // (the lane that issued: the same one is elected every time)
            drain(bar_done, 0);
        }
        tc_fence_before();
        __syncthreads();
    }
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

// ---- the merge: one CTA per head of a sequence, four columns a thread, kGroups threads that take the parts in turn --------------------
template <int kGroups>
__global__ void __launch_bounds__(kGroups * 128) q8_merge_kernel(const __grid_constant__ MergeArgs a)
{
    constexpr int kMergeThreads = kGroups * 128;
    __shared__ float s_w[2 * kPairs + 2], s_l[2 * kPairs + 2];
    __shared__ int s_row[2 * kPairs + 2];
    __shared__ float s_red[kMergeThreads / 32];
    __shared__ float4 s_acc[kGroups > 1 ? kGroups - 1 : 1][128];
    pdl_launch_dependents();
    pdl_wait_prior_grids();
    const int t = blockIdx.x / a.H, h = blockIdx.x - t * a.H, tid = threadIdx.x, group = tid >> 7, x = tid & 127;
    const int q_tile = blockIdx.x / kM, n_prefix = a.prefix_n[q_tile], n = n_prefix + a.own_n[t];
    float mx = -INFINITY;
    for (int i = tid; i < n; i += kMergeThreads) {
        // prefix: item (tile of query rows, part); own: item (sequence, part)
        const int row = i < n_prefix ? a.prefix_row[q_tile] + i * a.tile_rows + blockIdx.x % kM : a.own_row[t] + (i - n_prefix) * a.H + h;
        const float2 ml = NM_LD(reinterpret_cast<const float2 *>(a.ml + 2 * (long)row), a.in_ml, a.status);
        s_row[i] = row;
        s_w[i] = ml.x; s_l[i] = ml.y;
        mx = fmaxf(mx, ml.x);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
    if ((tid & 31) == 0) s_red[tid >> 5] = mx;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kMergeThreads / 32; ++w) mx = fmaxf(mx, s_red[w]);
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int i = group; i < n; i += kGroups) {
        const float w = ex2(s_w[i] - mx);
        const float4 v = NM_LD(reinterpret_cast<const float4 *>(a.O + (long)s_row[i] * kKv + 4 * x), a.in_O, a.status);
        acc.x = fmaf(w, v.x, acc.x); acc.y = fmaf(w, v.y, acc.y); acc.z = fmaf(w, v.z, acc.z); acc.w = fmaf(w, v.w, acc.w);
    }
    if constexpr (kGroups > 1) {
        if (group > 0) s_acc[group - 1][x] = acc;
        __syncthreads();
        if (group > 0) return;
#pragma unroll
        for (int g = 0; g < kGroups - 1; ++g) {
            const float4 v = s_acc[g][x];
            acc.x += v.x; acc.y += v.y; acc.z += v.z; acc.w += v.w;
        }
    }
    float total = 0.f;                                             // (every thread adds the same sums in the same order)
    for (int i = 0; i < n; ++i) total = fmaf(ex2(s_w[i] - mx), s_l[i], total);
    const float inv = n > 0 ? 1.f / total : 0.f;                   // no rows: zeros, and minus infinity below
    const long at = (long)blockIdx.x * kKv + 4 * x;
    acc.x *= inv; acc.y *= inv; acc.z *= inv; acc.w *= inv;
    if (a.o_f32) NM_ST(reinterpret_cast<float4 *>(a.o_f32 + at), acc, a.in_f32, a.status);
    if (a.o_bf16) {
        const uint32_t lo = (uint32_t)__bfloat16_as_ushort(__float2bfloat16_rn(acc.x)) | ((uint32_t)__bfloat16_as_ushort(__float2bfloat16_rn(acc.y)) << 16);
        const uint32_t hi = (uint32_t)__bfloat16_as_ushort(__float2bfloat16_rn(acc.z)) | ((uint32_t)__bfloat16_as_ushort(__float2bfloat16_rn(acc.w)) << 16);
        NM_ST(reinterpret_cast<uint2 *>(a.o_bf16 + at), make_uint2(lo, hi), a.in_bf16, a.status);
    }
    if (a.lse && tid == 0) NM_ST(&a.lse[blockIdx.x], n > 0 ? (mx - kHeadroom + log2f(total)) * 0.6931471805599453f : -INFINITY, a.in_lse, a.status);
}

#ifdef NM_BOUNDS_CHECK
std::atomic<unsigned long long> g_q8_pause{0};     // place | warp | nanoseconds, from the top
#endif

// ---- host ------------------------------------------------------------------------------------------------------------------
struct Layout { size_t q_rows, mult, ml, O, total; };
Layout layout_of(int T, int H, long part_rows)
{
    auto up = [](size_t x) { return (x + 1023) & ~(size_t)1023; };
    Layout l;
    l.q_rows = 0;
    l.mult = up((size_t)T * H * kQRow);
    l.ml = l.mult + up((size_t)T * H * sizeof(float));
    l.O = l.ml + up((size_t)part_rows * 2 * sizeof(float));
    l.total = l.O + (size_t)part_rows * kKv * sizeof(float);
    return l;
}

// How the work is shared out: the tiles of all units (a tile of query rows over the prefix, a sequence over its own rows), one unit
// after another, are cut into even shares for the pairs of CTAs; a share's piece of a unit is an item.  An item costs about as much
// as three tiles beside its own (queries in, pipeline filled and drained, partial results out), so a piece is at least `cost` long:
// three where the pairs have six tiles and more, one or none where there is less to do than that and latency counts (257 rows:
// 12 us instead of 18).
inline int item_cost(long work) { return work >= 6 * kPairs ? 3 : (work >= 2 * kPairs ? 1 : 0); }
struct Unit { int source, q_row, n_q, tiles, rows, out_rows; };
// The pairs that shares of `share` need; with `place`, every item is told to it: (unit, first tile, tiles, pair).
template <typename Place>
int share_out(const Unit *units, int n, int share, int cost, Place place)
{
    int pair = 0, room = share;
    for (int u = 0; u < n; ++u) {
        for (int at = 0; at < units[u].tiles;) {
            const int rest = units[u].tiles - at;
            int take = room - cost;
            if (take < rest && take < cost) {                 // not worth a piece: the next pair's
                if (room < share) { ++pair; room = share; continue; }
                take = cost;
            }
            if (take > rest) take = rest;
            if (rest - take > 0 && rest - take < cost && rest <= share) take = rest;      // (nor is what would be left)
            place(u, at, take, pair);
            at += take;
            room -= take + cost;
            if (room <= cost) { ++pair; room = share; }
        }
    }
    return pair + (room < share);
}

bool encode_bytes_map(CUtensorMap *map, const void *ptr, long rows, long pitch, int box_rows)
{
    EncodeTiledFn enc = tensor_map_encoder();
    if (!enc) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)pitch, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)pitch};
    const cuuint32_t box[2] = {128, (cuuint32_t)box_rows}, estr[2] = {1, 1};
    return enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void *>(ptr), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename Kern, typename... Args>
cudaError_t launch_after(Kern kern, unsigned grid, unsigned threads, size_t smem, cudaStream_t stream, Args... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kern, args...);
}

}  // namespace

}  // namespace nm

using namespace nm;

extern "C" {
#pragma GCC visibility push(default)

size_t nm_mla_attention_q8_workspace_bytes(int T, int H)
{
    if (T < 1 || T > kMaxT || H < 1 || H > kM) return 0;
    return layout_of(T, H, (long)kMaxItems * std::min(kM, T * H)).total;
}

int nm_debug_set_attention_q8_pause(int where, int warp, unsigned ns)
{
#ifdef NM_BOUNDS_CHECK
    if (where < 0 || where > kPausePlaces || warp < 0 || warp >= kThreads / 32 || ns > 2000000000u) return NM_ERR_INVALID_ARG;
    g_q8_pause.store(((unsigned long long)where << 40) | ((unsigned long long)warp << 32) | ns, std::memory_order_relaxed);
    return NM_OK;
#else
    (void)where; (void)warp; (void)ns;
    return NM_ERR_UNSUPPORTED;
#endif
}

int nm_mla_attention_q8(const void *Q, long q_stride, const void *prefix, long prefix_rows, const void *cache, long cache_stride, const int *seq_lens,
                        void *o_bf16, float *o_f32, float *lse, int T, int H, int kv_lora, int rope, float scale, void *workspace,
                        size_t workspace_bytes, nm_stream stream)
{
    if (!Q || !seq_lens || T < 1 || T > kMaxT || H < 1 || prefix_rows < 0 || prefix_rows > kMaxRows || (prefix_rows > 0 && !prefix) ||
        q_stride < (long)H * (kv_lora + rope))
        return NM_ERR_INVALID_ARG;
    if (kv_lora != kKv || rope != kRope || H > kM) return NM_ERR_UNSUPPORTED;
    int longest = 0;
    for (int t = 0; t < T; ++t) {
        if (seq_lens[t] < 0 || seq_lens[t] > kMaxRows) return NM_ERR_INVALID_ARG;
        longest = std::max(longest, seq_lens[t]);
    }
    if (longest > 0 && (!cache || (T > 1 && cache_stride < (long)longest * kRec))) return NM_ERR_INVALID_ARG;
    if (((uintptr_t)Q & 15u) || q_stride % 8 || ((uintptr_t)prefix & 15u) || ((uintptr_t)cache & 15u) || cache_stride % 16 || ((uintptr_t)o_bf16 & 7u) ||
        ((uintptr_t)o_f32 & 15u) || ((uintptr_t)lse & 3u))
        return NM_ERR_ALIGNMENT;
    if (!workspace || workspace_bytes < nm_mla_attention_q8_workspace_bytes(T, H)) return NM_ERR_WORKSPACE;
    if ((uintptr_t)workspace & 15u) return NM_ERR_ALIGNMENT;

    // units: the prefix once per tile of query rows, each sequence's own rows once
    const int total_q = T * H, q_tiles = ceil_div(total_q, kM), prefix_tiles = (int)((prefix_rows + kR - 1) / kR), tile_rows = std::min(kM, total_q);
    Unit units[kMaxUnits];
    int n = 0;
    long work = 0;
    if (prefix_tiles)
        for (int q = 0; q < q_tiles; ++q) units[n++] = Unit{0, q * kM, std::min(kM, total_q - q * kM), prefix_tiles, (int)prefix_rows, tile_rows};
    for (int t = 0; t < T; ++t)
        if (seq_lens[t]) units[n++] = Unit{1 + t, t * H, H, ceil_div(seq_lens[t], kR), seq_lens[t], H};
    for (int u = 0; u < n; ++u) work += units[u].tiles;
    // the least share that does with the pairs there are
    const int cost = item_cost(work);
    long lo = std::max<long>(2 * cost, 1), hi = work + (long)cost * (n + 3) + 1;
    lo = std::max(lo, (work + (long)cost * n) / kPairs);
    while (lo < hi) {
        const long mid = (lo + hi) / 2;
        if (share_out(units, n, (int)mid, cost, [](int, int, int, int) {}) <= kPairs) hi = mid; else lo = mid + 1;
    }

    cudaStream_t s = (cudaStream_t)stream;
    const Layout lay = layout_of(T, H, (long)kMaxItems * std::min(kM, total_q));
    unsigned char *ws = static_cast<unsigned char *>(workspace);
    PassArgs pa{};
    MergeArgs ma{};
    pa.q_rows = ws + lay.q_rows;
    pa.q_mult = reinterpret_cast<float *>(ws + lay.mult);
    pa.ml = reinterpret_cast<float *>(ws + lay.ml);
    pa.O = reinterpret_cast<float *>(ws + lay.O);
    pa.total_q = total_q;
    ma.ml = pa.ml; ma.O = pa.O;
    ma.o_bf16 = static_cast<uint16_t *>(o_bf16); ma.o_f32 = o_f32; ma.lse = lse;
    ma.H = H;
    ma.tile_rows = tile_rows;
    int items = 0, out_row = 0, pairs = 0, last_unit = -1;
    share_out(units, n, (int)lo, cost, [&](int u, int at, int tiles, int pair) {
        const Unit &w = units[u];
        if (u != last_unit) {
            last_unit = u;
            (w.source ? ma.own_row[w.source - 1] : ma.prefix_row[w.q_row / kM]) = out_row;
        }
        ++(w.source ? ma.own_n[w.source - 1] : ma.prefix_n[w.q_row / kM]);
        while (pairs <= pair) pa.first[pairs++] = (short)items;
        pa.items[items++] = Item{w.q_row, w.n_q, w.source, at * kR, std::min(w.rows, (at + tiles) * kR), out_row};
        out_row += w.out_rows;
    });
    pa.first[pairs] = (short)items;
    ma.status = bounds_status_ptr();
#ifdef NM_BOUNDS_CHECK
    ma.in_ml = make_span(pa.ml, 8 * (size_t)out_row); ma.in_O = make_span(pa.O, 4 * (size_t)out_row * kKv);
    ma.in_bf16 = make_span(o_bf16, 2 * (size_t)total_q * kKv); ma.in_f32 = make_span(o_f32, 4 * (size_t)total_q * kKv); ma.in_lse = make_span(lse, 4 * (size_t)total_q);
#endif
    if (items) {
        pa.status = device_status_ptr();
#ifdef NM_BOUNDS_CHECK
        for (int i = 0; i <= T; ++i)
            pa.in_records[i] = i == 0 ? make_span(prefix, (size_t)prefix_rows * kRec) : make_span(static_cast<const unsigned char *>(cache) + (long)(i - 1) * cache_stride, (size_t)seq_lens[i - 1] * kRec);
        pa.in_q = make_span(pa.q_rows, (size_t)total_q * kQRow); pa.in_mult = make_span(pa.q_mult, 4 * (size_t)total_q);
        pa.in_ml = ma.in_ml; pa.in_O = ma.in_O;
        const unsigned long long pause = g_q8_pause.load(std::memory_order_relaxed);
        pa.pause_ns = (unsigned)pause; pa.pause_warp = (int)(pause >> 32) & 0xff; pa.pause_where = (int)(pause >> 40);
#endif
        if (!encode_bytes_map(&pa.q, pa.q_rows, total_q, kQRow, kM)) return record_cuda_error(cudaErrorInvalidValue, "cuTensorMapEncodeTiled");
        // The maps cover exactly the rows attended: what lies behind them reads as zeros (and has no weight), whatever it holds.
        for (int i = 0; i <= T; ++i) {
            const long rows = i == 0 ? prefix_rows : seq_lens[i - 1];
            const unsigned char *p = i == 0 ? static_cast<const unsigned char *>(prefix) : static_cast<const unsigned char *>(cache) + (long)(i - 1) * cache_stride;
            pa.records[i] = p;
            if (rows && !encode_bytes_map(&pa.k[i], p, rows, kRec, kR)) return record_cuda_error(cudaErrorInvalidValue, "cuTensorMapEncodeTiled");
        }
        static std::atomic<unsigned long long> configured{0};
        cudaError_t e = ensure_dynamic_smem(attn_q8_kernel, kSmemBytes, configured);
        if (e != cudaSuccess) return record_cuda_error(e, "quantised attention kernel attribute");
        q8_prepare_kernel<<<ceil_div(total_q, 4), 128, 0, s>>>(static_cast<const uint16_t *>(Q), q_stride, T, H, ws + lay.q_rows,
                                                              reinterpret_cast<float *>(ws + lay.mult), scale * 1.4426950408889634f, bounds_status_ptr());
        e = cudaGetLastError();
        if (e == cudaSuccess) e = launch_after(attn_q8_kernel, 2 * pairs, kThreads, kSmemBytes, s, pa);
        if (e != cudaSuccess) return record_cuda_error(e, "quantised attention launch");
    }
    // Four threads a part's column while their CTAs, four to an SM, need no more than two waves (8 x 128 heads, 4096 rows each: 32.7 us
    // against 35.4, 1 x 128, 16384: 26.8 against 30.6); one beyond (16 x 128, ragged 4096: 49 us against 53; 64 x 128, 1000: 62 against 78).
    const cudaError_t e = total_q <= 8 * kSMs ? launch_after(q8_merge_kernel<4>, (unsigned)total_q, 512, 0, s, ma)
                                              : launch_after(q8_merge_kernel<1>, (unsigned)total_q, 128, 0, s, ma);
    return e == cudaSuccess ? NM_OK : record_cuda_error(e, "quantised attention merge launch");
}

#pragma GCC visibility pop
}  // extern "C"
