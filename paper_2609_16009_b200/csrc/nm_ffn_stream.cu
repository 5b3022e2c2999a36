// The products of the feed-forward operators on the tensor cores: weights streamed once from HBM past the rows of their expert.
//
//     D[128 outputs x rows] += W[128 outputs x 64 k] * X[rows x 64 k]^T         (the operands swapped: weights are the MMA's M dimension)
//
// Bound by the bytes of the weights while an expert has fewer than ~200 rows, so the kernel is a stream: one CTA per SM, a ring of 64-k stages
// filled by TMA, and work that is dealt out until all CTAs end together, whatever experts and outputs it belongs to.  Alone it reads 7.1 TB/s (16 tokens through
// 6 of 64 experts of 7168 x 1536, 464 us); from about 100 rows an expert on, L2 -> shared memory (8.4 TB/s of weights and rows) comes first.
//
//   item   one row tile (up to R rows of one expert) x one column tile (kSlabs slabs of 128 outputs; where gated, one slab each of gate and up,
//          so that a thread ends up with both values of an output), kb steps of 64 k
//   chunk  an item, or for the last round or two one of `parts` runs of its steps; the cuts are a rule on sizes (schedule_of), the CTAs take chunks as they
//          get done: with equal shares the fastest SMs were done after 652 us where the slowest took 870.  A chunk's fp32 sums wait in the workspace for
//          the last of its item (a counter; nobody waits), which adds them in the order of k.  So results do not depend on who took what or came last.
//   warps  0: copies, and the next chunk; 1: MMAs; from 2: the epilogue, from the other one of two accumulators.  Eight warps, two to a
//          quarter of its lanes (16 rows of 18432 x 7168: 47.9 us, 49.9 with four), or four for up to four rows (they have nothing for more, and a launch of more
//          threads takes longer)
//
// A step's token rows are ONE copy: of the four box heights there are a tensor map of, the least that holds the tile's rows.  A request costs the copy
// engine and the thread that makes it 40 to 60 ns whatever its size, and requests made by several lanes at once take their turns (two boxes of 8 rows by two lanes:
// 0.2 us a step, as much as 16 KB of weights).  Scattered rows are gathered by token where they are few (tile::gather4, four rows a request), and sorted first where not.
// The number of accumulator columns is that of the rows there are, rounded up; what the columns beyond hold is not read.
//
// A hidden value is the sum of two 16-bit terms (bf16: 16 bits and more, fp16: 22), which keeps its rounding out of the result.  A row's terms are two rows of
// the token operand: up to 64 rows one MMA takes both, in columns of their own that the epilogue adds (an MMA of 16 columns takes as long as one of 32); beyond, an
// MMA each into the same columns.
#include <algorithm>
#include <type_traits>

#include "nm_ffn.cuh"
#include "nm_tcgen05.cuh"

namespace nm {

namespace {

constexpr int kMaxThreads = 64 + 32 * 8;
constexpr int kGathered = 16;                   // token rows are gathered in tiles of up to so many (with 32 the eight tests a step alone cost 20%)
constexpr int kQueue = 4;                       // chunks that the copies may be ahead of the epilogue
constexpr int kKT = 64;                        // k of a stage
constexpr int kSlab = 128;                     // outputs of a slab (the MMA's M)
constexpr int kSlabBytes = kSlab * kKT * 2;
constexpr int kMaxStages = 12;
constexpr int kRingBytes = 216 * 1024;

std::atomic<int> g_forced_parts{0};             // nm_debug_set_ffn_cut
std::atomic<unsigned long long> g_pause{0};     // nm_debug_set_ffn_pause: place | nanoseconds, from the top

struct StreamArgs {
    Schedule schedule;                          // where the rows are known on the host
    int kb, column_tiles, tile_n;               // steps of an item, column tiles of a row tile, outputs of one
    int rows, N, R, box_rows, nstage, stage_bytes;   // box_rows: the least of the box heights, the others its multiples
    int first_map;                              // of the token maps: one that there is, and that of the first tile where its rows are known
    int acc_columns;                            // of a slab: R, twice that where the terms have columns of their own
    bool apart, few;                            // few: four rows or fewer in a tile, as far as that is known: four epilogue warps then
    unsigned tmem_columns;
    bool gather, early_weights, programmatic;
    int act;
    RowPlan plan;
    CutModel model;                             // (of a plan made here)
    const uint16_t *bias, *residual; long ld_residual;
    void *out; long ldo; long out_term;
    const float *row_scale;
    float *partial; unsigned *counters; int ticket;
    Span in_bias, in_residual, in_out, in_scale, in_partial, in_tiles, in_order, in_experts, in_place;
    unsigned *status;
    int pause_where; unsigned pause_ns;         // see nm_debug_set_ffn_pause
};

__device__ __forceinline__ bool elect_one()
{
    unsigned r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r != 0;
}

// Debug build: the CTAs' threads can be held up at named places (nm_debug_set_ffn_pause), to show that nothing depends on their pace.
constexpr int kPausePlaces = 6;
#ifdef NM_BOUNDS_CHECK
__device__ __noinline__ void pause_here(unsigned ns)
{
    const uint64_t t0 = global_timer_ns();
    while (global_timer_ns() - t0 < ns) __nanosleep(1000);
}
#define NM_PAUSE(where) do { if (a.pause_where == (where) && !*static_cast<volatile int *>(&s_abort)) pause_here(a.pause_ns); } while (0)
#else
#define NM_PAUSE(where) do { } while (0)
#endif

// Four rows of a 2-D tensor, 64 k each, to consecutive 128-byte rows of shared memory.
__device__ __forceinline__ void tma_gather4(uint32_t dst, const CUtensorMap *map, int x, int r0, int r1, int r2, int r3, uint32_t bar, uint64_t policy)
{
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cta.global.tile::gather4.mbarrier::complete_tx::bytes.L2::cache_hint"
        " [%0], [%1, {%2, %3, %4, %5, %6}], [%7], %8;"
        ::"r"(dst), "l"(map), "r"(x), "r"(r0), "r"(r1), "r"(r2), "r"(r3), "r"(bar), "l"(policy) : "memory");
}

__device__ __forceinline__ unsigned ask_ticket(unsigned *counter)
{
    unsigned t;
    asm volatile("atom.global.add.u32 %0, [%1], 1;" : "=r"(t) : "l"(counter) : "memory");
    return t;
}

// Token rows: boxes of 1, 2, 3 and 4 times box_rows rows (the first alone for gathered rows).
struct TokenMaps { CUtensorMap of[4]; };

// Debug build: a token map is looked at before it is used, as an address is; one that was not made is all zeros.
#ifdef NM_BOUNDS_CHECK
__device__ __noinline__ bool map_made(const CUtensorMap *map, unsigned *status)
{
    const uint32_t *words = reinterpret_cast<const uint32_t *>(map);
    uint32_t any = 0u;
    for (unsigned i = 0; i < sizeof(CUtensorMap) / 4; ++i) any |= words[i];
    if (!any && status) atomicOr(status, kStatusOutOfBounds);
    return any != 0u;
}
#define NM_MAP_MADE(map, st) map_made((map), (st))
#else
#define NM_MAP_MADE(map, st) true
#endif

// A chunk: steps [k0, k1) of an item; where that is not all of it, the place of its sums and of the item's first chunk's, and the item's counter.
struct Chunk { int item, k0, k1, slot, first_slot, cut; };
__device__ __forceinline__ Chunk chunk_of(const Schedule &s, int kb, int id)
{
    if (id < s.whole) return Chunk{id, 0, kb, 0, 0, -1};
    const int at = id - s.whole, cut = at / s.parts, part = at - cut * s.parts, k0 = part * s.kc;
    return Chunk{s.whole + cut, k0, min(kb, k0 + s.kc), at, cut * s.parts, cut};
}

// A plan made by the CTA itself, see RowPlan: tiles as (expert and rows, first row), the tokens of the sorted rows, the schedule.
struct OwnPlan {
    Schedule schedule;
    uint2 tiles[kOwnPairs];
    uint16_t order[kOwnPairs], expert[kOwnPairs], tiles_of[kOwnPairs];
};
// By all threads of the CTA (at least kOwnPairs of them).  A thread a pair: how many pairs have lower experts, and how many of its own come before, is where its row lies;
// the first pair of an expert stands for it.
__device__ __forceinline__ void make_plan(const StreamArgs &a, OwnPlan &own, bool place_too)
{
    const int p = threadIdx.x, pairs = a.plan.own_pairs, lane = p & 31;
    int e = 0xffff;                                               // not held here
    if (p < pairs) {
        // (past L1, as all that is read ahead of the wait: the kernel that wrote it is two back, and no wait of this one makes its lines new)
        const int32_t *at = a.plan.experts + p;
        const long v = (long)(NM_INSIDE(at, 4, a.in_experts, a.status) ? __ldcg(at) : 0) - a.plan.first;
        if (v >= 0 && v < a.plan.E) e = (int)v;
        own.expert[p] = (uint16_t)e;
    }
    __syncthreads();
    int lower = 0, before = 0, all = 0;
    if (e != 0xffff)
        for (int q = 0; q < pairs; ++q) {
            const int other = own.expert[q];
            lower += other < e;
            before += other == e && q < p;
            all += other == e;
        }
    const int tiles = e != 0xffff && before == 0 ? ceil_div(all, a.R) : 0;
    if (p < pairs) own.tiles_of[p] = (uint16_t)tiles;
    if (e != 0xffff) {
        own.order[lower + before] = (uint16_t)(p / a.plan.top_k);
        if (place_too) NM_ST(a.plan.place + p, lower + before, a.in_place, a.status);
    }
    __syncthreads();
    if (tiles > 0) {
        int at = 0;
        for (int q = 0; q < pairs; ++q) at += own.expert[q] < e ? own.tiles_of[q] : 0;
        for (int i = 0; i < tiles; ++i) own.tiles[at + i] = make_uint2((unsigned)e | (unsigned)min(a.R, all - i * a.R) << 16, (unsigned)(lower + i * a.R));
    }
    if (p < 32) {                                                 // a lane for each number of parts
        int total = 0;
        for (int q = lane; q < pairs; q += 32) total += own.tiles_of[q];
        total = __reduce_add_sync(0xffffffffu, total);
        const Schedule s = best_schedule(a.model, total, lane);
        if (lane == 0) own.schedule = s;
    }
    __syncthreads();
}

// One item: its rows and outputs.
struct Item { int expert, row0, rows, n0; };
template <int kMode>
__device__ __forceinline__ Item item_of(const StreamArgs &a, const OwnPlan &own, int item)
{
    const int tile = item / a.column_tiles, n0 = (item - tile * a.column_tiles) * a.tile_n;
    if constexpr (kMode != kOutAct) {
        if (a.plan.own_pairs) {
            const uint2 t = own.tiles[tile];
            return Item{(int)(t.x & 0xffffu), (int)t.y, (int)(t.x >> 16), n0};
        }
        const RowTile *at = a.plan.tiles + tile;
        const int4 t = NM_INSIDE(at, 16, a.in_tiles, a.status) ? __ldcg(reinterpret_cast<const int4 *>(at)) : make_int4(0, 0, 1, 0);
        return Item{t.x, t.y, t.z, n0};
    }
    const int row0 = tile * a.R;
    return Item{0, row0, min(a.R, a.rows - row0), n0};
}

// What the epilogue reads beside the sums of four rows: their residual (16 bits, as it lies) or their factors.  Asked for a group of rows early, and used
// (widened) only then; the residual is brought into L2 when a chunk begins.
template <int kSlabs> struct Side { uint32_t of[kSlabs][4]; };
__device__ __forceinline__ void prefetch_l2(const void *p) { asm volatile("prefetch.global.L2 [%0];" ::"l"(p)); }

// Four rows of one output of each slab: where they lie and what there is of them.  The pointers walk with the rows.  (Instructions are what the epilogue
// costs: 128 rows of 1536 x 24576 took 10 us of 30 at forty an output.)
template <int kMode, bool kGated, int kSlabs, bool kF16>
struct Rows {
    static constexpr bool kWide = kMode == kOutDown || (kMode == kOutHidden && kF16);          // fp32 outputs
    static constexpr int kOutSlabs = kGated ? 1 : kSlabs;
    const StreamArgs &a;
    int n;                                       // output of the first slab; the others 128 further each
    long out_step, side_pitch;                   // bytes
    char *out[4];
    const char *side;
    float bias[kSlabs];

    __device__ __forceinline__ Rows(const StreamArgs &args, const Item &t, int j, int step, int n_lane) : a(args), n(t.n0 + n_lane)
    {
        const long r = t.row0 + j, pitch = a.ldo * (kWide ? 4 : 2);
        out_step = step * pitch;
        out[0] = static_cast<char *>(a.out) + r * pitch + (long)n * (kWide ? 4 : 2);
#pragma unroll
        for (int i = 1; i < 4; ++i) out[i] = out[i - 1] + pitch;
        side_pitch = kMode == kOutAct ? a.ld_residual * 2 : 4;
        side = kMode == kOutAct ? reinterpret_cast<const char *>(a.residual) + (a.residual ? r * side_pitch + 2l * n : 0)
                                : reinterpret_cast<const char *>(a.row_scale) + (a.row_scale ? r * side_pitch : 0);
#pragma unroll
        for (int sl = 0; sl < kSlabs; ++sl) {
            const int at = kGated ? n : n + sl * kSlab;
            bias[sl] = kMode == kOutAct && a.bias && at < a.N ? widen16(NM_LD(a.bias + (kGated && sl ? a.N : 0) + at, a.in_bias, a.status), kF16) : 0.f;
        }
    }
    // of rows `ahead` further; count: the rows there are
    __device__ __forceinline__ void ask(Side<kSlabs> &s, int ahead, int count) const
    {
        constexpr int kSideSlabs = kMode == kOutDown ? 1 : kMode == kOutHidden ? 0 : kOutSlabs;
        if (kMode == kOutAct ? !a.residual : !a.row_scale) return;
#pragma unroll
        for (int sl = 0; sl < kSideSlabs; ++sl)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const char *p = side + (ahead + i) * side_pitch + 256 * sl;
                s.of[sl][i] = 0u;
                if (i >= count) continue;
                if (kMode == kOutAct && n + sl * kSlab < a.N) s.of[sl][i] = NM_LD(reinterpret_cast<const uint16_t *>(p), a.in_residual, a.status);
                if (kMode == kOutDown) s.of[sl][i] = NM_LD(reinterpret_cast<const uint32_t *>(p), a.in_scale, a.status);
            }
    }
    // z[sl][i]: the sum of row i for output n of slab sl.  kSide: residual or factors are there; kAll: four rows are.
    template <bool kSide, bool kAll>
    __device__ __forceinline__ void store(float (&z)[kSlabs][4], const Side<kSlabs> &s, int count) const
    {
#pragma unroll
        for (int sl = 0; sl < kOutSlabs; ++sl) {
            if (n + sl * kSlab >= a.N) continue;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (!kAll && i >= count) continue;
                float v = z[sl][i];
                if constexpr (kMode == kOutDown) {
                    if (kSide) v *= __uint_as_float(s.of[0][i]);
                    NM_ST(reinterpret_cast<float *>(out[i]) + sl * kSlab, v, a.in_out, a.status);
                } else if constexpr (kMode == kOutAct) {
                    if (kSide) v += widen16((uint16_t)s.of[sl][i], kF16);
                    NM_ST(reinterpret_cast<uint16_t *>(out[i]) + sl * kSlab, round16(v, kF16), a.in_out, a.status);
                } else if constexpr (kF16) {
                    NM_ST(reinterpret_cast<float *>(out[i]) + sl * kSlab, v, a.in_out, a.status);
                } else {
                    // The upper half of the word (8 bits) and what is left of it (16), rounded to 8: 2^-16 of the value.  (Cut off, not rounded, so that no finite
                    // value becomes an infinite term; an infinity or a NaN is the first term alone.)
                    const uint32_t hi = __float_as_uint(v) & 0xffff0000u;
                    const float rest = v - __uint_as_float(hi);
                    const bool finite = (hi & 0x7f800000u) != 0x7f800000u;
                    uint16_t *h = reinterpret_cast<uint16_t *>(out[i]) + sl * kSlab;
                    NM_ST(h, (uint16_t)((hi >> 16) | (v != v ? 0x40u : 0u)), a.in_out, a.status);
                    NM_ST(h + a.out_term, finite ? __bfloat16_as_ushort(__float2bfloat16_rn(rest)) : (uint16_t)0, a.in_out, a.status);
                }
            }
        }
    }
    __device__ __forceinline__ void put(float (&z)[kSlabs][4], const Side<kSlabs> &s, int count)
    {
        if constexpr (kMode != kOutDown) {
            if (kMode == kOutAct && a.bias)
#pragma unroll
                for (int sl = 0; sl < kSlabs; ++sl)
#pragma unroll
                    for (int i = 0; i < 4; ++i) z[sl][i] += bias[sl];
            activate(a.act, z[0]);
            if constexpr (!kGated && kSlabs > 1) activate(a.act, z[1]);
            if constexpr (kGated) {
#pragma unroll
                for (int i = 0; i < 4; ++i) z[0][i] *= z[1][i];
            }
        }
        const bool with = kMode != kOutHidden && (kMode == kOutAct ? a.residual != nullptr : a.row_scale != nullptr);
        if (count < 4) { if (with) store<true, false>(z, s, count); else store<false, false>(z, s, count); }
        else if (with) store<true, true>(z, s, 4);
        else store<false, true>(z, s, 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) out[i] += out_step;
    }
};

// What only one kind of product does: the first gathers rows, the second has two terms.
template <int kMode> constexpr bool kGathers = kMode == kOutHidden;
template <int kMode> constexpr int kTerms = kMode == kOutDown ? 2 : 1;
// How an item's token rows are copied: gathered (their tokens), or one box for each term; and the bytes of a step, weights and all.
template <bool kGather> struct TokenCopy { int ids[kGather ? kGathered : 1], boxes; uint32_t term_bytes, step_bytes; };
template <int kMode>
__device__ __forceinline__ TokenCopy<kGathers<kMode>> token_copy(const StreamArgs &a, const OwnPlan &own, const Item &t, int slabs)
{
    TokenCopy<kGathers<kMode>> x;
    x.boxes = ceil_div(t.rows, a.box_rows);
    x.term_bytes = (uint32_t)((a.apart ? x.boxes * a.box_rows : a.R) * 128);
    x.step_bytes = (uint32_t)slabs * kSlabBytes + (kGathers<kMode> && a.gather ? (uint32_t)ceil_div(t.rows, 4) * 512u : (uint32_t)(x.boxes * a.box_rows * kTerms<kMode>) * 128u);
    if (kGathers<kMode> && a.gather) {
#pragma unroll
        for (int i = 0; i < (kGathers<kMode> ? kGathered : 0); ++i) {
            const int *at = a.plan.order + t.row0 + i;
            x.ids[i] = i >= t.rows ? 0 : a.plan.own_pairs ? own.order[t.row0 + i] : NM_INSIDE(at, 4, a.in_order, a.status) ? __ldcg(at) : 0;
        }
    }
    return x;
}

// Sums of a chunk lie in groups of four rows, [group][slab][128 outputs][4 rows]: a thread moves 16 bytes at a time.  Adds up the `parts` chunks of an
// item from slot `first` on for the groups from rows j, j + step .. on, in the order of k; kAhead chunks are asked for at once.
template <int kSlabs, int kGroups, int kAhead>
__device__ __forceinline__ void join(const StreamArgs &a, int j, int step, int first, int parts, int n_lane, float (&z)[kGroups][kSlabs][4])
{
#pragma unroll
    for (int g = 0; g < kGroups; ++g)
#pragma unroll
        for (int sl = 0; sl < kSlabs; ++sl)
#pragma unroll
            for (int i = 0; i < 4; ++i) z[g][sl][i] = 0.f;
    const size_t piece = (size_t)a.R * (kSlabs * kSlab) / 4;
    const float4 *from = reinterpret_cast<const float4 *>(a.partial) + first * piece + (size_t)(j / 4) * (kSlabs * kSlab) + n_lane;
    const int further = step / 4 * (kSlabs * kSlab);
    for (int p0 = 0; p0 < parts; p0 += kAhead) {
        float4 v[kAhead][kGroups][kSlabs];
        // (the last chunk again where there are no more: a load under a condition would wait for the one before it)
#pragma unroll
        for (int q = 0; q < kAhead; ++q)
#pragma unroll
            for (int g = 0; g < kGroups; ++g)
#pragma unroll
                for (int sl = 0; sl < kSlabs; ++sl) {
                    const float4 *at = from + min(p0 + q, parts - 1) * piece + g * further + sl * kSlab;
                    v[q][g][sl] = NM_INSIDE(at, 16, a.in_partial, a.status) ? __ldcg(at) : make_float4(0.f, 0.f, 0.f, 0.f);
                }
#pragma unroll
        for (int q = 0; q < kAhead; ++q)
            if (p0 + q < parts)
#pragma unroll
                for (int g = 0; g < kGroups; ++g)
#pragma unroll
                    for (int sl = 0; sl < kSlabs; ++sl) {
                        z[g][sl][0] += v[q][g][sl].x; z[g][sl][1] += v[q][g][sl].y; z[g][sl][2] += v[q][g][sl].z; z[g][sl][3] += v[q][g][sl].w;
                    }
    }
}

template <int kMode, bool kGated, int kSlabs, bool kCol, bool kF16>
__global__ void __launch_bounds__(kMaxThreads, 1)
stream_kernel(const __grid_constant__ CUtensorMap map_w0, const __grid_constant__ CUtensorMap map_w1, const __grid_constant__ TokenMaps maps_x, const __grid_constant__ StreamArgs a)
{
    static_assert(!kGated || kSlabs == 2, "gate and up are a slab each");
    extern __shared__ unsigned char smem_raw[];
    const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
    __shared__ __align__(8) uint64_t s_bars[2 * kMaxStages + 2 * kQueue + 5];
    __shared__ uint32_t s_tmem;
    __shared__ int s_abort, s_queue[kQueue], s_next[2];
    __shared__ unsigned s_last;
    __shared__ typename std::conditional<kMode == kOutAct, char, OwnPlan>::type s_plan;
    const OwnPlan &own = reinterpret_cast<const OwnPlan &>(s_plan);
    const uint32_t full0 = smem_u32(s_bars), empty0 = full0 + 8 * kMaxStages, queued0 = empty0 + 8 * kMaxStages, taken0 = queued0 + 8 * kQueue,
                   acc_full0 = taken0 + 8 * kQueue, acc_empty0 = acc_full0 + 16, drained = acc_empty0 + 16;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int NS = a.nstage, finishers = (int)blockDim.x - 64;

    if (warp == 0) {
        if (lane == 0) { tma_prefetch_descriptor(&map_w0); if (kGated) tma_prefetch_descriptor(&map_w1); if (NM_MAP_MADE(&maps_x.of[a.first_map], a.status)) tma_prefetch_descriptor(&maps_x.of[a.first_map]); s_abort = 0; }
        if (lane < NS) { mbar_init(full0 + 8 * lane, 1); mbar_init(empty0 + 8 * lane, 1); }
        if (lane < kQueue) { mbar_init(queued0 + 8 * lane, 1); mbar_init(taken0 + 8 * lane, 2); }      // (taken by the MMA warp and the epilogue)
        if (lane < 2) { mbar_init(acc_full0 + 8 * lane, 1); mbar_init(acc_empty0 + 8 * lane, (uint32_t)finishers / 32); }
        if (lane == 2) mbar_init(drained, 1);
        mbar_init_fence();
        __syncwarp();
    }
    const int first_id = blockIdx.x;
    int head = 0;                                              // stages that are filled before the warps part
    const uint64_t stream = l2_policy_evict_first(), keep = l2_policy_evict_last();
    auto weights = [&](const Item &t, int k, int s) {
        const uint32_t dst = base + (uint32_t)s * a.stage_bytes, bar = full0 + 8 * s;
#pragma unroll
        for (int sl = 0; sl < kSlabs; ++sl) {
            const CUtensorMap *m = kGated && sl ? &map_w1 : &map_w0;
            const int n = t.n0 + (kGated ? 0 : sl * kSlab);
            if constexpr (kCol) {
                tma_load_3d(dst + sl * kSlabBytes, m, k * kKT, n, t.expert, bar, stream);
            } else {
                tma_load_3d(dst + sl * kSlabBytes, m, n, k * kKT, t.expert, bar, stream);
                tma_load_3d(dst + sl * kSlabBytes + kSlabBytes / 2, m, n + 64, k * kKT, t.expert, bar, stream);
            }
        }
    };
    auto tokens = [&](const Item &t, const TokenCopy<kGathers<kMode>> &x, int k, int s) {
        const uint32_t dst = base + (uint32_t)s * a.stage_bytes + kSlabs * kSlabBytes, bar = full0 + 8 * s;
        if constexpr (kGathers<kMode>) {
            if (a.gather) {
#pragma unroll
                for (int g = 0; g < kGathered / 4; ++g)
                    if (4 * g < t.rows) tma_gather4(dst + g * 512, &maps_x.of[0], k * kKT, x.ids[4 * g], x.ids[4 * g + 1], x.ids[4 * g + 2], x.ids[4 * g + 3], bar, keep);
                return;
            }
        }
        tma_load_3d(dst, &maps_x.of[x.boxes - 1], k * kKT, t.row0, 0, bar, keep);
        if constexpr (kTerms<kMode> == 2) tma_load_3d(dst + x.term_bytes, &maps_x.of[x.boxes - 1], k * kKT, t.row0, 1, bar, keep);
    };
    if (warp == 1) tmem_alloc(&s_tmem, a.tmem_columns);
    __syncthreads();                                           // (the barriers are there)
    // The plan of a programmatic chain (or the experts it is made of) is two kernels back and complete, as the kernel before waited for it: only what the kernel
    // before wrote has to be waited for.  Without early_weights everything is behind the wait.
    if (!a.early_weights) pdl_wait_prior_grids();
    pdl_launch_dependents();
    // The first fills are dealt out to all of the warps: a request costs the thread that makes it 100 clocks and more, so one thread took 2 us for a ring of twelve stages.
    Schedule sched = a.schedule;
    if constexpr (kMode != kOutAct) {
        if (a.plan.own_pairs) {
            make_plan(a, s_plan, kMode == kOutHidden && blockIdx.x == 0);
            sched = own.schedule;
        } else {
            const int4 v = __ldcg(reinterpret_cast<const int4 *>(a.plan.schedule));
            sched = Schedule{v.x, v.y, v.z, v.w};
        }
    }
    if (first_id < sched.chunks) {
        const Chunk c = chunk_of(sched, a.kb, first_id);
        head = min(NS, c.k1 - c.k0);
        if (lane == 0 && warp < head) {
            const int warps = (int)blockDim.x / 32;
            const Item t = item_of<kMode>(a, own, c.item);
            const auto x = token_copy<kMode>(a, own, t, kSlabs);
            for (int i = warp; i < head; i += warps) {
                mbar_arrive_expect_tx(full0 + 8 * i, x.step_bytes);
                weights(t, c.k0 + i, i);
                if (!a.early_weights) tokens(t, x, c.k0 + i, i);
            }
            if (a.early_weights) {
                pdl_wait_prior_grids();
                for (int i = warp; i < head; i += warps) tokens(t, x, c.k0 + i, i);
            }
        }
    }
    int filled = head;                                         // (where a wait runs out, the copies begun are known by it: lane 0 of warp 0)
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = s_tmem;
    const bool more_than_one = sched.chunks > (int)gridDim.x;

    if (warp == 0) {
        if (lane == 0) {
            int s = 0, n = 0, queue = 0;
            uint32_t ph = 1, queue_ph = 1;                      // a fresh barrier passes a wait for the phase before its first
            bool ok = true;
            // The next chunk is asked for eight steps before this one's last copy, and its item read three steps before: in time for neither to be waited for
            // (a ticket takes 1 to 2 us), and late enough that whoever is done first takes what is left.
            Item t{}, t_next{};
            unsigned ticket = 0u;
            if (first_id < sched.chunks) t = item_of<kMode>(a, own, chunk_of(sched, a.kb, first_id).item);
            for (int id = first_id; ok && id < sched.chunks;) {
                const Chunk c = chunk_of(sched, a.kb, id);
                const auto x = token_copy<kMode>(a, own, t, kSlabs);
                const int ask_at = max(c.k0, c.k1 - 8), read_at = max(c.k0, c.k1 - 3);
                id = sched.chunks;
                for (int k = c.k0; k < c.k1; ++k, ++n) {
                    if (more_than_one) {
                        if (k == ask_at) ticket = ask_ticket(a.counters + a.ticket);
                        if (k == read_at) {
                            id = (int)min(gridDim.x + ticket, (unsigned)sched.chunks);
                            if (id < sched.chunks) t_next = item_of<kMode>(a, own, chunk_of(sched, a.kb, id).item);
                        }
                    }
                    if (n >= head) {
                        NM_PAUSE(1);                              // before a copy
                        ok = mbar_try_wait(empty0 + 8 * s, ph) || mbar_wait(empty0 + 8 * s, ph, &s_abort, a.status);
                        if (!ok) break;
                        mbar_arrive_expect_tx(full0 + 8 * s, x.step_bytes);
                        weights(t, k, s);
                        tokens(t, x, k, s);
                        filled = n + 1;
                    }
                    if (++s == NS) { s = 0; ph ^= 1; }
                }
                t = t_next;
                NM_PAUSE(2);                                      // before the next chunk is passed on
                if (ok && more_than_one) {
                    ok = mbar_try_wait(taken0 + 8 * queue, queue_ph) || mbar_wait(taken0 + 8 * queue, queue_ph, &s_abort, a.status);
                    if (ok) { s_queue[queue] = id; mbar_arrive(queued0 + 8 * queue); }
                    if (++queue == kQueue) { queue = 0; queue_ph ^= 1; }
                }
            }
            // Every CTA has had its last ticket (the value is looked at, so it has come): whoever is last to say so clears them.  Every product leaves the counters
            // at zero, whoever made its plan: what uses the workspace next may be any call that has counters there.
            if (more_than_one && ticket != 0xffffffffu && atomicAdd(a.counters + kDone, 1u) == gridDim.x - 1) {
                a.counters[a.ticket] = 0u;
                a.counters[kDone] = 0u;
            }
        }
    } else if (warp == 1) {
        // The whole warp walks, one elected lane issues: descriptors are then uniform values.
        const bool leader = elect_one();
        int s = 0, acc = 0, queue = 0;
        uint32_t ph = 0, acc_ph = 1, queue_ph = 0;
        bool ok = true;
        for (int id = first_id; id < sched.chunks;) {
            const Chunk c = chunk_of(sched, a.kb, id);
            const Item t = item_of<kMode>(a, own, c.item);
            const int columns = kTerms<kMode> == 2 && a.apart ? 2 * ceil_div(t.rows, a.box_rows) * a.box_rows : (t.rows + 15) & ~15;
            const uint32_t idesc = kF16 ? instr_desc_f16(kSlab, columns, !kCol, false) : instr_desc(kSlab, columns, !kCol, false);
            const bool twice = kTerms<kMode> == 2 && !a.apart;
            ok = mbar_try_wait(acc_empty0 + 8 * acc, acc_ph) || mbar_wait(acc_empty0 + 8 * acc, acc_ph, &s_abort, a.status);
            if (!__all_sync(0xffffffffu, ok)) break;
            tc_fence_after();
            const uint32_t d = tmem + (uint32_t)acc * kSlabs * a.acc_columns;
            NM_PAUSE(3);                                          // before a chunk's products
            for (int k = c.k0; k < c.k1; ++k) {
                ok = mbar_try_wait(full0 + 8 * s, ph) || mbar_wait(full0 + 8 * s, ph, &s_abort, a.status);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                tc_fence_after();
                const uint32_t sw = base + (uint32_t)s * a.stage_bytes, sx = sw + kSlabs * kSlabBytes;
                // descriptors count 16 bytes: 16 k further are 32 bytes of a row of k, 2048 of rows of outputs
                const uint64_t w0 = kCol ? smem_desc(sw, 16, 1024) : smem_desc(sw, kSlabBytes / 2, 1024), x0 = smem_desc(sx, 16, 1024);
                if (leader) {
#pragma unroll
                    for (int kk = 0; kk < kKT / 16; ++kk)
#pragma unroll
                        for (int sl = 0; sl < kSlabs; ++sl) {
                            const uint64_t wd = w0 + kk * (kCol ? 2 : 128) + sl * (kSlabBytes >> 4);
                            mma_ss(d + sl * a.acc_columns, wd, x0 + kk * 2, idesc, k != c.k0 || kk != 0);
                            if (twice) mma_ss(d + sl * a.acc_columns, wd, x0 + kk * 2 + a.R * 8, idesc, true);
                        }
                    mma_commit(empty0 + 8 * s);
                }
                if (++s == NS) { s = 0; ph ^= 1; }
            }
            if (!ok) break;
            if (leader) mma_commit(acc_full0 + 8 * acc);
            if (acc) acc_ph ^= 1;
            acc ^= 1;
            id = sched.chunks;
            if (more_than_one) {
                ok = mbar_try_wait(queued0 + 8 * queue, queue_ph) || mbar_wait(queued0 + 8 * queue, queue_ph, &s_abort, a.status);
                if (!__all_sync(0xffffffffu, ok)) break;
                id = *static_cast<volatile int *>(s_queue + queue);
                __syncwarp();
                if (lane == 0) mbar_arrive(taken0 + 8 * queue);
                if (++queue == kQueue) { queue = 0; queue_ph ^= 1; }
            }
        }
    } else {
        const int quad = warp & 3, turn = (warp - 2) >> 2, step = finishers / 32, n_lane = quad * 32 + lane, thread = tid - 64;
        if (a.early_weights) pdl_wait_prior_grids();            // nothing is written, and nothing of earlier kernels read, before they are done
        int acc = 0, queue = 0, round = 0;
        uint32_t ph = 0, queue_ph = 0;
        for (int id = first_id; id < sched.chunks; round ^= 1) {
            const Chunk c = chunk_of(sched, a.kb, id);
            const Item t = item_of<kMode>(a, own, c.item);
            Rows<kMode, kGated, kSlabs, kF16> rows(a, t, 4 * turn, step, n_lane);
            if (kMode == kOutAct && a.residual) {
                // (a lane a row: this warp's rows are four of every `step`)
                const int r = 4 * turn + (lane >> 2) * step + (lane & 3), n_warp = t.n0 + quad * 32;
#pragma unroll
                for (int sl = 0; sl < (kGated ? 1 : kSlabs); ++sl)
                    if (r < t.rows && n_warp + sl * kSlab < a.N) prefetch_l2(a.residual + (t.row0 + r) * a.ld_residual + n_warp + sl * kSlab);
            }
            Side<kSlabs> side;
            rows.ask(side, 0, t.rows - 4 * turn);
            mbar_wait(acc_full0 + 8 * acc, ph, &s_abort, a.status);   // (where it ran out the walk goes on, over values that the status disowns: the
                                                                    // barriers below are for all of the warps)
            tc_fence_after();
            const uint32_t d = tmem + ((uint32_t)(quad * 32) << 16) + (uint32_t)acc * kSlabs * a.acc_columns;
            const int second = ceil_div(t.rows, a.box_rows) * a.box_rows;     // (where the terms are apart: the other one's first column)
            float4 *mine = reinterpret_cast<float4 *>(a.partial) + (size_t)c.slot * a.R * (kSlabs * kSlab / 4);
            for (int j = 4 * turn; j < t.rows; j += step) {
                uint32_t bits[kSlabs][4];
                float z[kSlabs][4];
#pragma unroll
                for (int sl = 0; sl < kSlabs; ++sl) tmem_ld4(d + sl * a.acc_columns + j, bits[sl]);
                tmem_wait_ld();
#pragma unroll
                for (int sl = 0; sl < kSlabs; ++sl)
#pragma unroll
                    for (int i = 0; i < 4; ++i) z[sl][i] = __uint_as_float(bits[sl][i]);
                if (kMode == kOutDown && a.apart) {
#pragma unroll
                    for (int sl = 0; sl < kSlabs; ++sl) tmem_ld4(d + sl * a.acc_columns + second + j, bits[sl]);
                    tmem_wait_ld();
#pragma unroll
                    for (int sl = 0; sl < kSlabs; ++sl)
#pragma unroll
                        for (int i = 0; i < 4; ++i) z[sl][i] += __uint_as_float(bits[sl][i]);
                }
                if (c.cut < 0) {
                    const Side<kSlabs> now = side;
                    rows.ask(side, j - 4 * turn + step, t.rows - j - step);
                    rows.put(z, now, t.rows - j);
                } else {
#pragma unroll
                    for (int sl = 0; sl < kSlabs; ++sl)
                        NM_ST(mine + (j / 4 * kSlabs + sl) * kSlab + n_lane, make_float4(z[sl][0], z[sl][1], z[sl][2], z[sl][3]), a.in_partial, a.status);
                }
            }
            NM_PAUSE(4);                                          // before an accumulator is given back
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(acc_empty0 + 8 * acc);
            if (acc) ph ^= 1;
            acc ^= 1;

            if (c.cut >= 0) {
                if (turn == 0) NM_PAUSE(5);                       // (half of the warps) before an item's chunks are counted
                named_barrier_sync(1, finishers);
                if (thread == 0) {
                    __threadfence();                             // (all of the CTA's sums: the barrier comes first)
                    s_last = atomicAdd(a.counters + kItemCounters + c.cut, 1u) == (unsigned)(sched.parts - 1);
                    if (s_last) a.counters[kItemCounters + c.cut] = 0u;             // ready for the next product
                }
                named_barrier_sync(1, finishers);
                if (s_last) {
                    __threadfence();
                    auto put_next = [&](float (&z)[kSlabs][4], int j) {
                        const Side<kSlabs> now = side;
                        rows.ask(side, j - 4 * turn + step, t.rows - j - step);
                        rows.put(z, now, t.rows - j);
                    };
                    int j = 4 * turn;
                    for (; j + step < t.rows; j += 2 * step) {
                        float z[2][kSlabs][4];
                        // (items of the experts' products are cut into few parts; asking for more of them cost 67 tokens through 3 of 24 experts 4 us of 72)
                        join<kSlabs, 2, (kMode == kOutAct ? 8 : 4) / kSlabs>(a, j, step, c.first_slot, sched.parts, n_lane, z);
                        put_next(z[0], j);
                        put_next(z[1], j + step);
                    }
                    if (j < t.rows) {
                        float z[1][kSlabs][4];
                        join<kSlabs, 1, 8 / kSlabs>(a, j, step, c.first_slot, sched.parts, n_lane, z);
                        put_next(z[0], j);
                    }
                }
            }
            if (!more_than_one) break;
            // One thread takes the next chunk for all, so that they agree where a wait runs out.
            if (turn == 0 && quad == 1) NM_PAUSE(6);              // (a warp) before the next chunk is taken
            if (thread == 0) {
                const bool ok = mbar_wait(queued0 + 8 * queue, queue_ph, &s_abort, a.status);
                s_next[round] = ok ? *static_cast<volatile int *>(s_queue + queue) : sched.chunks;
                mbar_arrive(taken0 + 8 * queue);
            }
            if (++queue == kQueue) { queue = 0; queue_ph ^= 1; }
            named_barrier_sync(1, finishers);
            id = *static_cast<volatile int *>(s_next + round);
        }
    }

    tc_fence_before();
    __syncthreads();
    if (s_abort) {
        // A wait ran out: the copies begun are waited for, each stage at the phase of its last fill, before shared memory is given back, and the
        // products issued before tensor memory is.
        if (warp == 0 && lane == 0)
            for (int i = 0; i < NS && i < filled; ++i) {
                const int fills = (filled - 1 - i) / NS + 1;
                for (int j = 0; j < (1 << 14) && !mbar_try_wait(full0 + 8 * i, (fills - 1) & 1); ++j) {}
            }
        if (warp == 1) {
            if (elect_one()) mma_commit(drained);              // (the lane that issued: the same one is elected every time)
            for (int j = 0; j < (1 << 14) && !mbar_try_wait(drained, 0); ++j) {}
        }
        __syncthreads();
    }
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem, a.tmem_columns);
    }
}

bool encode_map(CUtensorMap *map, const void *p, bool f16, int rank, const cuuint64_t *dims, const cuuint64_t *strides, const cuuint32_t *box)
{
    EncodeTiledFn enc = tensor_map_encoder();
    if (!enc) return false;
    const cuuint32_t ones[3] = {1, 1, 1};
    return enc(map, f16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, rank, const_cast<void *>(p), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int kMode, bool kGated, int kSlabs, bool kCol, bool kF16>
cudaError_t launch_stream(const CUtensorMap &w0, const CUtensorMap &w1, const TokenMaps &x, const StreamArgs &a, long ctas, cudaStream_t s)
{
    static std::atomic<unsigned long long> configured{0};
    auto kern = stream_kernel<kMode, kGated, kSlabs, kCol, kF16>;
    cudaError_t e = ensure_dynamic_smem(kern, kRingBytes + 1024, configured);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ctas);
    cfg.blockDim = dim3(a.few ? kMaxThreads - 128 : kMaxThreads);
    cfg.dynamicSmemBytes = (size_t)a.nstage * a.stage_bytes + 1024;
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = a.programmatic ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kern, w0, w1, x, a);
}

}  // namespace

int stream_tile_rows(double average, int most)
{
    for (int R = 16; R < 128; R *= 2)
        if (R >= most || R >= 2 * average + 8) return R;
    return 128;
}

// Two slabs halve how often the token rows are read (and the MMAs that share them come in pairs); of a narrow matrix too much of the last tile would be empty.
int stream_slabs(int N, bool gated) { return gated || N >= 2048 ? 2 : 1; }

// Sums of chunks: as many as 64 MB hold, no more than 1024, and no more than the items of the last rounds have steps.
static size_t sum_bytes(int R, int N, bool gated) { return (size_t)R * stream_slabs(N, gated) * kSlab * sizeof(float); }
static int most_chunks(int R, int N, int K, bool gated, long row_tiles)
{
    const long tile_n = gated ? kSlab : stream_slabs(N, gated) * kSlab, items = std::min<long>(2 * kSMs, row_tiles * ((N + tile_n - 1) / tile_n));
    return (int)std::min<long>(std::min<long>(1024, items * ceil_div(K, kKT)), ((long)64 << 20) / (long)sum_bytes(R, N, gated));
}
size_t stream_partial_bytes(int R, int N, int K, bool gated, long row_tiles) { return (size_t)most_chunks(R, N, K, gated, row_tiles) * sum_bytes(R, N, gated); }

CutModel stream_cut_model(int R, float rows, int N, int K, bool gated, int terms, long row_tiles)
{
    const int slabs = stream_slabs(N, gated);
    const float step_bytes = slabs * kSlabBytes + terms * rows * 128;
    CutModel m;
    m.kb = ceil_div(K, kKT);
    m.column_tiles = ceil_div(N, gated ? kSlab : slabs * kSlab);
    m.most_chunks = most_chunks(R, N, K, gated, row_tiles);
    m.alone_us = std::max(0.245f, step_bytes / 96e3f);
    m.busy_us = std::max(m.alone_us, kSMs * (float)(slabs * kSlabBytes) / 6.9e6f);
    m.sums_us = std::max(4.f, rows) * slabs * kSlab * 4 / 35e3f;
    m.chunk_us = 8.f + 0.1f * rows * slabs;
    m.forced = g_forced_parts.load(std::memory_order_relaxed);
    return m;
}

cudaError_t launch_product(int mode, bool gated, const ProductArgs &p, cudaStream_t s, const char **what)
{
    StreamArgs a{};
    const int slabs = stream_slabs(p.N, gated);
    const CutModel m = stream_cut_model(p.R, p.expected_rows, p.N, p.K, gated, p.terms, p.row_tiles);
    a.kb = m.kb;
    a.tile_n = gated ? kSlab : slabs * kSlab;
    a.column_tiles = m.column_tiles;
    a.box_rows = std::max(8, p.R / 4);
    a.rows = p.rows; a.N = p.N; a.R = p.R;
    if (!p.planned) {
        const int items = ceil_div(p.rows, p.R) * a.column_tiles, rest = items - whole_items(items);
        // (one number of parts for each length that a chunk can have)
        const int most = std::min(std::min(a.kb, kSMs), m.most_chunks / rest);
        int best = 1;
        float least = cut_cost(m, rest, 1);
        for (int parts = 2; parts <= most;) {
            const float cost = cut_cost(m, rest, parts);
            if (cost < least) { least = cost; best = parts; }
            const int kc = ceil_div(a.kb, parts);
            parts = kc > 1 ? std::max(parts + 1, ceil_div(a.kb, kc - 1)) : most + 1;
        }
        a.schedule = schedule_of(items, a.kb, best);
    }
    a.stage_bytes = slabs * kSlabBytes + p.terms * p.R * 128;
    a.nstage = std::min(kMaxStages, kRingBytes / a.stage_bytes);
    a.apart = p.terms == 2 && p.R <= 64;
    a.few = p.expected_rows <= 4.f;
    a.acc_columns = a.apart ? 2 * p.R : p.R;
    a.tmem_columns = std::max(32, 2 * slabs * a.acc_columns);
    a.gather = p.gather; a.early_weights = p.early_weights; a.programmatic = p.programmatic;
    a.act = p.act; a.plan = p.plan; a.model = m;
    a.bias = static_cast<const uint16_t *>(p.bias); a.residual = static_cast<const uint16_t *>(p.residual); a.ld_residual = p.ld_residual;
    a.out = p.out; a.ldo = p.ldo; a.out_term = (long)p.rows * p.ldo; a.row_scale = p.row_scale;
    a.partial = p.partial; a.counters = p.counters; a.ticket = p.ticket;
    const int parts = gated ? 2 : 1;
    a.in_bias = make_span(p.bias, p.bias ? 2 * (size_t)parts * p.N : 0);
    a.in_residual = make_span(p.residual, p.residual ? 2 * ((size_t)(p.rows - 1) * p.ld_residual + p.N) : 0);
    a.in_out = make_span(p.out, mode == kOutAct ? 2 * ((size_t)(p.rows - 1) * p.ldo + p.N) : 4 * (size_t)p.rows * p.ldo);
    a.in_scale = make_span(p.row_scale, p.row_scale ? 4 * (size_t)p.rows : 0);
    a.in_partial = make_span(p.partial, stream_partial_bytes(p.R, p.N, p.K, gated, p.row_tiles));
    a.in_tiles = make_span(p.plan.tiles, sizeof(RowTile) * ((size_t)p.E + p.rows / p.R));
    a.in_order = make_span(p.plan.order, 4 * (size_t)p.rows);
    a.in_experts = make_span(p.plan.experts, 4 * (size_t)p.plan.own_pairs); a.in_place = make_span(p.plan.place, 4 * (size_t)p.plan.own_pairs);
    a.status = device_status_ptr();
    const unsigned long long pause = g_pause.load(std::memory_order_relaxed);
    a.pause_ns = (unsigned)pause; a.pause_where = (int)(pause >> 32);

    CUtensorMap w[2];
    TokenMaps x{};                              // (heights that there cannot be stay zero)
    const uint16_t *W = static_cast<const uint16_t *>(p.W);
    bool ok = true;
    auto weight_map = [&](CUtensorMap *map, const uint16_t *W, long expert, int N, int K, int wide) {
        if (p.col) {
            const cuuint64_t dims[3] = {(cuuint64_t)K, (cuuint64_t)N, (cuuint64_t)p.E}, strides[2] = {(cuuint64_t)K * 2, (cuuint64_t)expert * 2};
            const cuuint32_t box[3] = {kKT, kSlab, 1};
            return encode_map(map, W, p.f16, 3, dims, strides, box);
        }
        const cuuint64_t dims[3] = {(cuuint64_t)N, (cuuint64_t)K, (cuuint64_t)p.E}, strides[2] = {(cuuint64_t)wide * 2, (cuuint64_t)expert * 2};
        const cuuint32_t box[3] = {64, kKT, 1};
        return encode_map(map, W, p.f16, 3, dims, strides, box);
    };
    for (int part = 0; part < parts; ++part) ok = ok && weight_map(&w[part], W + (size_t)part * p.N * (p.col ? p.K : 1), p.w_expert, p.N, p.K, parts * p.N);
    if (!gated) w[1] = w[0];
    if (p.gather) {
        const cuuint64_t dims[2] = {(cuuint64_t)p.K, (cuuint64_t)p.x_rows}, strides[1] = {(cuuint64_t)p.ldx * 2};
        const cuuint32_t box[2] = {kKT, 1};
        ok = ok && encode_map(&x.of[0], p.x, p.f16, 2, dims, strides, box);
    } else {
        const cuuint64_t dims[3] = {(cuuint64_t)p.K, (cuuint64_t)p.x_rows, (cuuint64_t)p.terms}, strides[2] = {(cuuint64_t)p.ldx * 2, (cuuint64_t)p.x_term * 2};
        // (only the heights that there can be: of a full tile and of the last one, where the rows are known)
        const int whole_box = p.R / a.box_rows - 1, last_box = p.planned ? 0 : (p.rows - 1) % p.R / a.box_rows;
        a.first_map = p.planned ? 0 : p.rows < p.R ? last_box : whole_box;
        for (int i = 0; i <= whole_box; ++i) {
            if (!p.planned && i != last_box && (i != whole_box || p.rows < p.R)) continue;
            const cuuint32_t box[3] = {kKT, (cuuint32_t)((i + 1) * a.box_rows), 1};
            ok = ok && encode_map(&x.of[i], p.x, p.f16, 3, dims, strides, box);
        }
    }
    if (!ok) { *what = "cuTensorMapEncodeTiled"; return cudaErrorInvalidValue; }
    if (!a.status) { *what = "device status word"; return cudaErrorInvalidValue; }
    *what = "streamed product launch";
    const long ctas = p.planned ? kSMs : std::min(kSMs, a.schedule.chunks);
    auto launch = [&](auto mode_, auto gated_, auto slabs_) {
        constexpr int kM = decltype(mode_)::value, kS = decltype(slabs_)::value;
        constexpr bool kG = decltype(gated_)::value;
        if (p.f16) return p.col ? launch_stream<kM, kG, kS, true, true>(w[0], w[1], x, a, ctas, s) : launch_stream<kM, kG, kS, false, true>(w[0], w[1], x, a, ctas, s);
        return p.col ? launch_stream<kM, kG, kS, true, false>(w[0], w[1], x, a, ctas, s) : launch_stream<kM, kG, kS, false, false>(w[0], w[1], x, a, ctas, s);
    };
    auto of_mode = [&](auto mode_) {
        if constexpr (decltype(mode_)::value != kOutDown)
            if (gated) return launch(mode_, std::true_type{}, std::integral_constant<int, 2>{});
        return slabs == 2 ? launch(mode_, std::false_type{}, std::integral_constant<int, 2>{}) : launch(mode_, std::false_type{}, std::integral_constant<int, 1>{});
    };
    switch (mode) {
    case kOutAct: return of_mode(std::integral_constant<int, kOutAct>{});
    case kOutHidden: return of_mode(std::integral_constant<int, kOutHidden>{});
    default: return of_mode(std::integral_constant<int, kOutDown>{});
    }
}

}  // namespace nm

extern "C" {
#pragma GCC visibility push(default)

int nm_debug_set_ffn_pause(int where, unsigned ns)
{
#ifdef NM_BOUNDS_CHECK
    if (where < 0 || where > nm::kPausePlaces || ns > 2000000000u) return NM_ERR_INVALID_ARG;
    nm::g_pause.store(((unsigned long long)where << 32) | ns, std::memory_order_relaxed);
    return NM_OK;
#else
    (void)where; (void)ns;
    return NM_ERR_UNSUPPORTED;
#endif
}

int nm_debug_set_ffn_cut(int parts)
{
    if (parts < 0) return NM_ERR_INVALID_ARG;
    nm::g_forced_parts.store(parts, std::memory_order_relaxed);
    return NM_OK;
}

#pragma GCC visibility pop
}  // extern "C"
