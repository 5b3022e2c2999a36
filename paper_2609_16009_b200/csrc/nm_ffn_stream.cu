// The products of the feed-forward operators on the tensor cores: weights streamed once from HBM past the rows of their expert.
//
//     D[128 outputs x rows] += W[128 outputs x 64 k] * X[rows x 64 k]^T         (the operands swapped: weights are the MMA's M dimension)
//
// Bound by the bytes of the weights while an expert has fewer than ~200 rows, so the kernel is a stream: one CTA per SM, a ring of 64-k stages
// filled by TMA, and an even share of ALL 64-k steps for every CTA, whatever experts and outputs they belong to.
//
//   item   one row tile (up to R rows of one expert) x one column tile (kSlabs slabs of 128 outputs; where gated, one slab each of gate and up,
//          so that a thread ends up with both values of an output), kb steps of 64 k
//   share  steps [c U / C, (c + 1) U / C) of the U = items * kb steps go to CTA c of C.  An item that is cut is finished by whoever of its CTAs
//          arrives last (a counter; nobody waits): every CTA leaves its fp32 sums in the workspace, the last adds them in the order of k.
//          So sums do not depend on who came last, and equal calls give equal bits.
//   warps  0: copies (all lanes: up to 32 row groups a step); 1: MMAs; 2-5: the epilogue, from the other one of two accumulators
//
// Token rows are copied as they lie in groups of eight, or gathered by token four at a time (tile::gather4) where the rows of an expert are
// scattered.  The number of accumulator columns is that of the rows there are, rounded up to 16; what the columns beyond hold is not read.
// A hidden value is the sum of two 16-bit terms (bf16: 16 bits and more, fp16: 22), both multiplied into the same accumulator: the MMAs are far
// from being the bound, and the second term keeps the rounding of the hidden values out of the result.
#include <algorithm>

#include "nm_ffn.cuh"
#include "nm_tcgen05.cuh"

namespace nm {

namespace {

constexpr int kThreads = 192;
constexpr int kKT = 64;                        // k of a stage
constexpr int kSlab = 128;                     // outputs of a slab (the MMA's M)
constexpr int kSlabBytes = kSlab * kKT * 2;
constexpr int kMaxStages = 12;
constexpr int kRingBytes = 216 * 1024;

struct StreamArgs {
    long units, items;                          // where the plan is on the host
    int kb, column_tiles, tile_n;               // steps of an item, column tiles of a row tile, outputs of one
    int n_second;                               // where the second slab's rows (columns) start within its map: +128, or +0 in a map of its own
    int rows, N, R, terms, nstage, stage_bytes;
    unsigned tmem_columns;
    bool col, f16, gather, planned, early_weights, programmatic;
    int act;
    RowPlan plan;
    const uint16_t *bias, *residual; long ld_residual;
    void *out; long ldo; long out_term;
    const float *row_scale;
    float *partial; unsigned *counters;
    Span in_bias, in_residual, in_out, in_scale, in_partial, in_tiles, in_order;
    unsigned *status;
};

__device__ __forceinline__ bool elect_one()
{
    unsigned r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r != 0;
}

// Four rows of a 2-D tensor, 64 k each, to consecutive 128-byte rows of shared memory.
__device__ __forceinline__ void tma_gather4(uint32_t dst, const CUtensorMap *map, int x, const int (&row)[4], uint32_t bar, uint64_t policy)
{
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cta.global.tile::gather4.mbarrier::complete_tx::bytes.L2::cache_hint"
        " [%0], [%1, {%2, %3, %4, %5, %6}], [%7], %8;"
        ::"r"(dst), "l"(map), "r"(x), "r"(row[0]), "r"(row[1]), "r"(row[2]), "r"(row[3]), "r"(bar), "l"(policy) : "memory");
}

// A CTA's share of the steps, item by item.
struct Walk {
    long unit, end;
    int kb;
    long item; int k0, k1;
    __device__ bool next()
    {
        if (unit >= end) return false;
        item = unit / kb;
        k0 = (int)(unit - item * kb);
        k1 = (int)min((long)kb, k0 + (end - unit));
        unit += k1 - k0;
        return true;
    }
};

// One item: its rows and outputs.
struct Item { int expert, row0, rows, n0; };
__device__ __forceinline__ Item item_of(const StreamArgs &a, long item)
{
    const int tile = (int)(item / a.column_tiles), n0 = (int)(item % a.column_tiles) * a.tile_n;
    if (a.planned) {
        const RowTile t = NM_LD(a.plan.tiles + tile, a.in_tiles, a.status);
        return Item{t.expert, t.row0, t.rows, n0};
    }
    const int row0 = tile * a.R;
    return Item{0, row0, min(a.R, a.rows - row0), n0};
}

// What becomes of finished outputs: z[i] is output n of row r + i, i < count; z2 the same of the up part.
template <int kMode, bool kGated, int kW>
__device__ __forceinline__ void finish(const StreamArgs &a, int r, int count, int n, const float (&z)[kW], const float (&z2)[kW])
{
    if (n >= a.N) return;
    if constexpr (kMode == kOutAct) {
        const float b0 = a.bias ? widen16(NM_LD(a.bias + n, a.in_bias, a.status), a.f16) : 0.f;
        const float b1 = kGated && a.bias ? widen16(NM_LD(a.bias + a.N + n, a.in_bias, a.status), a.f16) : 0.f;
        // All of the residual before the first store: it may be the output itself, so no load would be moved ahead of a store.
        float more[kW];
#pragma unroll
        for (int i = 0; i < kW; ++i)
            more[i] = a.residual && i < count ? widen16(NM_LD(a.residual + (long)(r + i) * a.ld_residual + n, a.in_residual, a.status), a.f16) : 0.f;
#pragma unroll
        for (int i = 0; i < kW; ++i) {
            if (i < count) {
                float v = activate(a.act, a.bias ? z[i] + b0 : z[i]);
                if constexpr (kGated) v *= a.bias ? z2[i] + b1 : z2[i];
                if (a.residual) v += more[i];
                NM_ST(static_cast<uint16_t *>(a.out) + (long)(r + i) * a.ldo + n, round16(v, a.f16), a.in_out, a.status);
            }
        }
    } else if constexpr (kMode == kOutHidden) {
#pragma unroll
        for (int i = 0; i < kW; ++i) {
            if (i < count) {
                float v = activate(a.act, z[i]);
                if constexpr (kGated) v *= z2[i];
                if (a.f16) {
                    NM_ST(static_cast<float *>(a.out) + (long)(r + i) * a.ldo + n, v, a.in_out, a.status);
                } else {
                    // The upper half of the word and what is left of it, rounded: 2^-17 of the value.  (Cut off, not rounded, so that no finite
                    // value becomes an infinite term; an infinity or a NaN is the first term alone.)
                    const uint32_t hi = __float_as_uint(v) & 0xffff0000u;
                    const float rest = v - __uint_as_float(hi);
                    const bool finite = (hi & 0x7f800000u) != 0x7f800000u;
                    uint16_t *h = static_cast<uint16_t *>(a.out) + (long)(r + i) * a.ldo + n;
                    NM_ST(h, (uint16_t)((hi >> 16) | (v != v ? 0x40u : 0u)), a.in_out, a.status);
                    NM_ST(h + a.out_term, finite ? __bfloat16_as_ushort(__float2bfloat16_rn(rest)) : (uint16_t)0, a.in_out, a.status);
                }
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < kW; ++i) {
            if (i < count) {
                const float s = a.row_scale ? NM_LD(a.row_scale + r + i, a.in_scale, a.status) : 1.f;
                NM_ST(static_cast<float *>(a.out) + (long)(r + i) * a.ldo + n, z[i] * s, a.in_out, a.status);
            }
        }
    }
}

// Partial sums lie in groups of four rows, [group][slab][128 outputs][4 rows]: a thread moves 16 bytes at a time.  Adds up the pieces of an item
// (CTAs first .. last) for kGroups groups from row j on, in the order of k, and finishes them; kAhead pieces are asked for at once.
template <int kMode, bool kGated, int kSlabs, int kGroups, int kAhead>
__device__ __forceinline__ void join(const StreamArgs &a, const Item &t, int j, int first, int last, int n_lane)
{
    float z[kSlabs][4 * kGroups];
#pragma unroll
    for (int sl = 0; sl < kSlabs; ++sl)
#pragma unroll
        for (int i = 0; i < 4 * kGroups; ++i) z[sl][i] = 0.f;
    const size_t piece = (size_t)a.R * (kSlabs * kSlab) / 4;
    for (int p0 = first; p0 <= last; p0 += kAhead) {
        float4 v[kAhead][kGroups][kSlabs];
#pragma unroll
        for (int q = 0; q < kAhead; ++q) {
            const int p = p0 + q;
            const float4 *from = reinterpret_cast<const float4 *>(a.partial) + (size_t)(2 * p + (p == first ? 1 : 0)) * piece + (size_t)(j / 4) * (kSlabs * kSlab) + n_lane;
#pragma unroll
            for (int g = 0; g < kGroups; ++g)
#pragma unroll
                for (int sl = 0; sl < kSlabs; ++sl) {
                    const bool there = p <= last && j + 4 * g < t.rows;
                    const float4 *at = from + (g * kSlabs + sl) * kSlab;
                    v[q][g][sl] = there && NM_INSIDE(at, 16, a.in_partial, a.status) ? __ldcg(at) : make_float4(0.f, 0.f, 0.f, 0.f);
                }
        }
#pragma unroll
        for (int q = 0; q < kAhead; ++q)
#pragma unroll
            for (int g = 0; g < kGroups; ++g)
#pragma unroll
                for (int sl = 0; sl < kSlabs; ++sl) {
                    z[sl][4 * g] += v[q][g][sl].x; z[sl][4 * g + 1] += v[q][g][sl].y; z[sl][4 * g + 2] += v[q][g][sl].z; z[sl][4 * g + 3] += v[q][g][sl].w;
                }
    }
    const int count = min(4 * kGroups, t.rows - j);
    if constexpr (kGated) {
        finish<kMode, true>(a, t.row0 + j, count, t.n0 + n_lane, z[0], z[kSlabs - 1]);
    } else {
#pragma unroll
        for (int sl = 0; sl < kSlabs; ++sl) finish<kMode, false>(a, t.row0 + j, count, t.n0 + sl * kSlab + n_lane, z[sl], z[sl]);
    }
}

template <int kMode, bool kGated, int kSlabs>
__global__ void __launch_bounds__(kThreads, 1)
stream_kernel(const __grid_constant__ CUtensorMap map_w0, const __grid_constant__ CUtensorMap map_w1, const __grid_constant__ CUtensorMap map_x, const StreamArgs a)
{
    static_assert(!kGated || kSlabs == 2, "gate and up are a slab each");
    extern __shared__ unsigned char smem_raw[];
    const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
    __shared__ __align__(8) uint64_t s_bars[2 * kMaxStages + 5];
    __shared__ uint32_t s_tmem;
    __shared__ int s_abort;
    __shared__ unsigned s_last;
    const uint32_t full0 = smem_u32(s_bars), empty0 = full0 + 8 * kMaxStages, acc_full0 = empty0 + 8 * kMaxStages, acc_empty0 = acc_full0 + 16, drained = acc_empty0 + 16;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int NS = a.nstage;

    if (tid == 0) {
        s_abort = 0;
        for (int i = 0; i < NS; ++i) { mbar_init(full0 + 8 * i, 1); mbar_init(empty0 + 8 * i, 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(acc_full0 + 8 * i, 1); mbar_init(acc_empty0 + 8 * i, 4); }
        mbar_init(drained, 1);
        mbar_init_fence();
    }
    if (warp == 1) tmem_alloc(&s_tmem, a.tmem_columns);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = s_tmem;

    // The plan of a programmatic chain is two kernels back and complete (the kernel before waited for it): only what the kernel before wrote has to
    // be waited for.  Without early_weights everything is behind the wait.
    if (!a.early_weights) pdl_wait_prior_grids();
    if (a.programmatic) pdl_launch_dependents();
    long units = a.units;
    if (a.planned) {
        units = (long)*a.plan.n_tiles * a.column_tiles * a.kb;
    }
    const long C = min((long)gridDim.x, units), c = blockIdx.x;   // no more CTAs than steps: then none between the first and the last of an item is without a share
    Walk all{0, 0, a.kb, 0, 0, 0};
    if (c < C) { all.unit = c * units / C; all.end = (c + 1) * units / C; }
    int filled = 0;                                            // stages filled so far (warp 0)

    if (warp == 0) {
        const uint64_t stream = l2_policy_evict_first(), keep = l2_policy_evict_last();
        if (lane == 0) { tma_prefetch_descriptor(&map_w0); tma_prefetch_descriptor(&map_w1); tma_prefetch_descriptor(&map_x); }
        auto weights = [&](const Item &t, int k, int s) {      // one lane
            const uint32_t dst = base + (uint32_t)s * a.stage_bytes, bar = full0 + 8 * s;
#pragma unroll
            for (int sl = 0; sl < kSlabs; ++sl) {
                const CUtensorMap *m = kGated && sl ? &map_w1 : &map_w0;
                const int n = t.n0 + (kGated ? 0 : sl * kSlab);
                if (a.col) {
                    tma_load_3d(dst + sl * kSlabBytes, m, k * kKT, n, t.expert, bar, stream);
                } else {
                    tma_load_3d(dst + sl * kSlabBytes, m, n, k * kKT, t.expert, bar, stream);
                    tma_load_3d(dst + sl * kSlabBytes + kSlabBytes / 2, m, n + 64, k * kKT, t.expert, bar, stream);
                }
            }
        };
        // bytes of a step's token rows: groups of four gathered rows, or of eight rows as they lie, for each term
        auto token_bytes = [&](const Item &t) { return a.gather ? (uint32_t)ceil_div(t.rows, 4) * 512u : (uint32_t)ceil_div(t.rows, 8) * 1024u * a.terms; };
        auto rows_of = [&](const Item &t, int (&ids)[4]) {     // lane i: the token rows of group i
            if (!a.gather) return;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = 4 * lane + i;
                ids[i] = r < t.rows ? NM_LD(a.plan.order + t.row0 + r, a.in_order, a.status) / a.plan.top_k : 0;
            }
        };
        auto tokens = [&](const Item &t, const int (&ids)[4], int k, int s) {
            const uint32_t dst = base + (uint32_t)s * a.stage_bytes + kSlabs * kSlabBytes, bar = full0 + 8 * s;
            if (a.gather) {
                if (4 * lane < t.rows) tma_gather4(dst + lane * 512, &map_x, k * kKT, ids, bar, keep);
            } else {
                const int group = lane & 15, term = lane >> 4;
                if (8 * group < t.rows && term < a.terms)
                    tma_load_3d(dst + (uint32_t)term * a.R * 128 + group * 1024, &map_x, k * kKT, t.row0 + 8 * group, term, bar, keep);
            }
        };
        // The first fills: weights before the wait, tokens behind it.
        int head = 0;
        if (a.early_weights) {
            Walk w = all;
            while (head < NS && w.next()) {
                const Item t = item_of(a, w.item);
                for (int k = w.k0; k < w.k1 && head < NS; ++k, ++head) {
                    if (lane == 0) {
                        mbar_arrive_expect_tx(full0 + 8 * head, kSlabs * kSlabBytes + token_bytes(t));
                        weights(t, k, head);
                    }
                }
            }
            filled = head;
            pdl_wait_prior_grids();
        }
        __syncwarp();
        Walk w = all;
        int s = 0, n = 0;
        uint32_t ph = 1;                                        // a fresh barrier passes a wait for the phase before its first
        bool ok = true;
        while (ok && w.next()) {
            const Item t = item_of(a, w.item);
            int ids[4] = {0, 0, 0, 0};
            rows_of(t, ids);
            for (int k = w.k0; k < w.k1; ++k, ++n) {
                if (n >= head) {
                    if (lane == 0) {
                        ok = mbar_try_wait(empty0 + 8 * s, ph) || mbar_wait(empty0 + 8 * s, ph, &s_abort, a.status);
                        if (ok) {
                            mbar_arrive_expect_tx(full0 + 8 * s, kSlabs * kSlabBytes + token_bytes(t));
                            weights(t, k, s);
                            filled = n + 1;
                        }
                    }
                    ok = __shfl_sync(0xffffffffu, ok, 0);
                    if (!ok) break;
                }
                tokens(t, ids, k, s);
                if (++s == NS) { s = 0; ph ^= 1; }
            }
        }
    } else if (warp == 1) {
        // The whole warp walks, one elected lane issues: descriptors are then uniform values.
        const bool leader = elect_one();
        Walk w = all;
        int s = 0, acc = 0;
        uint32_t ph = 0, acc_ph = 1;
        bool ok = true;
        while (ok && w.next()) {
            const Item t = item_of(a, w.item);
            const int columns = max(16, (t.rows + 15) & ~15);
            const uint32_t idesc = a.f16 ? instr_desc_f16(kSlab, columns, !a.col, false) : instr_desc(kSlab, columns, !a.col, false);
            ok = mbar_try_wait(acc_empty0 + 8 * acc, acc_ph) || mbar_wait(acc_empty0 + 8 * acc, acc_ph, &s_abort, a.status);
            if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
            tc_fence_after();
            const uint32_t d = tmem + (uint32_t)acc * kSlabs * a.R;
            for (int k = w.k0; k < w.k1; ++k) {
                ok = mbar_try_wait(full0 + 8 * s, ph) || mbar_wait(full0 + 8 * s, ph, &s_abort, a.status);
                if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
                tc_fence_after();
                const uint32_t sw = base + (uint32_t)s * a.stage_bytes, sx = sw + kSlabs * kSlabBytes;
                if (leader) {
#pragma unroll
                    for (int kk = 0; kk < kKT / 16; ++kk)
#pragma unroll
                        for (int sl = 0; sl < kSlabs; ++sl) {
                            const uint32_t swl = sw + sl * kSlabBytes;
                            const uint64_t wd = a.col ? smem_desc(swl + kk * 32, 16, 1024) : smem_desc(swl + kk * 2048, kSlabBytes / 2, 1024);
                            mma_ss(d + sl * a.R, wd, smem_desc(sx + kk * 32, 16, 1024), idesc, k != w.k0 || kk != 0);
                            if (a.terms == 2) mma_ss(d + sl * a.R, wd, smem_desc(sx + a.R * 128 + kk * 32, 16, 1024), idesc, true);
                        }
                    mma_commit(empty0 + 8 * s);
                }
                if (++s == NS) { s = 0; ph ^= 1; }
            }
            if (!ok) break;
            if (leader) mma_commit(acc_full0 + 8 * acc);
            if (acc) acc_ph ^= 1;
            acc ^= 1;
        }
    } else {
        const int quad = warp & 3, n_lane = quad * 32 + lane, thread = tid - 64;
        if (a.early_weights) pdl_wait_prior_grids();            // nothing is written, and nothing of earlier kernels read, before they are done
        Walk w = all;
        int acc = 0;
        uint32_t ph = 0;
        while (w.next()) {
            const Item t = item_of(a, w.item);
            mbar_wait(acc_full0 + 8 * acc, ph, &s_abort, a.status);   // (where it ran out the walk goes on, over values that the status disowns: the
                                                                    // barriers below are for all four warps)
            tc_fence_after();
            const uint32_t d = tmem + ((uint32_t)(quad * 32) << 16) + (uint32_t)acc * kSlabs * a.R;
            const bool whole = w.k0 == 0 && w.k1 == a.kb;
            float *mine = a.partial + (size_t)(2 * c + (w.k0 == 0 ? 1 : 0)) * a.R * (kSlabs * kSlab);
            for (int j = 0; j < t.rows; j += 16) {
                uint32_t bits[kSlabs][16];
                float z[kSlabs][16];
#pragma unroll
                for (int sl = 0; sl < kSlabs; ++sl) tmem_ld16(d + sl * a.R + j, bits[sl]);
                tmem_wait_ld();
#pragma unroll
                for (int sl = 0; sl < kSlabs; ++sl)
#pragma unroll
                    for (int i = 0; i < 16; ++i) z[sl][i] = __uint_as_float(bits[sl][i]);
                const int count = min(16, t.rows - j);
                if (whole) {
                    if constexpr (kGated) {
                        finish<kMode, true>(a, t.row0 + j, count, t.n0 + n_lane, z[0], z[kSlabs - 1]);
                    } else {
#pragma unroll
                        for (int sl = 0; sl < kSlabs; ++sl)
                            finish<kMode, false>(a, t.row0 + j, count, t.n0 + sl * kSlab + n_lane, z[sl], z[sl]);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 16; i += 4)
                        if (i < count)
#pragma unroll
                            for (int sl = 0; sl < kSlabs; ++sl)
                                NM_ST(reinterpret_cast<float4 *>(mine) + ((j + i) / 4 * kSlabs + sl) * kSlab + n_lane,
                                      make_float4(z[sl][i], z[sl][i + 1], z[sl][i + 2], z[sl][i + 3]), a.in_partial, a.status);
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(acc_empty0 + 8 * acc);
            if (acc) ph ^= 1;
            acc ^= 1;
            if (whole) continue;

            // The CTAs that share the item: those of its first and last step, and all between.
            const long u0 = w.item * a.kb, u1 = u0 + a.kb - 1;
            const int first = (int)(((u0 + 1) * C - 1) / units), last = (int)(((u1 + 1) * C - 1) / units);
            __threadfence();
            named_barrier_sync(1, 128);
            if (thread == 0) {
                const unsigned there = atomicAdd(a.counters + first, 1u);
                s_last = there == (unsigned)(last - first);
                if (s_last) a.counters[first] = 0u;             // ready for the next call
            }
            named_barrier_sync(1, 128);
            if (!s_last) continue;
            __threadfence();
            // Few rows: many pieces on their way at once; more rows: more of each piece.
            if (t.rows <= 4) join<kMode, kGated, kSlabs, 1, 8>(a, t, 0, first, last, n_lane);
            else for (int j = 0; j < t.rows; j += 16) join<kMode, kGated, kSlabs, 4, 2>(a, t, j, first, last, n_lane);
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

template <int kMode, bool kGated, int kSlabs>
cudaError_t launch_stream(const CUtensorMap &w0, const CUtensorMap &w1, const CUtensorMap &x, const StreamArgs &a, long ctas, cudaStream_t s)
{
    static std::atomic<unsigned long long> configured{0};
    auto kern = stream_kernel<kMode, kGated, kSlabs>;
    cudaError_t e = ensure_dynamic_smem(kern, kRingBytes + 1024, configured);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ctas);
    cfg.blockDim = dim3(kThreads);
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

size_t stream_partial_bytes(int R, int slabs) { return (size_t)2 * kSMs * R * slabs * kSlab * sizeof(float); }

int stream_tile_rows(double average, int most)
{
    for (int R = 16; R < 128; R *= 2)
        if (R >= most || R >= 2 * average + 8) return R;
    return 128;
}

int stream_slabs(int R, bool gated) { return gated || R == 128 ? 2 : 1; }

cudaError_t launch_product(int mode, bool gated, const ProductArgs &p, cudaStream_t s, const char **what)
{
    StreamArgs a{};
    const int slabs = stream_slabs(p.R, gated);
    a.kb = ceil_div(p.K, kKT);
    a.tile_n = gated ? kSlab : slabs * kSlab;
    a.column_tiles = ceil_div(p.N, a.tile_n);
    a.rows = p.rows; a.N = p.N; a.R = p.R; a.terms = p.terms;
    a.items = p.planned ? 0 : (long)ceil_div(p.rows, p.R) * a.column_tiles;
    a.units = a.items * a.kb;
    a.stage_bytes = slabs * kSlabBytes + p.terms * p.R * 128;
    a.nstage = std::min(kMaxStages, kRingBytes / a.stage_bytes);
    a.tmem_columns = std::max(32, 2 * slabs * p.R);
    a.col = p.col; a.f16 = p.f16; a.gather = p.gather; a.planned = p.planned; a.early_weights = p.early_weights; a.programmatic = p.programmatic;
    a.act = p.act; a.plan = p.plan;
    a.bias = static_cast<const uint16_t *>(p.bias); a.residual = static_cast<const uint16_t *>(p.residual); a.ld_residual = p.ld_residual;
    a.out = p.out; a.ldo = p.ldo; a.out_term = (long)p.rows * p.ldo; a.row_scale = p.row_scale;
    a.partial = p.partial; a.counters = p.counters;
    const int parts = gated ? 2 : 1;
    a.in_bias = make_span(p.bias, p.bias ? 2 * (size_t)parts * p.N : 0);
    a.in_residual = make_span(p.residual, p.residual ? 2 * ((size_t)(p.rows - 1) * p.ld_residual + p.N) : 0);
    a.in_out = make_span(p.out, mode == kOutAct ? 2 * ((size_t)(p.rows - 1) * p.ldo + p.N) : 4 * (size_t)p.rows * p.ldo);
    a.in_scale = make_span(p.row_scale, p.row_scale ? 4 * (size_t)p.rows : 0);
    a.in_partial = make_span(p.partial, stream_partial_bytes(p.R, slabs));
    a.in_tiles = make_span(p.plan.tiles, sizeof(RowTile) * ((size_t)p.E + p.rows / p.R));
    a.in_order = make_span(p.plan.order, 4 * (size_t)p.rows);
    a.status = device_status_ptr();

    CUtensorMap w[2], x;
    const uint16_t *W = static_cast<const uint16_t *>(p.W);
    bool ok = true;
    for (int part = 0; part < parts; ++part) {
        const cuuint64_t wide = (cuuint64_t)parts * p.N;
        if (p.col) {
            const cuuint64_t dims[3] = {(cuuint64_t)p.K, (cuuint64_t)p.N, (cuuint64_t)p.E}, strides[2] = {(cuuint64_t)p.K * 2, (cuuint64_t)p.w_expert * 2};
            const cuuint32_t box[3] = {kKT, kSlab, 1};
            ok = ok && encode_map(&w[part], W + (size_t)part * p.N * p.K, p.f16, 3, dims, strides, box);
        } else {
            const cuuint64_t dims[3] = {(cuuint64_t)p.N, (cuuint64_t)p.K, (cuuint64_t)p.E}, strides[2] = {wide * 2, (cuuint64_t)p.w_expert * 2};
            const cuuint32_t box[3] = {64, kKT, 1};
            ok = ok && encode_map(&w[part], W + (size_t)part * p.N, p.f16, 3, dims, strides, box);
        }
    }
    if (p.gather) {
        const cuuint64_t dims[2] = {(cuuint64_t)p.K, (cuuint64_t)p.x_rows}, strides[1] = {(cuuint64_t)p.ldx * 2};
        const cuuint32_t box[2] = {kKT, 1};
        ok = ok && encode_map(&x, p.x, p.f16, 2, dims, strides, box);
    } else {
        const cuuint64_t dims[3] = {(cuuint64_t)p.K, (cuuint64_t)p.x_rows, (cuuint64_t)p.terms}, strides[2] = {(cuuint64_t)p.ldx * 2, (cuuint64_t)p.x_term * 2};
        const cuuint32_t box[3] = {kKT, 8, 1};
        ok = ok && encode_map(&x, p.x, p.f16, 3, dims, strides, box);
    }
    if (!ok) { *what = "cuTensorMapEncodeTiled"; return cudaErrorInvalidValue; }
    if (!a.status) { *what = "device status word"; return cudaErrorInvalidValue; }
    *what = "streamed product launch";
    const long ctas = p.planned ? kSMs : std::min<long>(kSMs, a.units);
    if (!gated) w[1] = w[0];
    switch (mode) {
    case kOutAct:
        return gated ? launch_stream<kOutAct, true, 2>(w[0], w[1], x, a, ctas, s)
                     : slabs == 2 ? launch_stream<kOutAct, false, 2>(w[0], w[1], x, a, ctas, s) : launch_stream<kOutAct, false, 1>(w[0], w[1], x, a, ctas, s);
    case kOutHidden:
        return gated ? launch_stream<kOutHidden, true, 2>(w[0], w[1], x, a, ctas, s)
                     : slabs == 2 ? launch_stream<kOutHidden, false, 2>(w[0], w[1], x, a, ctas, s) : launch_stream<kOutHidden, false, 1>(w[0], w[1], x, a, ctas, s);
    default:
        return slabs == 2 ? launch_stream<kOutDown, false, 2>(w[0], w[1], x, a, ctas, s) : launch_stream<kOutDown, false, 1>(w[0], w[1], x, a, ctas, s);
    }
}

}  // namespace nm
