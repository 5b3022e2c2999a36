// Narrow product with 4-bit weights: C[m][n] = sum_k A[m][k] * (code[n][k] - 8) * scale[n][k / group], 1 <= M <= 16.
//
// Bound: the packed weights, N * K / 2 bytes, read once (plus 2 bytes of scale per group).  At 6.5 TB/s that is about 46 codes
// per clock and SM, so unpacking has to cost less than three lane-instructions per code for every M, and the products have to
// be matrix instructions: mma.m16n8k16 with the weights as the 16-row operand and the tokens as the 8-column one, fed from
// registers.  (tcgen05 takes its operands from shared or tensor memory only: the unpacked 16-bit codes would cost a store and
// a read of four times the packed bytes there, and at 2 * 16 flops per code the warp-level matrix pipe is not the limit.)
// The storage of nm_w4.cuh makes a lane's 16-byte load its operand.
//   unpack   A code c in the low (high) nibble of a 16-bit half IS the fp16 number c * 2^-24 (c * 2^-20): a subnormal, which the
//            matrix unit multiplies exactly.  So w & 0x000f000f, w & 0x00f000f0 and the same of w >> 8 are the four registers of the
//            weight operand: five instructions for eight codes.  Low nibbles are rows g of the product and high ones rows g + 8, so
//            the factor 16 goes into the scale of those rows.  (With the usual detour over 128 + c in bf16 - shift, mask, subtract
//            - the kernel was bound by issue slots: 78 instructions a block of 1024 codes, 26 clocks of an SM against 22 of HBM.)
//   minus 8  sum_k a (c - 8) = sum_k a c - 8 sum_k a: the second term, one number per token and scale group, is computed when
//            the tokens are copied to shared memory and is what the group's accumulator starts from.  All of it is fp32; the
//            error is that of adding terms of size 15 |a| instead of 8 |a|.
//   tokens   fp16 as they are; bf16 ones times a power of two that puts the largest of the 64 (32) tokens that share a sum into
//            fp16's last two binades, 2^14 to 2^16: bf16's eight bits fit fp16's eleven, exactly down to 2^-28 of that largest value and to
//            2^-39 of it absolutely below.  The inverse is a square, one root of which multiplies the sum and one the scale: neither product
//            leaves fp32 unless the result does, whatever the tokens' size.
//   scale    multiplies the fp32 sum of its group; nothing is rounded before the output.
//   split    a CTA is eight warps, wn of them side by side over units (a unit: one strip, or two for M > 8), 8 / wn along k; up
//            to eight CTAs of a cluster split k further.  Two to four CTAs share an SM, so that one fills its tokens while another
//            streams.  Partial sums meet in shared memory, then in that of the cluster's first CTA, added in a fixed order:
//            no workspace, no atomics, the same bits every time, and calls on different streams share nothing.
// Measured back to back, weights from HBM: M = 1, 16384 x 7168, groups of 64: 16.7 us (62 MB, 3.7 TB/s; loads without the
// products take 13), M = 8: 22.0; 7168 x 576: 4.5 us; 1536 x 24576: 8.7 us, M = 4: 9.7; M = 16, 7168 x 18432: 28.8 us.  What bounds it: M <= 8 a start and an end
// of about 5 us around a stream at 5 to 6 TB/s; M > 8 the tokens - made ready once per SM, and read from shared memory
// by every warp.  Built, measured and left: one CTA per SM whose warps walk evenly over all blocks of its share (20.8 us for the first: its
// start and end are not hidden by another CTA), rings in shared memory by asynchronous copies (the same stream, more instructions).
#include <type_traits>

#include "nm_async.cuh"
#include "nm_w4.cuh"

namespace nm {

namespace {

// Warps of a CTA: for M > 8 one CTA of sixteen per SM, so that the tokens are made ready once per SM; else two of eight, one of
// which streams while the other starts or ends.
__host__ __device__ constexpr int w4_warps(int nt) { return nt == 1 ? 8 : 16; }
constexpr int kSmemMost = 224 * 1024;              // of an SM; a CTA of eight warps takes half of it

// Bytes of the partial sums' exchange: tiles of the cluster's CTAs and of the other warps along k, or the finished tile.
inline int w4_sum_bytes(int nt, int wn, int cl)
{
    const int tile = wn * nt * nt * 4 * 32, wk = w4_warps(nt) / wn, red = ((cl > 1 ? cl : 0) + wk - 1) * tile;
    return (red > tile ? red : tile) * (int)sizeof(float);          // (a finished tile is as large: 8 nt rows of 16 nt wn columns)
}

struct W4Args {
    const uint16_t *A;
    const uint4 *packed;
    const uint32_t *scales;
    void *C;
    long lda, ldc;
    int M, N, K;
    int nb, kb;                                    // strips, blocks along k
    int groups;                                    // groups along k
    int group_shift;                               // log2 of the 64-k blocks a scale covers (groups of 64 and more)
    int wn_log2;                                   // log2 of the warps side by side over units
    int cl, blocks_each, blocks_more;              // CTAs of a cluster, each a part of k: quotient and remainder of the shares
    int chunk;                                     // blocks along k whose tokens a CTA holds at a time
    int pitch;                                     // bytes between token rows in shared memory
    int tok_bytes;                                 // of the tokens, the starts of the sums and the powers of two
    int scale_bytes;
    int vec;                                       // token rows start on 16 bytes
    unsigned *status;                              // of the debug build's checks
};
// extents of the operands, for the same
[[maybe_unused]] __device__ __forceinline__ Span span_of_tokens(const W4Args &a) { return make_span(a.A, 2 * ((a.M - 1) * (size_t)a.lda + a.K)); }
[[maybe_unused]] __device__ __forceinline__ Span span_of_codes(const W4Args &a) { return make_span(a.packed, (size_t)a.nb * a.kb * kW4BlockBytes); }
[[maybe_unused]] __device__ __forceinline__ Span span_of_scales(const W4Args &a) { return make_span(a.scales, (size_t)a.groups * a.nb * kW4Cols * 2); }
template <typename TO> [[maybe_unused]] __device__ __forceinline__ Span span_of_result(const W4Args &a) { return make_span(a.C, sizeof(TO) * ((a.M - 1) * (size_t)a.ldc + a.N)); }

// eight codes of a word -> the four registers of the weight operand
__device__ __forceinline__ void unpack_codes(uint32_t w, uint32_t (&r)[4])
{
    const uint32_t v = w >> 8;
    r[0] = w & 0x000f000fu; r[1] = w & 0x00f000f0u;
    r[2] = v & 0x000f000fu; r[3] = v & 0x00f000f0u;
}
__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// scales of rows g and g + 8, the latter with the 1 / 16 of its codes' place; fp16 tokens have no power of two of their own, so the
// 2^24 of the codes goes in here
template <typename T> __device__ __forceinline__ float2 scale_pair(uint32_t v)
{
    if constexpr (std::is_same<T, bf16_t>::value) return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u) * 0.0625f);
    else {
        const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&v));
        return make_float2(f.x * 16777216.f, f.y * 1048576.f);
    }
}

__device__ __forceinline__ void cp_async4(uint32_t dst, const void *src)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_wait_all() { asm volatile("cp.async.wait_all;" ::: "memory"); }
// Predicated load: no branch, so that the loads of a ring stay in flight behind each other.
__device__ __forceinline__ void ld_weights_if(uint4 &v, const void *p, bool ok)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %5, 0;\n\t@p ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];\n\t}"
                 : "+r"(v.x), "+r"(v.y), "+r"(v.z), "+r"(v.w) : "l"(p), "r"((uint32_t)ok));
}

// Tokens of n k from k0 on to shared memory, ready for the product, zeros beyond K; the row pitch is 64 bytes off a multiple of
// 128, so that the eight 16-byte reads of a quarter warp (two rows, 64 bytes each) hit 32 different banks.  One pass: the eight
// (four) lanes that hold the tokens of a sum find their largest and their sum by shuffles.  Per sum and eight rows goes to
// s_start what lane (g, t) needs for tokens 2 t and 2 t + 1: where the accumulators start, -8 sum a in units of 2^-24, for row g
// and 16 times that for row g + 8; and to s_inv the roots of the powers of two taken out of the tokens and the codes.  Every CTA begins at a place of its own
// (`turn`, a multiple of 8): all of them read the same few rows, and in step they would queue for the same lines of L2.
template <typename T, bool kG32>
__device__ __forceinline__ void stage_tokens(unsigned char *s, float *s_start, float *s_inv, const W4Args &a, int k0, int n, int turn)
{
    constexpr bool kBf16 = std::is_same<T, bf16_t>::value;
    constexpr int kPer = kG32 ? 4 : 8;                             // vectors of eight tokens that share a sum
    const int per = n / 8, tiles = (a.M + 7) / 8;                  // n is a multiple of 64
    const unsigned mates = 0xffu << (threadIdx.x & 24);            // (eight lanes run together: per and blockDim are multiples of 8)
    auto fetch = [&](int c, int m, uint32_t (&w)[4]) {
        const int k = k0 + 8 * c;
        const uint16_t *src = a.A + m * a.lda + k;
        w[0] = w[1] = w[2] = w[3] = 0u;
        if (a.vec) {
            if (k < a.K) {
                const uint4 x = NM_LDG16(reinterpret_cast<const uint4 *>(src), span_of_tokens(a), a.status);
                w[0] = x.x; w[1] = x.y; w[2] = x.z; w[3] = x.w;
            }
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                w[j] = (k + 2 * j < a.K ? (uint32_t)NM_LD(src + 2 * j, span_of_tokens(a), a.status) : 0u) |
                       ((k + 2 * j + 1 < a.K ? (uint32_t)NM_LD(src + 2 * j + 1, span_of_tokens(a), a.status) : 0u) << 16);
        }
    };
    auto finish = [&](int c, int m, uint32_t (&w)[4]) {
        float inv = 1.f, sum = 0.f;
        if constexpr (kBf16) {
            uint32_t top = __vmaxu2(__vmaxu2(w[0] & 0x7fff7fffu, w[1] & 0x7fff7fffu), __vmaxu2(w[2] & 0x7fff7fffu, w[3] & 0x7fff7fffu));
            top = __vmaxu2(top, __shfl_xor_sync(mates, top, 1));
            top = __vmaxu2(top, __shfl_xor_sync(mates, top, 2));
            if constexpr (!kG32) top = __vmaxu2(top, __shfl_xor_sync(mates, top, 4));
            // exponent e of the largest, at least -112, or one more to make it odd; up = 2^(15 - e), inv^2 = 2^(24 - 15 + e)
            const int e = max((int)(max(top >> 16, top & 0xffffu) >> 7) - 127, -112) | 1;
            const float up = __uint_as_float((uint32_t)(127 + 15 - min(e, 127)) << 23);
            inv = e > 127 ? __uint_as_float(0x7fc00000u)           // (an infinity or a NaN among them: the sum is NaN)
                          : __uint_as_float((uint32_t)(127 + (9 + e) / 2) << 23);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float x = __uint_as_float(w[j] << 16) * up, y = __uint_as_float(w[j] & 0xffff0000u) * up;
                const __half2 h = __floats2half2_rn(x, y);
                w[j] = *reinterpret_cast<const uint32_t *>(&h);
                sum += x + y;                                      // (what fp16 drops of them is below 2^-39 of the largest)
            }
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w[j]));
                sum += f.x + f.y;
            }
        }
        *reinterpret_cast<uint4 *>(s + m * a.pitch + 16 * c) = make_uint4(w[0], w[1], w[2], w[3]);
        sum += __shfl_xor_sync(mates, sum, 1);
        sum += __shfl_xor_sync(mates, sum, 2);
        if constexpr (!kG32) sum += __shfl_xor_sync(mates, sum, 4);
        if (c % kPer == 0) {
            const int at = (c / kPer) * tiles + (m >> 3);
            const float st = sum * (-8.f / 16777216.f);
            float *d = s_start + at * 16 + ((m & 7) >> 1) * 4 + (m & 1);
            d[0] = st; d[2] = 16.f * st;
            if constexpr (kBf16) s_inv[at * 8 + (m & 7)] = inv;
        }
    };
    auto place = [&](int i) { const int c = i + turn; return c >= per ? c - per : c; };
    // four loads on their way: of four rows, or where there are fewer of four places in a row
    const int step = blockDim.x;
    if (a.M >= 4) {
        for (int i = threadIdx.x; i < per; i += step)
            for (int m = 0; m < a.M; m += 4) {
                uint32_t w[4][4];
#pragma unroll
                for (int j = 0; j < 4; ++j) if (m + j < a.M) fetch(place(i), m + j, w[j]);
#pragma unroll
                for (int j = 0; j < 4; ++j) if (m + j < a.M) finish(place(i), m + j, w[j]);
            }
    } else {
        for (int m = 0; m < a.M; ++m)
            for (int i = threadIdx.x; i < per; i += 4 * step) {
                uint32_t w[4][4];
#pragma unroll
                for (int j = 0; j < 4; ++j) if (i + j * step < per) fetch(place(i + j * step), m, w[j]);
#pragma unroll
                for (int j = 0; j < 4; ++j) if (i + j * step < per) finish(place(i + j * step), m, w[j]);
            }
    }
}

__device__ __forceinline__ void cluster_arrive()
{
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

// kNT: groups of eight tokens; kG32: groups of 32 k (two scales per block).  A warp multiplies kNT strips side by side, so that the
// tokens of up to sixteen rows are read from shared memory half as often (their 16-byte reads would bound M > 8 otherwise).
template <typename T, typename TO, int kNT, bool kG32>
__global__ void __launch_bounds__(w4_warps(kNT) * 32, kNT == 1 ? 2 : 1) w4_kernel(const W4Args a)
{
    constexpr bool kBf16 = std::is_same<T, bf16_t>::value;
    constexpr int kS = kG32 ? 2 : 1, kSide = kNT;                    // scales of a block; strips of a unit
    constexpr int kWarps = w4_warps(kNT), kThreads = kWarps * 32, kWarpsLog2 = kNT == 1 ? 3 : 4;
    // blocks of weights on their way, per warp (bf16 in groups of 32, M > 8: 2, which spill 32 bytes a thread where three spill 172; 16 x 7168 x
    // 18432 took 35.8 us against 37.7)
    constexpr int kDepth = kNT == 1 ? 8 : (kG32 && kBf16 ? 2 : 3);
    constexpr int kVals = kSide * kNT * 4;                         // sums a lane holds
    extern __shared__ __align__(16) unsigned char s_raw[];
    unsigned char *s_tok = s_raw;
    float *s_start = reinterpret_cast<float *>(s_tok + a.M * a.pitch);     // [block (half)][eight tokens][t][4]: where the sums start
    float *s_inv = s_start + a.chunk * kS * kNT * 16;                      // [block (half)][eight tokens][8]: roots of the tokens' powers of two
    uint32_t *s_scale = reinterpret_cast<uint32_t *>(s_raw + a.tok_bytes); // [warp of the row][block (half)][side][8 pairs]
    float *s_red = reinterpret_cast<float *>(s_raw + a.tok_bytes + a.scale_bytes);
    const int tid = threadIdx.x, lane = tid & 31, g = lane >> 2, t = lane & 3;
    const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);       // the same for the whole warp, and the compiler knows
    const int wn = 1 << a.wn_log2, wk_log2 = kWarpsLog2 - a.wn_log2, wr = warp & (wn - 1), wki = warp >> a.wn_log2;
    const int rank = blockIdx.y, tile = blockIdx.x;                // (a cluster runs along y)
    const int strip = (tile * wn + wr) * kSide;
    const bool live = strip < a.nb, both = kSide == 2 && strip + 1 < a.nb;
    const int cta0 = rank * a.blocks_each + min(rank, a.blocks_more), cta1 = cta0 + a.blocks_each + (rank < a.blocks_more);
    if (a.cl > 1) cluster_arrive();                                // first half of a barrier: see the sums' exchange
    pdl_launch_dependents();

    float acc[kSide][kNT][4] = {};
    const uint4 *wp = a.packed + (long)(live ? strip : 0) * a.kb * 32 + lane;
    const long side_step = both ? (long)a.kb * 32 : 0;             // (an odd last strip is multiplied twice, the second time for nothing)
    for (int c0 = cta0; c0 < cta1; c0 += a.chunk) {                // one chunk unless the tokens of the CTA's k exceed its shared memory
        const int R = min(cta1, c0 + a.chunk) - c0;
        const int b0 = (R * wki) >> wk_log2, b1 = live ? (R * (wki + 1)) >> wk_log2 : b0;      // the warp's blocks, from c0 on
        // they pass through a ring of registers: a slot is loaded anew as soon as its block has been multiplied
        uint4 w[kDepth][kSide] = {};
        const uint4 *next = wp + (long)(c0 + b0) * 32;
#pragma unroll
        for (int i = 0; i < kDepth; ++i)
#pragma unroll
            for (int r = 0; r < kSide; ++r) {
                const uint4 *p = next + r * side_step + i * 32;
                ld_weights_if(w[i][r], p, b0 + i < b1 && NM_INSIDE(p, 16, span_of_codes(a), a.status));
            }
        next += kDepth * 32;
        if (c0 > cta0) __syncthreads();                            // the chunk before has been read
        // the scales of the warp's own blocks - a block has its own entry even where it shares a scale, so that it is found without arithmetic
        uint32_t *sw = s_scale + wr * (a.chunk * kS * kSide * 8);
        for (int j = b0 * (kS * kSide) + (lane >> 3); j < b1 * (kS * kSide); j += 4) {
            const int side = both ? j & 1 : 0, half = kG32 ? (j / kSide) & 1 : 0, blk = c0 + j / (kS * kSide);
            const int grp = kG32 ? min(2 * blk + half, a.groups - 1) : blk >> a.group_shift;
            const uint32_t *p = a.scales + (size_t)(unsigned)grp * (unsigned)(a.nb * 8) + (unsigned)(strip + side) * 8u + (lane & 7);
            if (NM_INSIDE(p, 4, span_of_scales(a), a.status)) cp_async4(smem_u32(sw + j * 8 + (lane & 7)), p);
        }
        if (c0 == cta0) pdl_wait_prior_grids();                    // weights may come early, tokens not
        stage_tokens<T, kG32>(s_tok, s_start, s_inv, a, c0 * kW4Rows, R * kW4Rows, (int)((long)R * tile / gridDim.x) * 8);
        cp_async_wait_all();
        __syncthreads();
        // lanes of tokens beyond M read the last token's: their columns of the product are never stored
        const unsigned char *tp[kNT];
#pragma unroll
        for (int n = 0; n < kNT; ++n) tp[n] = s_tok + min(g + 8 * n, a.M - 1) * a.pitch + 16 * t + b0 * (kW4Rows * 2);
        const float *st = s_start + b0 * (kS * kNT * 16) + 4 * t, *iv = s_inv + b0 * (kS * kNT * 8) + 2 * t;
        const uint32_t *sc = sw + b0 * (kS * kSide * 8) + g;
        auto multiply = [&](const uint4 (&code)[kSide], int j) {   // j: blocks from where the pointers stand
            uint4 tok[2][kNT];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int n = 0; n < kNT; ++n) tok[h][n] = *reinterpret_cast<const uint4 *>(tp[n] + j * (kW4Rows * 2) + 64 * h);
#pragma unroll
            for (int r = 0; r < kSide; ++r) {
                const uint32_t word[4] = {code[r].x, code[r].y, code[r].z, code[r].w};
                float sum[kNT][4];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if (kG32 || h == 0) {
#pragma unroll
                        for (int n = 0; n < kNT; ++n) {
                            const float4 q = *reinterpret_cast<const float4 *>(st + ((j * kS + h) * kNT + n) * 16);
                            sum[n][0] = q.x; sum[n][1] = q.y; sum[n][2] = q.z; sum[n][3] = q.w;
                        }
                    }
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        uint32_t op[4];
                        unpack_codes(word[2 * h + q], op);
#pragma unroll
                        for (int n = 0; n < kNT; ++n) mma16816(sum[n], op, q ? tok[h][n].z : tok[h][n].x, q ? tok[h][n].w : tok[h][n].y);
                    }
                    if (kG32 || h == 1) {                          // the group's sum is complete (or the block's): its scale
                        const int hs = kG32 ? h : 0;
                        const float2 f = scale_pair<T>(sc[((j * kS + hs) * kSide + r) * 8]);
#pragma unroll
                        for (int n = 0; n < kNT; ++n) {
                            float2 inv = make_float2(1.f, 1.f);
                            if constexpr (kBf16) inv = *reinterpret_cast<const float2 *>(iv + ((j * kS + hs) * kNT + n) * 8);
                            acc[r][n][0] = fmaf(f.x * inv.x, sum[n][0] * inv.x, acc[r][n][0]); acc[r][n][1] = fmaf(f.x * inv.y, sum[n][1] * inv.y, acc[r][n][1]);
                            acc[r][n][2] = fmaf(f.y * inv.x, sum[n][2] * inv.x, acc[r][n][2]); acc[r][n][3] = fmaf(f.y * inv.y, sum[n][3] * inv.y, acc[r][n][3]);
                        }
                    }
                }
            }
        };
        auto turn = [&]() {
#pragma unroll
            for (int n = 0; n < kNT; ++n) tp[n] += kDepth * (kW4Rows * 2);
            st += kDepth * (kS * kNT * 16); iv += kDepth * (kS * kNT * 8); sc += kDepth * (kS * kSide * 8);
            next += kDepth * 32;
        };
        int left = b1 - b0;
        for (; left >= 2 * kDepth; left -= kDepth) {
#pragma unroll
            for (int i = 0; i < kDepth; ++i) {
                multiply(w[i], i);
#pragma unroll
                for (int r = 0; r < kSide; ++r) w[i][r] = NM_LD_STREAM16(next + r * side_step + i * 32, span_of_codes(a), a.status);
            }
            turn();
        }
        for (; left > 0; left -= kDepth) {                         // the last one or two turns of the ring
#pragma unroll
            for (int i = 0; i < kDepth; ++i) {
                if (i < left) multiply(w[i], i);
#pragma unroll
                for (int r = 0; r < kSide; ++r) {
                    const uint4 *p = next + r * side_step + i * 32;
                    ld_weights_if(w[i][r], p, kDepth + i < left && NM_INSIDE(p, 16, span_of_codes(a), a.status));
                }
            }
            turn();
        }
    }

    // ---- partial sums: over the CTA's warps along k, then over the cluster's CTAs, each in index order --------------------
    const int wk = kWarps >> a.wn_log2, tile_vals = wn * kVals * 32;       // floats of the CTA's tile, [unit][value][lane]
    float *slots = s_red;                                          // [cluster rank][tile], used in rank 0
    float *local = s_red + (a.cl > 1 ? a.cl : 0) * tile_vals;      // [wk - 1][tile]
    const int mine = wr * kVals * 32 + lane;
    float *sums = &acc[0][0][0];
    if (wki > 0) {
        float *d = local + (wki - 1) * tile_vals + mine;
#pragma unroll
        for (int i = 0; i < kVals; ++i) d[i * 32] = sums[i];
    }
    __syncthreads();
    if (wki == 0) {
        for (int q = 0; q < wk - 1; ++q) {
            const float *v = local + q * tile_vals + mine;
#pragma unroll
            for (int i = 0; i < kVals; ++i) sums[i] += v[i * 32];
        }
    }
    if (a.cl > 1) {
        cluster_wait();                                            // every peer has started: its shared memory exists
        if (wki == 0 && rank > 0) {
            uint32_t dst;
            asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(dst) : "r"(smem_u32(slots + rank * tile_vals + mine)), "r"(0));
#pragma unroll
            for (int i = 0; i < kVals; ++i) asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(dst + 128u * i), "f"(sums[i]) : "memory");
        }
        cluster_arrive();
        cluster_wait();
        if (rank > 0) return;
        if (wki == 0) {
            for (int p = 1; p < a.cl; ++p) {
                const float *v = slots + p * tile_vals + mine;
#pragma unroll
                for (int i = 0; i < kVals; ++i) sums[i] += v[i * 32];
            }
        }
    }
    // ---- the tile leaves as rows of C: lane (g, t) holds columns g and g + 8 of tokens 2 t and 2 t + 1 ------------------------
    __syncthreads();
    constexpr int kCols = kSide * kW4Cols;
    const int cols_log2 = a.wn_log2 + (kSide == 2 ? 5 : 4), cols = 1 << cols_log2;
    if (wki == 0) {
#pragma unroll
        for (int r = 0; r < kSide; ++r)
#pragma unroll
            for (int n = 0; n < kNT; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    s_red[(8 * n + 2 * t + (i & 1)) * cols + wr * kCols + r * kW4Cols + g + 8 * (i >> 1)] = acc[r][n][i];
    }
    __syncthreads();
    TO *C = static_cast<TO *>(a.C);
    const long n0 = (long)tile * cols;
    for (int i = tid; i < a.M * cols; i += kThreads) {
        const int m = i >> cols_log2, c = i & (cols - 1);
        if (n0 + c < a.N) NM_ST(&C[(long)m * a.ldc + n0 + c], round_out<TO>(s_red[i]), span_of_result<TO>(a), a.status);
    }
}

// How many warps side by side and how many CTAs along k: the least time by a model in microseconds, fitted to sweeps of both on B200
// (shapes of 0.6 to 18 thousand columns and 1.5 to 16 thousand k).  Per wave of resident CTAs: a fixed start and end, a block of
// 1024 codes per 12.6 ns and SM (15 for two strips side by side), a block of a token row per 3 (6) ns, and a cluster's exchange of 0.8
// (3).  (With 0.8 for M > 8 too, 16 x 1536 x 40000 took 31 us instead of 23 and 16 x 7168 x 12288 34 instead of 27; with 1.6 for
// M <= 8, 4 x 7168 x 1536 10 instead of 7.)
// `resident`: clusters of each size that run at once (their CTAs need SMs of one GPC, so not every size fills the machine).
struct W4Plan { int wn, cl; };
std::atomic<unsigned> g_w4_forced{0};              // nm_debug_set_w4_plan: warps across | CTAs << 8 | blocks of a piece << 16
W4Plan plan_w4(int M, int units, int kb, const int (&resident)[9])
{
    const bool wide = M > 8;
    const int warps = w4_warps(wide ? 2 : 1);
    W4Plan best{warps, 1};
    double least = 1e300;
    for (int wn = 1; wn <= warps; wn *= 2)
        for (int cl = 1; cl <= 8 && cl <= kb; ++cl) {
            if (resident[cl] < 1 || w4_sum_bytes(wide ? 2 : 1, wn, cl) > (wide ? 96 : 40) * 1024) continue;      // (the tokens want room too)
            const int tiles = ceil_div(units, wn), blocks = ceil_div(kb, cl), run = ceil_div(blocks, warps / wn);
            const int waves = ceil_div(tiles, resident[cl]), on_sm = wide || (long)tiles * cl <= kSMs ? 1 : 2;
            const double stream = on_sm * warps * run * (wide ? 2 * 0.015 : 0.0126), tokens = on_sm * M * blocks * (wide ? 0.006 : 0.003);
            const double cost = waves * ((wide ? 2.0 : 1.5) + stream + tokens + (cl > 1 ? (wide ? 3.0 : 0.8) : 0.0));
            if (cost < least) { least = cost; best = W4Plan{wn, cl}; }
        }
    return best;
}

// Asked of one instance for all of its kind: they differ in nothing that matters here.
template <int kNT>
cudaError_t resident_clusters(int (&resident)[9])
{
    static std::atomic<unsigned long long> configured{0};
    auto kern = w4_kernel<bf16_t, bf16_t, kNT, false>;
    cudaError_t e = ensure_dynamic_smem(kern, kSmemMost, configured);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 1; attr[0].val.clusterDim.z = 1;
    cfg.blockDim = dim3(w4_warps(kNT) * 32);
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    cfg.dynamicSmemBytes = kNT == 1 ? kSmemMost / 2 : kSmemMost;
    resident[0] = 0;
    resident[1] = kNT == 1 ? 2 * kSMs : kSMs;
    for (int cl = 2; cl <= 8; ++cl) {
        attr[0].val.clusterDim.y = cl;
        cfg.gridDim = dim3(1, cl, 1);
        resident[cl] = max_clusters_cached(kern, cfg, cl);
    }
    return cudaSuccess;
}

template <typename T, typename TO, int kNT, bool kG32>
cudaError_t launch_w4(W4Args a, cudaStream_t stream, bool pdl)
{
    static std::atomic<unsigned long long> configured{0};
    auto kern = w4_kernel<T, TO, kNT, kG32>;
    cudaError_t e = ensure_dynamic_smem(kern, kSmemMost, configured);
    if (e != cudaSuccess) return e;
    constexpr int kS = kG32 ? 2 : 1, kSide = kNT, kWarps = w4_warps(kNT), kStart = kS * kNT * (std::is_same<T, bf16_t>::value ? 96 : 64);
    const int units = ceil_div(a.nb, kSide);
    int resident[9];
    e = resident_clusters<kNT>(resident);
    if (e != cudaSuccess) return e;
    W4Plan p = plan_w4(a.M, units, a.kb, resident);
    const unsigned forced = g_w4_forced.load(std::memory_order_relaxed);
    if (forced) {                                                  // (where the shape and the machine can have it)
        const W4Plan f{forced & 0xff ? (int)(forced & 0xff) : p.wn, forced >> 8 & 0xff ? (int)(forced >> 8 & 0xff) : p.cl};
        if (f.wn <= kWarps && f.cl <= a.kb && resident[f.cl] > 0 && w4_sum_bytes(kNT, f.wn, f.cl) <= (kNT == 2 ? 96 : 40) * 1024) p = f;
    }
    for (a.wn_log2 = 0; (1 << a.wn_log2) < p.wn; ++a.wn_log2) {}
    a.cl = p.cl;
    a.blocks_each = a.kb / a.cl; a.blocks_more = a.kb % a.cl;
    // per block of the CTA's k: M x 128 bytes of tokens, the starts of their sums, the scales of wn units
    const int scale_block = kS * kSide * 32 * p.wn, run = ceil_div(a.kb, a.cl), sum_bytes = w4_sum_bytes(kNT, p.wn, p.cl);
    const int fit = ((kNT == 1 ? kSmemMost / 2 : kSmemMost) - sum_bytes - a.M * 64) / (a.M * kW4Rows * 2 + kStart + scale_block);
    a.chunk = ceil_div(run, ceil_div(run, fit));
    if (forced >> 16 && a.chunk > (int)(forced >> 16)) a.chunk = (int)(forced >> 16);
    a.pitch = a.chunk * (kW4Rows * 2) + 64;
    a.tok_bytes = a.M * a.pitch + a.chunk * kStart;
    a.scale_bytes = a.chunk * scale_block;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(ceil_div(units, p.wn), a.cl, 1);
    cfg.blockDim = dim3(kWarps * 32);
    cfg.dynamicSmemBytes = a.tok_bytes + a.scale_bytes + sum_bytes;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    int n = 0;
    if (a.cl > 1) {
        attr[n].id = cudaLaunchAttributeClusterDimension;
        attr[n].val.clusterDim.x = 1; attr[n].val.clusterDim.y = a.cl; attr[n].val.clusterDim.z = 1;
        ++n;
    }
    if (pdl) {
        attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[n].val.programmaticStreamSerializationAllowed = 1;
        ++n;
    }
    cfg.attrs = attr;
    cfg.numAttrs = n;
    return cudaLaunchKernelEx(&cfg, kern, a);
}

template <typename T, typename TO>
cudaError_t dispatch_w4(const W4Args &a, bool g32, cudaStream_t s, bool pdl)
{
    if (a.M <= 8) return g32 ? launch_w4<T, TO, 1, true>(a, s, pdl) : launch_w4<T, TO, 1, false>(a, s, pdl);
    return g32 ? launch_w4<T, TO, 2, true>(a, s, pdl) : launch_w4<T, TO, 2, false>(a, s, pdl);
}

}  // namespace

}  // namespace nm

using namespace nm;

extern "C" {
#pragma GCC visibility push(default)

int nm_debug_set_w4_plan(int warps_across, int ctas_along_k, int piece_blocks)
{
    if (warps_across < 0 || warps_across > 16 || (warps_across & (warps_across - 1)) || ctas_along_k < 0 || ctas_along_k > 8 || piece_blocks < 0 || piece_blocks > 0xffff)
        return NM_ERR_INVALID_ARG;
    g_w4_forced.store((unsigned)warps_across | (unsigned)ctas_along_k << 8 | (unsigned)piece_blocks << 16, std::memory_order_relaxed);
    return NM_OK;
}

int nm_matmul_w4(const void *A, const void *packed, const void *scales, void *C, int M, int N, int K, int group, long lda, long ldc,
                 nm_dtype dtype, nm_stream stream)
{
    if (!A || !packed || !scales || !C || M < 1 || M > NM_MAX_M || N < 1 || K < 1 || lda < K || ldc < N) return NM_ERR_INVALID_ARG;
    if (!w4_dtype_ok(dtype) || !w4_group_ok(group) || K > (1 << 30)) return NM_ERR_UNSUPPORTED;
    if (((uintptr_t)A & 1u) || ((uintptr_t)packed & 15u) || ((uintptr_t)scales & 3u) || ((uintptr_t)C & (dtype == NM_BF16_F32OUT ? 3u : 1u)))
        return NM_ERR_ALIGNMENT;
    W4Args a{};
    a.A = static_cast<const uint16_t *>(A);
    a.packed = static_cast<const uint4 *>(packed);
    a.scales = static_cast<const uint32_t *>(scales);
    a.C = C;
    a.lda = lda; a.ldc = ldc;
    a.M = M; a.N = N; a.K = K;
    a.nb = (int)(((long)N + kW4Cols - 1) / kW4Cols);
    a.kb = (int)(((long)K + kW4Rows - 1) / kW4Rows);
    a.group_shift = group == 256 ? 2 : (group == 128 ? 1 : 0);
    a.groups = (int)(((long)K + group - 1) / group);
    // 16-byte token loads want 16-byte aligned rows and a K that no such load straddles
    a.vec = !((uintptr_t)A & 15u) && lda % 8 == 0 && K % 8 == 0;
    a.status = bounds_status_ptr();
    const bool pdl = programmatic_launch_enabled(), g32 = group < kW4Rows;
    cudaStream_t s = (cudaStream_t)stream;
    const cudaError_t e = dtype == NM_F16            ? dispatch_w4<f16_t, f16_t>(a, g32, s, pdl)
                          : dtype == NM_BF16_F32OUT ? dispatch_w4<bf16_t, float>(a, g32, s, pdl)
                                                    : dispatch_w4<bf16_t, bf16_t>(a, g32, s, pdl);
    return e == cudaSuccess ? NM_OK : record_cuda_error(e, "4-bit narrow matmul launch");
}

#pragma GCC visibility pop
}  // extern "C"
