// Narrow product with 4-bit weights: C[m][n] = sum_k A[m][k] * (code[n][k] - 8) * scale[n][k / group], 1 <= M <= 16.
//
// Bound: the packed weights, N * K / 2 bytes, read once (plus 2 bytes of scale per group).  At 6.5 TB/s that is about 46 codes
// per clock and SM, so unpacking has to cost less than three lane-instructions per code for every M, and the products have to
// be matrix instructions: mma.m16n8k16 with the weights as the 16-row operand and the tokens as the 8-column one, fed from
// registers.  (tcgen05 takes its operands from shared or tensor memory only: the unpacked 16-bit codes would cost a store and
// a read of four times the packed bytes there, and at 2 * 16 flops per code the warp-level matrix pipe is not the limit.)
// The storage of nm_w4.cuh makes a lane's 16-byte load its operand.
//   unpack   a word w of eight codes: ((w >> 4 i) & 0x000f000f) | magic is a pair of 128 + code as bf16 (1024 + code as
//            fp16), minus 136 (1032) exactly code - 8.  The codes stay integers in the product: exact in 16 bits, the sums of a
//            group are fp32, and the scale multiplies the fp32 sum of its group - nothing is rounded before the output.
//   split    a CTA is eight warps, wn of them side by side over strips, 8 / wn along k; up to eight CTAs of a cluster split k
//            further.  Partial sums meet in shared memory, then in that of the cluster's first CTA, added in a fixed order:
//            no workspace, no atomics, the same bits every time, and calls on different streams share nothing.
#include <type_traits>

#include "nm_async.cuh"
#include "nm_w4.cuh"

namespace nm {

namespace {

constexpr int kThreads = 256, kWarps = 8;

struct W4Args {
    const uint16_t *A;
    const uint4 *packed;
    const uint32_t *scales;
    void *C;
    long lda, ldc;
    int M, N, K;
    int nb, kb;                                    // strips, blocks along k
    int blocks_per_group;                          // 64-k blocks a scale covers (groups of 64 and more)
    int wn;                                        // warps side by side over strips
    int cl;                                        // CTAs of a cluster, each a part of k
};

template <typename T> __device__ __forceinline__ uint32_t magic_sub(uint32_t v)
{
    if constexpr (std::is_same<T, bf16_t>::value) {
        const __nv_bfloat162 r = __hsub2(*reinterpret_cast<const __nv_bfloat162 *>(&v),
                                         __halves2bfloat162(__ushort_as_bfloat16(0x4308), __ushort_as_bfloat16(0x4308)));
        return *reinterpret_cast<const uint32_t *>(&r);
    } else {
        const __half2 r = __hsub2(*reinterpret_cast<const __half2 *>(&v), __halves2half2(__ushort_as_half(0x6408), __ushort_as_half(0x6408)));
        return *reinterpret_cast<const uint32_t *>(&r);
    }
}
// eight codes of a word -> the four registers of the weight operand
template <typename T> __device__ __forceinline__ void unpack_codes(uint32_t w, uint32_t (&r)[4])
{
    constexpr uint32_t magic = std::is_same<T, bf16_t>::value ? 0x43004300u : 0x64006400u;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = magic_sub<T>(((w >> (4 * i)) & 0x000f000fu) | magic);
}
template <typename T> __device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    if constexpr (std::is_same<T, bf16_t>::value)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <typename T> __device__ __forceinline__ float2 scale_pair(uint32_t v)
{
    if constexpr (std::is_same<T, bf16_t>::value) return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
    else return __half22float2(*reinterpret_cast<const __half2 *>(&v));
}

// Eight consecutive k of a token row, zeros beyond K and for token rows beyond M (row == nullptr).
template <bool kVec> __device__ __forceinline__ uint4 load_tokens(const uint16_t *row, int k, int K)
{
    if (!row || k >= K) return make_uint4(0u, 0u, 0u, 0u);
    if constexpr (kVec) return __ldg(reinterpret_cast<const uint4 *>(row + k));
    uint32_t v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t lo = k + 2 * i < K ? row[k + 2 * i] : 0u, hi = k + 2 * i + 1 < K ? row[k + 2 * i + 1] : 0u;
        v[i] = lo | (hi << 16);
    }
    return make_uint4(v[0], v[1], v[2], v[3]);
}

__device__ __forceinline__ void cluster_barrier()
{
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// kNT: groups of eight tokens; kG32: groups of 32 k (two scales per block); kVec: tokens in 16-byte loads
template <typename T, typename TO, int kNT, bool kG32, bool kVec>
__global__ void __launch_bounds__(kThreads, 2) w4_kernel(const W4Args a)
{
    constexpr int kDepth = kNT == 1 ? 4 : 2;                       // blocks on their way while as many are multiplied
    constexpr int kS = kG32 ? 2 : 1;
    extern __shared__ float s_red[];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    const int wn = a.wn, wk = kWarps / wn, wr = warp % wn, wki = warp / wn;
    const int rank = blockIdx.x, tile = blockIdx.y;
    const int strip = tile * wn + wr;
    const bool live = strip < a.nb;
    const int part = rank * wk + wki, parts = wk * a.cl;
    const int b0 = (int)((long)a.kb * part / parts), b1 = live ? (int)((long)a.kb * (part + 1) / parts) : b0;
    pdl_launch_dependents();

    float acc[kNT][4] = {};
    struct Stage { uint4 w; uint32_t s[kS]; };
    const uint4 *wp = a.packed + (long)(live ? strip : 0) * a.kb * 32 + lane;
    const uint32_t *sp = a.scales + (long)(live ? strip : 0) * 8 + g;
    auto load_stage = [&](Stage &st, int b) {
        if (b < b1) {
            st.w = ld_stream16(wp + (long)b * 32);
#pragma unroll
            for (int i = 0; i < kS; ++i) {
                const int grp = kG32 ? min(2 * b + i, (a.K - 1) / 32) : b / a.blocks_per_group;
                st.s[i] = __ldg(sp + (long)grp * a.nb * 8);
            }
        } else {
            st.w = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
            for (int i = 0; i < kS; ++i) st.s[i] = 0u;
        }
    };
    const uint16_t *row[kNT];
#pragma unroll
    for (int n = 0; n < kNT; ++n) row[n] = g + 8 * n < a.M ? a.A + (long)(g + 8 * n) * a.lda : nullptr;

    Stage cur[kDepth], nxt[kDepth];
#pragma unroll
    for (int i = 0; i < kDepth; ++i) load_stage(cur[i], b0 + i);
    pdl_wait_prior_grids();                                        // weights may come early, tokens not
    for (int b = b0; b < b1; b += kDepth) {
        uint4 tok[kDepth][kNT][2];
#pragma unroll
        for (int i = 0; i < kDepth; ++i)
#pragma unroll
            for (int n = 0; n < kNT; ++n)
#pragma unroll
                for (int h = 0; h < 2; ++h)                        // a block of the next warp's part meets zero codes' scales: not loaded
                    tok[i][n][h] = b + i < b1 ? load_tokens<kVec>(row[n], (b + i) * kW4Rows + 32 * h + 8 * t, a.K) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
        for (int i = 0; i < kDepth; ++i) load_stage(nxt[i], b + kDepth + i);
#pragma unroll
        for (int i = 0; i < kDepth; ++i) {
            const uint32_t w[4] = {cur[i].w.x, cur[i].w.y, cur[i].w.z, cur[i].w.w};
            float sum[kNT][4] = {};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint32_t op[4];
                unpack_codes<T>(w[j], op);
#pragma unroll
                for (int n = 0; n < kNT; ++n) {
                    const uint4 &v = tok[i][n][j >> 1];
                    mma16816<T>(sum[n], op, (j & 1) ? v.z : v.x, (j & 1) ? v.w : v.y);
                }
                if ((kG32 && j == 1) || j == 3) {                  // the group's sum is complete (or the block's): its scale
                    const float2 sc = scale_pair<T>(cur[i].s[kG32 ? j >> 1 : 0]);
#pragma unroll
                    for (int n = 0; n < kNT; ++n) {
                        acc[n][0] = fmaf(sc.x, sum[n][0], acc[n][0]); acc[n][1] = fmaf(sc.x, sum[n][1], acc[n][1]);
                        acc[n][2] = fmaf(sc.y, sum[n][2], acc[n][2]); acc[n][3] = fmaf(sc.y, sum[n][3], acc[n][3]);
                        sum[n][0] = sum[n][1] = sum[n][2] = sum[n][3] = 0.f;
                    }
                }
            }
        }
#pragma unroll
        for (int i = 0; i < kDepth; ++i) cur[i] = nxt[i];
    }

    // ---- partial sums: over the CTA's warps along k, then over the cluster's CTAs, each in index order --------------------
    constexpr int kVals = kNT * 4;                                 // floats a lane holds
    const int tile_vals = wn * kVals * 32;                         // floats of the CTA's tile, [strip warp][value][lane]
    float *slots = s_red;                                          // [cluster rank][tile], used in rank 0
    float *local = s_red + (a.cl > 1 ? a.cl : 0) * tile_vals;      // [wk - 1][tile]
    const int mine = wr * kVals * 32 + lane;
    if (wki > 0) {
        float *d = local + (wki - 1) * tile_vals + mine;
#pragma unroll
        for (int n = 0; n < kNT; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) d[(n * 4 + i) * 32] = acc[n][i];
    }
    __syncthreads();
    if (wki == 0) {
        for (int w = 0; w < wk - 1; ++w) {
            const float *s = local + w * tile_vals + mine;
#pragma unroll
            for (int n = 0; n < kNT; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[n][i] += s[(n * 4 + i) * 32];
        }
    }
    if (a.cl > 1) {
        // peers have all started (their shared memory exists) once this barrier is passed; the second one orders the stores
        cluster_barrier();
        if (wki == 0 && rank > 0) {
            uint32_t dst;
            asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(dst) : "r"(smem_u32(slots + rank * tile_vals + mine)), "r"(0));
#pragma unroll
            for (int n = 0; n < kNT; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(dst + 128u * (n * 4 + i)), "f"(acc[n][i]) : "memory");
        }
        cluster_barrier();
        if (rank > 0) return;
        if (wki == 0) {
            for (int p = 1; p < a.cl; ++p) {
                const float *s = slots + p * tile_vals + mine;
#pragma unroll
                for (int n = 0; n < kNT; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[n][i] += s[(n * 4 + i) * 32];
            }
        }
    }
    // ---- the tile leaves as rows of C: lane (g, t) holds columns g and g + 8 of tokens 2 t and 2 t + 1 ------------------------
    __syncthreads();
    const int cols = wn * kW4Cols;
    if (wki == 0) {
#pragma unroll
        for (int n = 0; n < kNT; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) s_red[(8 * n + 2 * t + (i & 1)) * cols + wr * kW4Cols + g + 8 * (i >> 1)] = acc[n][i];
    }
    __syncthreads();
    TO *C = static_cast<TO *>(a.C);
    const int n0 = tile * cols;
    for (int i = tid; i < a.M * cols; i += kThreads) {
        const int m = i / cols, c = i - m * cols;
        if (n0 + c < a.N) C[(long)m * a.ldc + n0 + c] = round_out<TO>(s_red[i]);
    }
}

struct W4Plan { int wn, cl; };

W4Plan plan_w4(int nb, int kb)
{
    W4Plan p{8, 1};
    while (p.wn > 1 && ceil_div(nb, p.wn) < 2 * kSMs && kb >= 2 * (kWarps / p.wn)) p.wn /= 2;
    while (p.cl < 8 && ceil_div(nb, p.wn) * p.cl < 2 * kSMs && kb / ((kWarps / p.wn) * p.cl * 2) >= 4) p.cl *= 2;
    return p;
}

template <typename T, typename TO, int kNT, bool kG32, bool kVec>
cudaError_t launch_w4(const W4Args &a, cudaStream_t stream, bool pdl)
{
    const int wk = kWarps / a.wn, tile_vals = a.wn * kNT * 4 * 32;
    const size_t red = (size_t)((a.cl > 1 ? a.cl : 0) + wk - 1) * tile_vals, out = (size_t)(8 * kNT) * a.wn * kW4Cols;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(a.cl, ceil_div(a.nb, a.wn), 1);
    cfg.blockDim = dim3(kThreads);
    // at most eight cluster slots of eight strips and seven more tiles of one: (8 * wn + 7) KB x kNT, below 48 KB only for
    // wn * kNT <= 4 with a full cluster; plan_w4 takes a cluster when there are few strips, so wn is 1 or 2 then
    cfg.dynamicSmemBytes = (red > out ? red : out) * sizeof(float);
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    int n = 0;
    if (a.cl > 1) {
        attr[n].id = cudaLaunchAttributeClusterDimension;
        attr[n].val.clusterDim.x = a.cl; attr[n].val.clusterDim.y = 1; attr[n].val.clusterDim.z = 1;
        ++n;
    }
    if (pdl) {
        attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[n].val.programmaticStreamSerializationAllowed = 1;
        ++n;
    }
    cfg.attrs = attr;
    cfg.numAttrs = n;
    return cudaLaunchKernelEx(&cfg, w4_kernel<T, TO, kNT, kG32, kVec>, a);
}

template <typename T, typename TO, int kNT>
cudaError_t dispatch_w4(const W4Args &a, bool g32, bool vec, cudaStream_t s, bool pdl)
{
    if (g32) return vec ? launch_w4<T, TO, kNT, true, true>(a, s, pdl) : launch_w4<T, TO, kNT, true, false>(a, s, pdl);
    return vec ? launch_w4<T, TO, kNT, false, true>(a, s, pdl) : launch_w4<T, TO, kNT, false, false>(a, s, pdl);
}

}  // namespace

}  // namespace nm

using namespace nm;

extern "C" {
#pragma GCC visibility push(default)

int nm_matmul_w4(const void *A, const void *packed, const void *scales, void *C, int M, int N, int K, int group, long lda, long ldc,
                 nm_dtype dtype, nm_stream stream)
{
    if (!A || !packed || !scales || !C || M < 1 || M > NM_MAX_M || N < 1 || K < 1 || lda < K || ldc < N) return NM_ERR_INVALID_ARG;
    if (!w4_dtype_ok(dtype) || !w4_group_ok(group)) return NM_ERR_UNSUPPORTED;
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
    a.blocks_per_group = group >= kW4Rows ? group / kW4Rows : 1;
    const W4Plan p = plan_w4(a.nb, a.kb);
    a.wn = p.wn; a.cl = p.cl;
    if (ceil_div(a.nb, p.wn) > 65535) return NM_ERR_UNSUPPORTED;
    // 16-byte token loads want 16-byte aligned rows and a K that no such load straddles
    const bool vec = !((uintptr_t)A & 15u) && lda % 8 == 0 && K % 8 == 0;
    const bool pdl = programmatic_launch_enabled(), g32 = group < kW4Rows;
    cudaStream_t s = (cudaStream_t)stream;
    cudaError_t e;
    if (dtype == NM_F16) e = M <= 8 ? dispatch_w4<f16_t, f16_t, 1>(a, g32, vec, s, pdl) : dispatch_w4<f16_t, f16_t, 2>(a, g32, vec, s, pdl);
    else if (dtype == NM_BF16_F32OUT) e = M <= 8 ? dispatch_w4<bf16_t, float, 1>(a, g32, vec, s, pdl) : dispatch_w4<bf16_t, float, 2>(a, g32, vec, s, pdl);
    else e = M <= 8 ? dispatch_w4<bf16_t, bf16_t, 1>(a, g32, vec, s, pdl) : dispatch_w4<bf16_t, bf16_t, 2>(a, g32, vec, s, pdl);
    return e == cudaSuccess ? NM_OK : record_cuda_error(e, "4-bit narrow matmul launch");
}

#pragma GCC visibility pop
}  // extern "C"
