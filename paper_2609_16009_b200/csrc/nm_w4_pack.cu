// Weights to 4 bits and back (storage: nm_w4.cuh).  Done once when weights are loaded; both are one pass over the weights.
//   scale = round16(max |w| of the group / 7), code = clamp(round(w / scale), -8, 7) + 8 (8 where the scale is 0),
//   back = round16((code - 8) * scale)
// A CTA takes 64 columns x 256 k through shared memory, so that either layout of the weights is read and written in runs of
// 128 bytes and more whichever way the codes run.  Bound by HBM: 2 bytes in and half a byte out per weight, and the reverse.
#include <type_traits>

#include "nm_w4.cuh"

namespace nm {

namespace {

constexpr int kCols = 64, kRows = 256, kThreads = 256;             // a CTA's tile; kRows is a multiple of every group
constexpr int kPad = kCols + 2;

template <typename T> __device__ __forceinline__ float widen16(uint16_t v) { T x; x.bits = v; return Elem<T>::widen(x); }

// The tile's weights, zeros outside N x K, as raw 16-bit values [k][column].
template <bool kColMajor>
__device__ __forceinline__ void load_tile(uint16_t (*s)[kPad], const uint16_t *__restrict__ B, int n0, int k0, int N, int K)
{
    for (int i = threadIdx.x; i < kCols * kRows; i += kThreads) {
        const int c = kColMajor ? i / kRows : i % kCols, r = kColMajor ? i % kRows : i / kCols;
        const int n = n0 + c, k = k0 + r;
        s[r][c] = (n < N && k < K) ? B[kColMajor ? (long)n * K + k : (long)k * N + n] : (uint16_t)0;
    }
}

template <typename T, bool kColMajor>
__global__ void __launch_bounds__(kThreads) w4_quantize_kernel(const uint16_t *__restrict__ B, uint4 *__restrict__ packed, uint16_t *__restrict__ scales, int N,
                                                               int K, int nb, int kb, int group)
{
    __shared__ uint16_t s_w[kRows][kPad];
    __shared__ float s_max[kRows / 32][kCols];                     // per 32 k; then the rounded scales of the groups
    const int tid = threadIdx.x, n0 = blockIdx.y * kCols, k0 = blockIdx.x * kRows;
    load_tile<kColMajor>(s_w, B, n0, k0, N, K);
    __syncthreads();
    for (int i = tid; i < kCols * (kRows / 32); i += kThreads) {
        const int c = i % kCols, q = i / kCols;
        float m = 0.f;
#pragma unroll 8
        for (int r = 0; r < 32; ++r) m = fmaxf(m, fabsf(widen16<T>(s_w[32 * q + r][c])));
        s_max[q][c] = m;
    }
    __syncthreads();
    const int per = group / 32, groups = kRows / group;
    for (int i = tid; i < kCols * groups; i += kThreads) {
        const int c = i % kCols, q = i / kCols;
        float m = 0.f;
        for (int j = 0; j < per; ++j) m = fmaxf(m, s_max[q * per + j][c]);
        const T r = round_out<T>(__fdiv_rn(m, 7.f));
        s_max[q * per][c] = Elem<T>::widen(r);                     // this thread alone reads and writes the group's entries
        const int n = n0 + c, strip = n / kW4Cols;
        if (strip < nb && k0 + q * group < K)
            scales[((long)(k0 / group + q) * nb + strip) * kW4Cols + 2 * (n % 8) + (n % kW4Cols) / 8] = r.bits;
    }
    __syncthreads();
    for (int i = tid; i < (kCols / kW4Cols) * (kRows / kW4Rows) * 32; i += kThreads) {
        const int lane = i % 32, blk = (i / 32) % (kRows / kW4Rows), st = i / (32 * (kRows / kW4Rows)), g = lane >> 2, t = lane & 3;
        const int strip = n0 / kW4Cols + st, kblk = k0 / kW4Rows + blk;
        if (strip >= nb || kblk >= kb) continue;
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            w[j] = 0;
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const int r = blk * kW4Rows + 32 * (j >> 1) + 8 * t + 4 * (j & 1) + 2 * (b & 1) + (b >> 1);
#pragma unroll
                for (int hi = 0; hi < 2; ++hi) {
                    const int c = st * kW4Cols + g + 8 * hi;
                    const float sc = s_max[(r / group) * per][c];
                    const float q = sc > 0.f ? fminf(fmaxf(rintf(__fdiv_rn(widen16<T>(s_w[r][c]), sc)), -8.f), 7.f) : 0.f;
                    w[j] |= (uint32_t)((int)q + 8) << (8 * b + 4 * hi);
                }
            }
        }
        packed[((long)strip * kb + kblk) * 32 + lane] = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

template <typename T, bool kColMajor>
__global__ void __launch_bounds__(kThreads) w4_dequantize_kernel(const uint4 *__restrict__ packed, const uint16_t *__restrict__ scales, uint16_t *__restrict__ B,
                                                                 int N, int K, int nb, int kb, int group)
{
    __shared__ uint16_t s_w[kRows][kPad];
    const int tid = threadIdx.x, n0 = blockIdx.y * kCols, k0 = blockIdx.x * kRows;
    for (int i = tid; i < (kCols / kW4Cols) * (kRows / kW4Rows) * 32; i += kThreads) {
        const int lane = i % 32, blk = (i / 32) % (kRows / kW4Rows), st = i / (32 * (kRows / kW4Rows)), g = lane >> 2, t = lane & 3;
        const int strip = n0 / kW4Cols + st, kblk = k0 / kW4Rows + blk;
        if (strip >= nb || kblk >= kb) continue;
        const uint4 v = ld_stream16(packed + ((long)strip * kb + kblk) * 32 + lane);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int k32 = k0 + blk * kW4Rows + 32 * (j >> 1);    // a word's codes share their group: a group is a multiple of 32 k
            const long at = ((long)(k32 < K ? k32 / group : 0) * nb + strip) * kW4Cols + 2 * g;
            const float sc[2] = {widen16<T>(scales[at]), widen16<T>(scales[at + 1])};
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const int r = blk * kW4Rows + 32 * (j >> 1) + 8 * t + 4 * (j & 1) + 2 * (b & 1) + (b >> 1);
#pragma unroll
                for (int hi = 0; hi < 2; ++hi)
                    s_w[r][st * kW4Cols + g + 8 * hi] = round_out<T>((float)((int)((w[j] >> (8 * b + 4 * hi)) & 15u) - 8) * sc[hi]).bits;
            }
        }
    }
    __syncthreads();
    for (int i = tid; i < kCols * kRows; i += kThreads) {
        const int c = kColMajor ? i / kRows : i % kCols, r = kColMajor ? i % kRows : i / kCols;
        const int n = n0 + c, k = k0 + r;
        if (n < N && k < K) B[kColMajor ? (long)n * K + k : (long)k * N + n] = s_w[r][c];
    }
}

int check_pack(const void *B, const void *packed, const void *scales, int N, int K, int group, int dtype, int layout)
{
    if (!B || !packed || !scales || N < 1 || K < 1) return NM_ERR_INVALID_ARG;
    if (!w4_dtype_ok(dtype) || !w4_group_ok(group) || (layout != NM_ROW_MAJOR && layout != NM_COL_MAJOR)) return NM_ERR_UNSUPPORTED;
    if (((uintptr_t)B & 1u) || ((uintptr_t)packed & 15u) || ((uintptr_t)scales & 3u)) return NM_ERR_ALIGNMENT;
    if (((long)N + kCols - 1) / kCols > 65535) return NM_ERR_UNSUPPORTED;
    return NM_OK;
}

}  // namespace

}  // namespace nm

using namespace nm;

extern "C" {
#pragma GCC visibility push(default)

size_t nm_w4_packed_bytes(int N, int K)
{
    if (N < 1 || K < 1) return 0;
    return (((size_t)N + kW4Cols - 1) / kW4Cols) * (((size_t)K + kW4Rows - 1) / kW4Rows) * kW4BlockBytes;
}

size_t nm_w4_scale_count(int N, int K, int group)
{
    if (N < 1 || K < 1 || !w4_group_ok(group)) return 0;
    return (((size_t)N + kW4Cols - 1) / kW4Cols) * kW4Cols * (((size_t)K + group - 1) / group);
}

int nm_w4_quantize(const void *B, void *packed, void *scales, int N, int K, int group, nm_dtype dtype, nm_layout layout_B, nm_stream stream)
{
    const int rc = check_pack(B, packed, scales, N, K, group, dtype, layout_B);
    if (rc != NM_OK) return rc;
    const int nb = (int)(((long)N + kW4Cols - 1) / kW4Cols), kb = (int)(((long)K + kW4Rows - 1) / kW4Rows);
    const dim3 grid((unsigned)(((long)K + kRows - 1) / kRows), (unsigned)(((long)N + kCols - 1) / kCols));
    auto go = [&](auto kern) {
        kern<<<grid, kThreads, 0, (cudaStream_t)stream>>>(static_cast<const uint16_t *>(B), static_cast<uint4 *>(packed), static_cast<uint16_t *>(scales), N, K, nb, kb, group);
    };
    if (dtype == NM_F16) layout_B == NM_COL_MAJOR ? go(w4_quantize_kernel<f16_t, true>) : go(w4_quantize_kernel<f16_t, false>);
    else layout_B == NM_COL_MAJOR ? go(w4_quantize_kernel<bf16_t, true>) : go(w4_quantize_kernel<bf16_t, false>);
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? NM_OK : record_cuda_error(e, "4-bit quantisation launch");
}

int nm_w4_dequantize(const void *packed, const void *scales, void *B, int N, int K, int group, nm_dtype dtype, nm_layout layout_B, nm_stream stream)
{
    const int rc = check_pack(B, packed, scales, N, K, group, dtype, layout_B);
    if (rc != NM_OK) return rc;
    const int nb = (int)(((long)N + kW4Cols - 1) / kW4Cols), kb = (int)(((long)K + kW4Rows - 1) / kW4Rows);
    const dim3 grid((unsigned)(((long)K + kRows - 1) / kRows), (unsigned)(((long)N + kCols - 1) / kCols));
    auto go = [&](auto kern) {
        kern<<<grid, kThreads, 0, (cudaStream_t)stream>>>(static_cast<const uint4 *>(packed), static_cast<const uint16_t *>(scales), static_cast<uint16_t *>(B), N, K, nb, kb, group);
    };
    if (dtype == NM_F16) layout_B == NM_COL_MAJOR ? go(w4_dequantize_kernel<f16_t, true>) : go(w4_dequantize_kernel<f16_t, false>);
    else layout_B == NM_COL_MAJOR ? go(w4_dequantize_kernel<bf16_t, true>) : go(w4_dequantize_kernel<bf16_t, false>);
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? NM_OK : record_cuda_error(e, "4-bit dequantisation launch");
}

#pragma GCC visibility pop
}  // extern "C"
