// Weights to 4 bits and back (storage: nm_w4.cuh).  Done once when weights are loaded; both are one pass over the weights.
//   scale = round16(max |w| of the group / 7), code = clamp(round(w / scale), -8, 7) + 8 (8 where the scale is 0),
//   back = round16((code - 8) * scale)
// A CTA takes 64 columns x 256 k through shared memory, laid out there as it is in memory (k contiguous or columns contiguous), so
// that either layout of the weights is read and written in 16-byte vectors, runs of 128 bytes and more, whichever way the codes
// run.  Bound by HBM: 2 bytes in and half a byte out per weight, and the reverse.
#include <type_traits>

#include "nm_w4.cuh"

namespace nm {

namespace {

constexpr int kCols = 64, kRows = 256, kThreads = 256;             // a CTA's tile; kRows is a multiple of every group

template <typename T> __device__ __forceinline__ float widen16(uint16_t v) { T x; x.bits = v; return Elem<T>::widen(x); }

// The tile in shared memory.  Pitches in elements: 264 puts the 16-byte vectors of eight columns into different banks, 66 the
// 2-byte accesses of lanes (g, t) at (column g, k = 8 t).
template <bool kColMajor> struct Tile {
    static constexpr int kPitch = kColMajor ? kRows + 8 : kCols + 2;
    uint16_t v[(kColMajor ? kCols : kRows) * kPitch];
    __device__ __forceinline__ uint16_t &at(int r, int c) { return v[kColMajor ? c * kPitch + r : r * kPitch + c]; }
};

// vec: every run of eight elements along the contiguous dimension starts on 16 bytes and ends inside the matrix
template <bool kColMajor>
__device__ __forceinline__ void load_tile(Tile<kColMajor> &s, const uint16_t *__restrict__ B, int n0, int k0, int N, int K, bool vec)
{
    constexpr int kInner = kColMajor ? kRows : kCols;
    if (vec) {
#pragma unroll 4
        for (int i = threadIdx.x; i < kCols * kRows / 8; i += kThreads) {
            const int in = (i % (kInner / 8)) * 8, out = i / (kInner / 8), c = kColMajor ? out : in, r = kColMajor ? in : out;
            const int n = n0 + c, k = k0 + r;
            uint4 u = make_uint4(0u, 0u, 0u, 0u);
            if (n < N && k < K) u = ld_stream16(B + (kColMajor ? (long)n * K + k : (long)k * N + n));
            uint32_t *d = reinterpret_cast<uint32_t *>(&s.at(r, c));
            if constexpr (kColMajor) *reinterpret_cast<uint4 *>(d) = u;
            else { d[0] = u.x; d[1] = u.y; d[2] = u.z; d[3] = u.w; }
        }
    } else {
        for (int i = threadIdx.x; i < kCols * kRows; i += kThreads) {
            const int in = i % kInner, out = i / kInner, c = kColMajor ? out : in, r = kColMajor ? in : out;
            const int n = n0 + c, k = k0 + r;
            s.at(r, c) = (n < N && k < K) ? B[kColMajor ? (long)n * K + k : (long)k * N + n] : (uint16_t)0;
        }
    }
}
template <bool kColMajor>
__device__ __forceinline__ void store_tile(Tile<kColMajor> &s, uint16_t *__restrict__ B, int n0, int k0, int N, int K, bool vec)
{
    constexpr int kInner = kColMajor ? kRows : kCols;
    if (vec) {
        for (int i = threadIdx.x; i < kCols * kRows / 8; i += kThreads) {
            const int in = (i % (kInner / 8)) * 8, out = i / (kInner / 8), c = kColMajor ? out : in, r = kColMajor ? in : out;
            const int n = n0 + c, k = k0 + r;
            if (n >= N || k >= K) continue;
            const uint32_t *d = reinterpret_cast<const uint32_t *>(&s.at(r, c));
            uint4 u;
            if constexpr (kColMajor) u = *reinterpret_cast<const uint4 *>(d);
            else u = make_uint4(d[0], d[1], d[2], d[3]);
            *reinterpret_cast<uint4 *>(B + (kColMajor ? (long)n * K + k : (long)k * N + n)) = u;
        }
    } else {
        for (int i = threadIdx.x; i < kCols * kRows; i += kThreads) {
            const int in = i % kInner, out = i / kInner, c = kColMajor ? out : in, r = kColMajor ? in : out;
            const int n = n0 + c, k = k0 + r;
            if (n < N && k < K) B[kColMajor ? (long)n * K + k : (long)k * N + n] = s.at(r, c);
        }
    }
}

template <typename T, bool kColMajor>
__global__ void __launch_bounds__(kThreads) w4_quantize_kernel(const uint16_t *__restrict__ B, uint4 *__restrict__ packed, uint16_t *__restrict__ scales, int N,
                                                               int K, int nb, int kb, int group, int vec)
{
    __shared__ __align__(16) Tile<kColMajor> s_w;
    __shared__ float s_max[kRows / 32][kCols + 1];                 // per 32 k: the largest, then the rounded scale of its group
    const int tid = threadIdx.x, n0 = blockIdx.y * kCols, k0 = blockIdx.x * kRows;
    load_tile<kColMajor>(s_w, B, n0, k0, N, K, vec != 0);
    __syncthreads();
    for (int i = tid; i < kCols * (kRows / 32); i += kThreads) {
        // (columns along the lanes where they are contiguous, 32-k pieces of a column otherwise)
        const int c = kColMajor ? i / (kRows / 32) : i % kCols, q = kColMajor ? i % (kRows / 32) : i / kCols;
        float m = 0.f;
        if constexpr (kColMajor) {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const uint4 u = *reinterpret_cast<const uint4 *>(&s_w.at(32 * q + 8 * r, c));
                const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) m = fmaxf(m, fmaxf(fabsf(widen16<T>((uint16_t)w[j])), fabsf(widen16<T>((uint16_t)(w[j] >> 16)))));
            }
        } else {
#pragma unroll 8
            for (int r = 0; r < 32; ++r) m = fmaxf(m, fabsf(widen16<T>(s_w.at(32 * q + r, c))));
        }
        s_max[q][c] = m;
    }
    __syncthreads();
    const int per = group / 32, groups = kRows / group;
    for (int i = tid; i < kCols * groups; i += kThreads) {
        const int c = i % kCols, q = i / kCols;
        float m = 0.f;
        for (int j = 0; j < per; ++j) m = fmaxf(m, s_max[q * per + j][c]);
        const T r = round_out<T>(__fdiv_rn(m, 7.f));
        for (int j = 0; j < per; ++j) s_max[q * per + j][c] = Elem<T>::widen(r);       // this thread alone reads and writes the group's entries
        const int n = n0 + c, strip = n / kW4Cols;
        if (strip < nb && k0 + q * group < K)
            scales[((long)(k0 / group + q) * nb + strip) * kW4Cols + 2 * (n % 8) + (n % kW4Cols) / 8] = r.bits;
    }
    __syncthreads();
    for (int i = tid; i < (kCols / kW4Cols) * (kRows / kW4Rows) * 32; i += kThreads) {
        const int lane = i % 32, blk = (i / 32) % (kRows / kW4Rows), st = i / (32 * (kRows / kW4Rows)), g = lane >> 2, t = lane & 3;
        const int strip = n0 / kW4Cols + st, kblk = k0 / kW4Rows + blk;
        if (strip >= nb || kblk >= kb) continue;
        uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
        for (int hi = 0; hi < 2; ++hi) {
            const int c = st * kW4Cols + g + 8 * hi;
#pragma unroll
            for (int h = 0; h < 2; ++h) {                          // words 2 h and 2 h + 1: eight consecutive k from 32 h + 8 t on
                const int r0 = blk * kW4Rows + 32 * h + 8 * t;
                const float sc = s_max[r0 / 32][c];
#pragma unroll
                for (int x = 0; x < 8; ++x) {                      // k = r0 + 4 (j & 1) + 2 (b & 1) + (b >> 1)
                    const int j = 2 * h + (x >> 2), b = ((x >> 1) & 1) + 2 * (x & 1);
                    const float q = sc > 0.f ? fminf(fmaxf(rintf(__fdiv_rn(widen16<T>(s_w.at(r0 + x, c)), sc)), -8.f), 7.f) : 0.f;
                    w[j] |= (uint32_t)((int)q + 8) << (8 * b + 4 * hi);
                }
            }
        }
        packed[((long)strip * kb + kblk) * 32 + lane] = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

template <typename T, bool kColMajor>
__global__ void __launch_bounds__(kThreads) w4_dequantize_kernel(const uint4 *__restrict__ packed, const uint16_t *__restrict__ scales, uint16_t *__restrict__ B,
                                                                 int N, int K, int nb, int kb, int group, int vec)
{
    __shared__ __align__(16) Tile<kColMajor> s_w;
    const int tid = threadIdx.x, n0 = blockIdx.y * kCols, k0 = blockIdx.x * kRows;
    for (int i = tid; i < (kCols / kW4Cols) * (kRows / kW4Rows) * 32; i += kThreads) {
        const int lane = i % 32, blk = (i / 32) % (kRows / kW4Rows), st = i / (32 * (kRows / kW4Rows)), g = lane >> 2, t = lane & 3;
        const int strip = n0 / kW4Cols + st, kblk = k0 / kW4Rows + blk;
        if (strip >= nb || kblk >= kb) continue;
        const uint4 v = ld_stream16(packed + ((long)strip * kb + kblk) * 32 + lane);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int r0 = blk * kW4Rows + 32 * h + 8 * t, k32 = k0 + r0 / 32 * 32;        // the codes of 32 k share their group
            const uint32_t pair = *reinterpret_cast<const uint32_t *>(scales + ((long)(k32 < K ? k32 / group : 0) * nb + strip) * kW4Cols + 2 * g);
#pragma unroll
            for (int hi = 0; hi < 2; ++hi) {
                const float sc = widen16<T>((uint16_t)(hi ? pair >> 16 : pair));
                const int c = st * kW4Cols + g + 8 * hi;
                uint32_t o[8];
#pragma unroll
                for (int x = 0; x < 8; ++x) {
                    const int j = 2 * h + (x >> 2), b = ((x >> 1) & 1) + 2 * (x & 1);
                    o[x] = round_out<T>((float)((int)((w[j] >> (8 * b + 4 * hi)) & 15u) - 8) * sc).bits;
                }
                if constexpr (kColMajor)
                    *reinterpret_cast<uint4 *>(&s_w.at(r0, c)) = make_uint4(o[0] | (o[1] << 16), o[2] | (o[3] << 16), o[4] | (o[5] << 16), o[6] | (o[7] << 16));
                else
#pragma unroll
                    for (int x = 0; x < 8; ++x) s_w.at(r0 + x, c) = (uint16_t)o[x];
            }
        }
    }
    __syncthreads();
    store_tile<kColMajor>(s_w, B, n0, k0, N, K, vec != 0);
}

// whether the contiguous dimension runs in whole, aligned 16-byte vectors
bool pack_vec(const void *B, int N, int K, int layout) { return !((uintptr_t)B & 15u) && (layout == NM_COL_MAJOR ? K : N) % 8 == 0; }

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
        kern<<<grid, kThreads, 0, (cudaStream_t)stream>>>(static_cast<const uint16_t *>(B), static_cast<uint4 *>(packed), static_cast<uint16_t *>(scales), N, K, nb, kb, group, (int)pack_vec(B, N, K, layout_B));
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
        kern<<<grid, kThreads, 0, (cudaStream_t)stream>>>(static_cast<const uint4 *>(packed), static_cast<const uint16_t *>(scales), static_cast<uint16_t *>(B), N, K, nb, kb, group, (int)pack_vec(B, N, K, layout_B));
    };
    if (dtype == NM_F16) layout_B == NM_COL_MAJOR ? go(w4_dequantize_kernel<f16_t, true>) : go(w4_dequantize_kernel<f16_t, false>);
    else layout_B == NM_COL_MAJOR ? go(w4_dequantize_kernel<bf16_t, true>) : go(w4_dequantize_kernel<bf16_t, false>);
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? NM_OK : record_cuda_error(e, "4-bit dequantisation launch");
}

#pragma GCC visibility pop
}  // extern "C"
