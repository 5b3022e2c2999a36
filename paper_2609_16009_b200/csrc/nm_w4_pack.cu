// Weights to 4 bits and back (storage: nm_w4.cuh).  Done once when weights are loaded; both are one pass over the weights.
//   scale = round16(max |w| of the group / 7), code = clamp(round(w / scale), -8, 7) + 8 (8 where the scale is 0),
//   back = round16((code - 8) * scale)
// A CTA takes 64 columns x 128 k (256 for groups of that many) through shared memory, laid out there as it is in memory (k
// contiguous or columns contiguous), so that either layout of the weights is read and written in 16-byte vectors, runs of 128
// bytes and more, whichever way the codes run.
// Bound by HBM: 2 bytes in and half a byte out per weight, and the reverse; 45 us either way for 16384 x 7168 weights.  Measured
// there (bf16): columns in groups of 64 are quantised in 77 us and brought back in 47, rows in 82 and 54, rows in groups of 256 in 79
// and 56.  Pieces of 64 k for the groups up to 64 took 101 and 60.  What the quantisation spends above the floor are instructions,
// some ten per weight: a division each and conversions to integers and back took 145 us.
#include <type_traits>

#include "nm_async.cuh"
#include "nm_w4.cuh"

namespace nm {

namespace {

constexpr int kCols = 64, kThreads = 256;          // columns of a CTA's tile; its k are kRows, a multiple of the group

template <typename T> __device__ __forceinline__ float widen16(uint16_t v) { T x; x.bits = v; return Elem<T>::widen(x); }

// Two elements at a time.  The largest of magnitudes passes over NaN, as fmaxf does.
template <typename T> __device__ __forceinline__ uint32_t max_abs2(uint32_t a, uint32_t b)
{
    b &= 0x7fff7fffu;
    if constexpr (std::is_same_v<T, f16_t>) {
        const __half2 m = __hmax2(*reinterpret_cast<const __half2 *>(&a), *reinterpret_cast<const __half2 *>(&b));
        return *reinterpret_cast<const uint32_t *>(&m);
    } else {
        const __nv_bfloat162 m = __hmax2(*reinterpret_cast<const __nv_bfloat162 *>(&a), *reinterpret_cast<const __nv_bfloat162 *>(&b));
        return *reinterpret_cast<const uint32_t *>(&m);
    }
}
// (code - 8) * scale of the codes in the low nibbles of both halves: the code is put behind the leading bits of 1024 (fp16) or 128
// (bf16), where a step is 1, so that the difference is exact; the product is rounded once.
template <typename T> __device__ __forceinline__ uint32_t decode2(uint32_t codes, uint32_t scale2)
{
    codes &= 0x000f000fu;
    if constexpr (std::is_same_v<T, f16_t>) {
        const uint32_t u = codes | 0x64006400u;
        const __half2 r = __hmul2_rn(__hsub2(*reinterpret_cast<const __half2 *>(&u), __float2half2_rn(1032.f)), *reinterpret_cast<const __half2 *>(&scale2));
        return *reinterpret_cast<const uint32_t *>(&r);
    } else {
        const uint32_t u = codes | 0x43004300u;
        const __nv_bfloat162 r = __hmul2_rn(__hsub2(*reinterpret_cast<const __nv_bfloat162 *>(&u), __float2bfloat162_rn(136.f)), *reinterpret_cast<const __nv_bfloat162 *>(&scale2));
        return *reinterpret_cast<const uint32_t *>(&r);
    }
}

// The tile in shared memory.  Pitches in elements: 8 more than the k puts the 16-byte vectors of eight columns into different banks,
// 66 the 2-byte accesses of lanes (g, t) at (column g, k = 8 t).
template <bool kColMajor, int kRows> struct Tile {
    static constexpr int kPitch = kColMajor ? kRows + 8 : kCols + 2;
    uint16_t v[(kColMajor ? kCols : kRows) * kPitch];
    __device__ __forceinline__ uint16_t &at(int r, int c) { return v[kColMajor ? c * kPitch + r : r * kPitch + c]; }
};

// Extents of the operands, for the debug build's checks.
[[maybe_unused]] __device__ __forceinline__ Span span_of_weights(const void *B, int N, int K) { return make_span(B, 2 * (size_t)N * K); }
[[maybe_unused]] __device__ __forceinline__ Span span_of_codes(const void *packed, int nb, int kb) { return make_span(packed, (size_t)nb * kb * kW4BlockBytes); }
[[maybe_unused]] __device__ __forceinline__ Span span_of_scales(const void *scales, int nb, int K, int group) { return make_span(scales, 2 * (size_t)((K + group - 1) / group) * nb * kW4Cols); }

// vec: every run of eight elements along the contiguous dimension starts on 16 bytes and ends inside the matrix
template <bool kColMajor, int kRows>
__device__ __forceinline__ void load_tile(Tile<kColMajor, kRows> &s, const uint16_t *__restrict__ B, int n0, int k0, int N, int K, bool vec, unsigned *status)
{
    constexpr int kInner = kColMajor ? kRows : kCols;
    if (vec) {
#pragma unroll 4
        for (int i = threadIdx.x; i < kCols * kRows / 8; i += kThreads) {
            const int in = (i % (kInner / 8)) * 8, out = i / (kInner / 8), c = kColMajor ? out : in, r = kColMajor ? in : out;
            const int n = n0 + c, k = k0 + r;
            uint4 u = make_uint4(0u, 0u, 0u, 0u);
            if (n < N && k < K) u = NM_LD_STREAM16(B + (kColMajor ? (long)n * K + k : (long)k * N + n), span_of_weights(B, N, K), status);
            uint32_t *d = reinterpret_cast<uint32_t *>(&s.at(r, c));
            if constexpr (kColMajor) *reinterpret_cast<uint4 *>(d) = u;
            else { d[0] = u.x; d[1] = u.y; d[2] = u.z; d[3] = u.w; }
        }
    } else {
        for (int i = threadIdx.x; i < kCols * kRows; i += kThreads) {
            const int in = i % kInner, out = i / kInner, c = kColMajor ? out : in, r = kColMajor ? in : out;
            const int n = n0 + c, k = k0 + r;
            s.at(r, c) = (n < N && k < K) ? NM_LD(&B[kColMajor ? (long)n * K + k : (long)k * N + n], span_of_weights(B, N, K), status) : (uint16_t)0;
        }
    }
}
template <bool kColMajor, int kRows>
__device__ __forceinline__ void store_tile(Tile<kColMajor, kRows> &s, uint16_t *__restrict__ B, int n0, int k0, int N, int K, bool vec, unsigned *status)
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
            NM_ST(reinterpret_cast<uint4 *>(B + (kColMajor ? (long)n * K + k : (long)k * N + n)), u, span_of_weights(B, N, K), status);
        }
    } else {
        for (int i = threadIdx.x; i < kCols * kRows; i += kThreads) {
            const int in = i % kInner, out = i / kInner, c = kColMajor ? out : in, r = kColMajor ? in : out;
            const int n = n0 + c, k = k0 + r;
            if (n < N && k < K) NM_ST(&B[kColMajor ? (long)n * K + k : (long)k * N + n], s.at(r, c), span_of_weights(B, N, K), status);
        }
    }
}

template <typename T, bool kColMajor, int kRows>
__global__ void __launch_bounds__(kThreads) w4_quantize_kernel(const uint16_t *__restrict__ B, uint4 *__restrict__ packed, uint16_t *__restrict__ scales, int N,
                                                               int K, int nb, int kb, int group, int vec, unsigned *status)
{
    __shared__ __align__(16) Tile<kColMajor, kRows> s_w;
    __shared__ float s_max[kRows / 32][kCols + 1];                 // per 32 k: the largest, then the rounded scale of its group
    const int tid = threadIdx.x, n0 = blockIdx.y * kCols, k0 = blockIdx.x * kRows;
    load_tile<kColMajor, kRows>(s_w, B, n0, k0, N, K, vec != 0, status);
    __syncthreads();
    for (int i = tid; i < (kColMajor ? kCols : kCols / 2) * (kRows / 32); i += kThreads) {
        // (pairs of columns along the lanes where columns are contiguous, 32-k pieces of a column otherwise)
        uint32_t m = 0u;
        if constexpr (kColMajor) {
            const int c = i / (kRows / 32), q = i % (kRows / 32);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const uint4 u = *reinterpret_cast<const uint4 *>(&s_w.at(32 * q + 8 * r, c));
                m = max_abs2<T>(max_abs2<T>(max_abs2<T>(max_abs2<T>(m, u.x), u.y), u.z), u.w);
            }
            s_max[q][c] = fmaxf(widen16<T>((uint16_t)m), widen16<T>((uint16_t)(m >> 16)));
        } else {
            const int c = 2 * (i % (kCols / 2)), q = i / (kCols / 2);
#pragma unroll 8
            for (int r = 0; r < 32; ++r) m = max_abs2<T>(m, *reinterpret_cast<const uint32_t *>(&s_w.at(32 * q + r, c)));
            s_max[q][c] = widen16<T>((uint16_t)m);
            s_max[q][c + 1] = widen16<T>((uint16_t)(m >> 16));
        }
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
            NM_ST(&scales[((long)(k0 / group + q) * nb + strip) * kW4Cols + 2 * (n % 8) + (n % kW4Cols) / 8], r.bits, span_of_scales(scales, nb, K, group), status);
    }
    __syncthreads();
    for (int i = tid; i < (kCols / kW4Cols) * (kRows / kW4Rows) * 32; i += kThreads) {
        const int lane = i % 32, blk = (i / 32) % (kRows / kW4Rows), st = i / (32 * (kRows / kW4Rows)), g = lane >> 2, t = lane & 3;
        const int strip = n0 / kW4Cols + st, kblk = k0 / kW4Rows + blk;
        if (strip >= nb || kblk >= kb) continue;
        // A quotient is rounded by adding 1.5 * 2^23 + 8, which leaves the code at the end of the sum's bits; the leading bits of the
        // eight sums of a word are taken off beforehand, all arithmetic being modulo 2^32.
        constexpr uint32_t kStart = 0u - 0x4b400000u * 0x11111111u;
        uint32_t w[4] = {kStart, kStart, kStart, kStart};
#pragma unroll
        for (int hi = 0; hi < 2; ++hi) {
            const int c = st * kW4Cols + g + 8 * hi;
#pragma unroll
            for (int h = 0; h < 2; ++h) {                          // words 2 h and 2 h + 1: eight consecutive k from 32 h + 8 t on
                const int r0 = blk * kW4Rows + 32 * h + 8 * t;
                const float sc = s_max[r0 / 32][c];
                float v[8];
                if constexpr (kColMajor) Elem<T>::unpack(*reinterpret_cast<const uint4 *>(&s_w.at(r0, c)), v);
                else
#pragma unroll
                    for (int x = 0; x < 8; ++x) v[x] = widen16<T>(s_w.at(r0 + x, c));
                // w / sc with one reciprocal for eight weights: a product, its exact error by a fused multiply-add, the corrected quotient
                // (Markstein, IBM J. Res. Dev. 34, 1990).  That is within 2^-23 of the quotient, and exact where fp32 holds it.  Quotients of two
                // numbers of a 16-bit type are ties, which fp32 holds, or at least 2^-15 of themselves away from one (all pairs of fp16
                // significands; 2^-11.9 for bf16), so the code is that of the rounded quotient.  (At the ends of fp32's range the
                // reciprocal or the error would leave it.)
                if (sc > 0x1p-60f && sc < 0x1p60f) {
                    const float inv = 1.f / sc;
#pragma unroll
                    for (int x = 0; x < 8; ++x) {
                        const float first = v[x] * inv;
                        v[x] = fmaf(fmaf(-first, sc, v[x]), inv, first);
                    }
                } else {
#pragma unroll
                    for (int x = 0; x < 8; ++x) v[x] = sc > 0.f ? (isinf(v[x]) ? v[x] : __fdiv_rn(v[x], sc)) : 0.f;      // (infinities keep their sign)
                }
#pragma unroll
                for (int x = 0; x < 8; ++x) {                      // k = r0 + 4 (j & 1) + 2 (b & 1) + (b >> 1)
                    const int j = 2 * h + (x >> 2), b = ((x >> 1) & 1) + 2 * (x & 1);
                    w[j] += __float_as_uint(fminf(fmaxf(v[x], -8.f), 7.f) + 12582920.f) << (8 * b + 4 * hi);
                }
            }
        }
        NM_ST(&packed[((long)strip * kb + kblk) * 32 + lane], make_uint4(w[0], w[1], w[2], w[3]), span_of_codes(packed, nb, kb), status);
    }
}

template <typename T, bool kColMajor, int kRows>
__global__ void __launch_bounds__(kThreads) w4_dequantize_kernel(const uint4 *__restrict__ packed, const uint16_t *__restrict__ scales, uint16_t *__restrict__ B,
                                                                 int N, int K, int nb, int kb, int group, int vec, unsigned *status)
{
    __shared__ __align__(16) Tile<kColMajor, kRows> s_w;
    const int tid = threadIdx.x, n0 = blockIdx.y * kCols, k0 = blockIdx.x * kRows;
    for (int i = tid; i < (kCols / kW4Cols) * (kRows / kW4Rows) * 32; i += kThreads) {
        const int lane = i % 32, blk = (i / 32) % (kRows / kW4Rows), st = i / (32 * (kRows / kW4Rows)), g = lane >> 2, t = lane & 3;
        const int strip = n0 / kW4Cols + st, kblk = k0 / kW4Rows + blk;
        if (strip >= nb || kblk >= kb) continue;
        const uint4 v = NM_LD_STREAM16(packed + ((long)strip * kb + kblk) * 32 + lane, span_of_codes(packed, nb, kb), status);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int r0 = blk * kW4Rows + 32 * h + 8 * t, k32 = k0 + r0 / 32 * 32;        // the codes of 32 k share their group
            const uint32_t pair = NM_LD(reinterpret_cast<const uint32_t *>(scales + ((long)(k32 < K ? k32 / group : 0) * nb + strip) * kW4Cols + 2 * g),
                                        span_of_scales(scales, nb, K, group), status);
#pragma unroll
            for (int hi = 0; hi < 2; ++hi) {
                const uint32_t sc = __byte_perm(pair, 0u, hi ? 0x3232 : 0x1010);
                const int c = st * kW4Cols + g + 8 * hi;
                uint32_t o[4];                                     // pairs of k: bytes b and b + 2 of a word
#pragma unroll
                for (int x = 0; x < 4; ++x) o[x] = decode2<T>(w[2 * h + (x >> 1)] >> (8 * (x & 1) + 4 * hi), sc);
                if constexpr (kColMajor) *reinterpret_cast<uint4 *>(&s_w.at(r0, c)) = make_uint4(o[0], o[1], o[2], o[3]);
                else
#pragma unroll
                    for (int x = 0; x < 8; ++x) s_w.at(r0 + x, c) = (uint16_t)(o[x / 2] >> (16 * (x & 1)));
            }
        }
    }
    __syncthreads();
    store_tile<kColMajor, kRows>(s_w, B, n0, k0, N, K, vec != 0, status);
}

// whether the contiguous dimension runs in whole, aligned 16-byte vectors
bool pack_vec(const void *B, int N, int K, int layout) { return !((uintptr_t)B & 15u) && (layout == NM_COL_MAJOR ? K : N) % 8 == 0; }

int check_pack(const void *B, const void *packed, const void *scales, int N, int K, int group, int dtype, int layout)
{
    if (!B || !packed || !scales || N < 1 || K < 1) return NM_ERR_INVALID_ARG;
    if (!w4_dtype_ok(dtype) || !w4_group_ok(group) || (layout != NM_ROW_MAJOR && layout != NM_COL_MAJOR)) return NM_ERR_UNSUPPORTED;
    if (((uintptr_t)B & 1u) || ((uintptr_t)packed & 15u) || ((uintptr_t)scales & 3u)) return NM_ERR_ALIGNMENT;
    if (((long)N + kCols - 1) / kCols > 65535 || K > (1 << 30)) return NM_ERR_UNSUPPORTED;       // the grid; k past the end of a tile stays an int
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
    auto go = [&](auto rows, auto kern) {
        const dim3 grid((unsigned)(((long)K + rows - 1) / rows), (unsigned)(((long)N + kCols - 1) / kCols));
        kern<<<grid, kThreads, 0, (cudaStream_t)stream>>>(static_cast<const uint16_t *>(B), static_cast<uint4 *>(packed), static_cast<uint16_t *>(scales), N, K, nb, kb, group, (int)pack_vec(B, N, K, layout_B), bounds_status_ptr());
    };
    auto by_rows = [&](auto t, auto col) {
        using T = decltype(t);
        constexpr bool kCol = decltype(col)::value;
        if (group <= 128) go(128, w4_quantize_kernel<T, kCol, 128>);
        else go(256, w4_quantize_kernel<T, kCol, 256>);
    };
    if (dtype == NM_F16) layout_B == NM_COL_MAJOR ? by_rows(f16_t{}, std::true_type{}) : by_rows(f16_t{}, std::false_type{});
    else layout_B == NM_COL_MAJOR ? by_rows(bf16_t{}, std::true_type{}) : by_rows(bf16_t{}, std::false_type{});
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? NM_OK : record_cuda_error(e, "4-bit quantisation launch");
}

int nm_w4_dequantize(const void *packed, const void *scales, void *B, int N, int K, int group, nm_dtype dtype, nm_layout layout_B, nm_stream stream)
{
    const int rc = check_pack(B, packed, scales, N, K, group, dtype, layout_B);
    if (rc != NM_OK) return rc;
    const int nb = (int)(((long)N + kW4Cols - 1) / kW4Cols), kb = (int)(((long)K + kW4Rows - 1) / kW4Rows);
    auto go = [&](auto rows, auto kern) {
        const dim3 grid((unsigned)(((long)K + rows - 1) / rows), (unsigned)(((long)N + kCols - 1) / kCols));
        kern<<<grid, kThreads, 0, (cudaStream_t)stream>>>(static_cast<const uint4 *>(packed), static_cast<const uint16_t *>(scales), static_cast<uint16_t *>(B), N, K, nb, kb, group, (int)pack_vec(B, N, K, layout_B), bounds_status_ptr());
    };
    auto by_rows = [&](auto t, auto col) {
        using T = decltype(t);
        constexpr bool kCol = decltype(col)::value;
        if (group <= 128) go(128, w4_dequantize_kernel<T, kCol, 128>);
        else go(256, w4_dequantize_kernel<T, kCol, 256>);
    };
    if (dtype == NM_F16) layout_B == NM_COL_MAJOR ? by_rows(f16_t{}, std::true_type{}) : by_rows(f16_t{}, std::false_type{});
    else layout_B == NM_COL_MAJOR ? by_rows(bf16_t{}, std::true_type{}) : by_rows(bf16_t{}, std::false_type{});
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? NM_OK : record_cuda_error(e, "4-bit dequantisation launch");
}

#pragma GCC visibility pop
}  // extern "C"
