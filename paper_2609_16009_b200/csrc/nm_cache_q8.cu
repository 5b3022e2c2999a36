// Rows of the latent cache quantised as they are written (RMSNorm of the latent part, RoPE of the key part, one power of two for the
// row, e4m3 codes), and read back to bf16.  Record: nm_mla_q8.cuh.
//
// One warp per row: the whole row lives in the warp's registers (16 values a lane at kv_lora = 512), its sum of squares (fp64, so that
// a code next to a tie falls where the definition puts it) and its largest value are warp reductions, and nothing is read or
// written twice.  Bound: 1152 bytes in and 656 out per row (reversed when read back), in runs of 16 bytes a lane.  Measured, 131072
// rows of 512 + 64 in random order: written in 78 us with norm and rotation (41 for the bytes; conversions, the fp64 sum and the rounding
// to odd bind it by issue), read back in 45 (36 for the bytes); 16 rows are written in 2.5 us.
// Four rows a CTA; eight take 9 % longer for the first, two 69 us to read back.
#include <cuda_fp8.h>

#include "nm_async.cuh"
#include "nm_mla_q8.cuh"

namespace nm {

namespace {

constexpr int kWarpsQ8 = 4;
constexpr int kMaxCall = 1 << 30;                  // rows of a call: their numbers stay an int in a CTA's last warp too

__device__ __forceinline__ float bf_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    return (uint32_t)__bfloat16_as_ushort(__float2bfloat16_rn(lo)) | ((uint32_t)__bfloat16_as_ushort(__float2bfloat16_rn(hi)) << 16);
}

// kVecs: 16-byte vectors of the latent part a lane holds at most (kv_lora <= 256 * kVecs)
template <int kVecs>
__global__ void __launch_bounds__(kWarpsQ8 * 32) cache_write_q8_kernel(const uint16_t *__restrict__ ckr, long stride, const uint16_t *__restrict__ gamma,
                                                                       const float *__restrict__ cos_sin, const int64_t *__restrict__ rows,
                                                                       unsigned char *__restrict__ cache, long n_cache_rows, int T, int kv, int rope, double inv_kv,
                                                                       float eps, unsigned *status)
{
    const Span in_rows = make_span(ckr, 2 * ((T - 1) * (size_t)stride + kv + rope)), in_cache = make_span(cache, (size_t)n_cache_rows * q8_row_bytes(kv, rope)),
               in_gamma = make_span(gamma, 2 * (size_t)kv), in_angles = make_span(cos_sin, 4 * (size_t)T * rope);
    (void)in_rows; (void)in_cache; (void)in_gamma; (void)in_angles; (void)status;      // (the debug build's)
    const int t = blockIdx.x * kWarpsQ8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    pdl_launch_dependents();
    if (t >= T) return;
    pdl_wait_prior_grids();
    const int64_t row = rows ? NM_LD(&rows[t], make_span(rows, 8 * (size_t)T), status) : t;
    if (row < 0 || row >= n_cache_rows) return;                    // a padding token, or no such row: written nowhere
    const uint16_t *x = ckr + (long)t * stride;
    const int vecs = kv / 8;
    // all that the row needs is asked for at once; the key part's first 64 values (all there are, mostly) among it
    uint4 weight[kVecs] = {};
    if (gamma) {
#pragma unroll
        for (int i = 0; i < kVecs; ++i)
            if (lane + 32 * i < vecs) weight[i] = NM_LDG16(reinterpret_cast<const uint4 *>(gamma + 8 * (lane + 32 * i)), in_gamma, status);
    }
    auto key_at = [&](int p) { return NM_LD(reinterpret_cast<const uint32_t *>(x + kv + 2 * p), in_rows, status); };
    auto angle_at = [&](int p) { return cos_sin ? NM_LD(reinterpret_cast<const float2 *>(cos_sin + (long)t * rope + 2 * p), in_angles, status) : make_float2(1.f, 0.f); };
    const bool has_key = lane < rope / 2;
    const uint32_t key0 = has_key ? key_at(lane) : 0u;
    const float2 angle0 = has_key ? angle_at(lane) : make_float2(1.f, 0.f);
    float y[kVecs][8];
    double squares = 0.;
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
        const int v = lane + 32 * i;
        uint4 u = make_uint4(0u, 0u, 0u, 0u);
        if (v < vecs) u = NM_LD(reinterpret_cast<const uint4 *>(x + 8 * v), in_rows, status);
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) { y[i][2 * j] = bf_lo(w[j]); y[i][2 * j + 1] = bf_hi(w[j]); }
        if (gamma) {
#pragma unroll
            for (int j = 0; j < 8; ++j) squares = fma((double)y[i][j], (double)y[i][j], squares);
        }
    }
    if (gamma) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) squares += __shfl_xor_sync(0xffffffffu, squares, o);
        // The normaliser in 64 bits, 2^-44 off at most, and used as two fp32 terms on the exact products x * gamma.  A code next to a tie of e4m3
        // falls wrongly by whatever the value is off, and a code is worth 2^-4 of it.
        const double mean = squares * inv_kv + (double)eps;
        double rd;
        if (mean > 0x1p-100 && mean < 0x1p100) {                   // from fp32's root by one Newton step, 2^-44 off
            const double r0 = (double)rsqrtf((float)mean);
            rd = fma(0.5 * r0, fma(-mean * r0, r0, 1.), r0);
        } else {
            // A row at an end of the range is brought to its middle by a power of two, or x * gamma, or the normaliser itself, leaves fp32
            // though y does not.
            const float shift = mean > 1. ? 0x1p-64f : 0x1p64f;
#pragma unroll
            for (int i = 0; i < kVecs; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) y[i][j] *= shift;
            rd = 1. / (sqrt(mean) * (double)shift);
        }
        const float r = (float)rd;
        float r_low = (float)(rd - (double)r);
        // y is rounded to odd: cut off, and its last bit set, so that what is left of a value beside a tie of e4m3, or beside 448 times a power of
        // two, stays on its side (rounded to fp32's nearest, 1.5 of 3 million land on a tie and fall wrongly from there).  Where r is an fp32 number
        // y may BE such a tie; where it has more bits, x * gamma * r has more than 24 too and is none.
        if (fabsf(r_low) <= 0x1p-40f * r) r_low = 0.f;
        const uint32_t odd = r_low != 0.f;
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
            const uint32_t w[4] = {weight[i].x, weight[i].y, weight[i].z, weight[i].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float a = y[i][2 * j] * bf_lo(w[j]), b = y[i][2 * j + 1] * bf_hi(w[j]);
                y[i][2 * j] = __uint_as_float(__float_as_uint(__fmaf_rz(a, r, a * r_low)) | odd);
                y[i][2 * j + 1] = __uint_as_float(__float_as_uint(__fmaf_rz(b, r, b * r_low)) | odd);
            }
        }
    }
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < kVecs; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(y[i][j]));      // (a NaN is passed over here and stays a NaN code)
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    // least e with top <= 448 * 2^e, 448 = 1.75 * 2^8
    int e = 0;
    if (top > 0x1p-149f) {                                         // (a zero's last bit may be set)
        const uint32_t b = __float_as_uint(top);
        e = (int)(b >> 23) - 127 - 8 + ((b & 0x7fffffu) > 0x600000u);
        e = min(max(e, kQ8LeastExp), kQ8MostExp);
    }
    const float inv = __uint_as_float((uint32_t)(127 - e) << 23), s = __uint_as_float((uint32_t)(127 + e) << 23);
    unsigned char *rec = cache + row * (long)q8_row_bytes(kv, rope);
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
        const int v = lane + 32 * i;
        if (v >= vecs) continue;
        uint32_t c[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(y[i][4 * j] * inv, y[i][4 * j + 1] * inv), __NV_SATFINITE, __NV_E4M3);
            const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(y[i][4 * j + 2] * inv, y[i][4 * j + 3] * inv), __NV_SATFINITE, __NV_E4M3);
            c[j] = lo | (hi << 16);
        }
        NM_ST(reinterpret_cast<uint2 *>(rec + 8 * v), make_uint2(c[0], c[1]), in_cache, status);
    }
    for (int p = lane; p < rope / 2; p += 32) {
        const uint32_t w = p == lane ? key0 : key_at(p);
        float a = bf_lo(w), b = bf_hi(w);
        if (cos_sin) {
            const float2 cs = p == lane ? angle0 : angle_at(p);
            const float ra = a * cs.x - b * cs.y, rb = a * cs.y + b * cs.x;
            a = ra; b = rb;
        }
        NM_ST(reinterpret_cast<uint32_t *>(rec + kv + 4 * p), pack_bf16(a * inv, b * inv), in_cache, status);
    }
    if (lane == 0) NM_ST(reinterpret_cast<float4 *>(rec + kv + 2 * rope), make_float4(s, 0.f, 0.f, 0.f), in_cache, status);
}

__global__ void __launch_bounds__(kWarpsQ8 * 32) cache_read_q8_kernel(const unsigned char *__restrict__ cache, long n_cache_rows, const int64_t *__restrict__ rows,
                                                                      uint16_t *__restrict__ out, long stride, int n, int kv, int rope, unsigned *status)
{
    const Span in_out = make_span(out, 2 * ((n - 1) * (size_t)stride + kv + rope)), in_cache = make_span(cache, (size_t)n_cache_rows * q8_row_bytes(kv, rope));
    (void)in_out; (void)in_cache; (void)status;                    // (the debug build's)
    const int i = blockIdx.x * kWarpsQ8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    pdl_launch_dependents();
    if (i >= n) return;
    pdl_wait_prior_grids();
    const int64_t row = rows ? NM_LD(&rows[i], make_span(rows, 8 * (size_t)n), status) : i;
    uint16_t *o = out + (long)i * stride;
    const bool there = row >= 0 && row < n_cache_rows;             // no such row: zeros
    const unsigned char *rec = cache + (there ? row : 0) * (long)q8_row_bytes(kv, rope);
    const float s = there ? NM_LD(reinterpret_cast<const float *>(rec + kv + 2 * rope), in_cache, status) : 0.f;
    for (int v = lane; v < kv / 16; v += 32) {
        uint4 r[2] = {};
        if (there) {
            const uint4 u = NM_LD(reinterpret_cast<const uint4 *>(rec + 16 * v), in_cache, status);
            const uint32_t w[4] = {u.x, u.y, u.z, u.w};
            uint32_t b[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w[j >> 1] >> (16 * (j & 1))), __NV_E4M3);
                const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&h));
                b[j] = pack_bf16(f.x * s, f.y * s);
            }
            r[0] = make_uint4(b[0], b[1], b[2], b[3]); r[1] = make_uint4(b[4], b[5], b[6], b[7]);
        }
        NM_ST(reinterpret_cast<uint4 *>(o + 16 * v), r[0], in_out, status);
        NM_ST(reinterpret_cast<uint4 *>(o + 16 * v + 8), r[1], in_out, status);
    }
    for (int v = lane; v < rope / 8; v += 32) {
        uint4 r = make_uint4(0u, 0u, 0u, 0u);
        if (there) {
            const uint4 u = NM_LD(reinterpret_cast<const uint4 *>(rec + kv + 16 * v), in_cache, status);
            r = make_uint4(pack_bf16(bf_lo(u.x) * s, bf_hi(u.x) * s), pack_bf16(bf_lo(u.y) * s, bf_hi(u.y) * s),
                           pack_bf16(bf_lo(u.z) * s, bf_hi(u.z) * s), pack_bf16(bf_lo(u.w) * s, bf_hi(u.w) * s));
        }
        NM_ST(reinterpret_cast<uint4 *>(o + kv + 8 * v), r, in_out, status);
    }
}

template <typename... Args>
cudaError_t launch_rows(void (*kern)(Args...), int rows, cudaStream_t stream, Args... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((rows + kWarpsQ8 - 1) / kWarpsQ8));
    cfg.blockDim = dim3(kWarpsQ8 * 32);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = programmatic_launch_enabled() ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kern, args...);
}

}  // namespace

}  // namespace nm

using namespace nm;

extern "C" {
#pragma GCC visibility push(default)

size_t nm_mla_q8_row_bytes(int kv_lora, int rope) { return q8_dims_ok(kv_lora, rope) ? (size_t)q8_row_bytes(kv_lora, rope) : 0; }

int nm_mla_cache_write_q8(const void *ckr, long ckr_stride, const void *gamma, const float *cos_sin, const int64_t *rows, void *cache,
                          long n_cache_rows, int T, int kv_lora, int rope, float eps, nm_stream stream)
{
    if (!ckr || !cache || T < 1 || T > kMaxCall || n_cache_rows < 1 || ckr_stride < (long)kv_lora + rope) return NM_ERR_INVALID_ARG;
    if (!q8_dims_ok(kv_lora, rope)) return NM_ERR_UNSUPPORTED;
    if (((uintptr_t)ckr & 15u) || ckr_stride % 8 || ((uintptr_t)cache & 15u) || ((uintptr_t)gamma & 15u) || ((uintptr_t)cos_sin & 7u) || ((uintptr_t)rows & 7u))
        return NM_ERR_ALIGNMENT;
    cudaStream_t s = (cudaStream_t)stream;
    const uint16_t *x = static_cast<const uint16_t *>(ckr), *gm = static_cast<const uint16_t *>(gamma);
    unsigned char *c = static_cast<unsigned char *>(cache);
    const cudaError_t e = kv_lora <= 512 ? launch_rows(cache_write_q8_kernel<2>, T, s, x, ckr_stride, gm, cos_sin, rows, c, n_cache_rows, T, kv_lora, rope, 1. / kv_lora, eps, bounds_status_ptr())
                                         : launch_rows(cache_write_q8_kernel<4>, T, s, x, ckr_stride, gm, cos_sin, rows, c, n_cache_rows, T, kv_lora, rope, 1. / kv_lora, eps, bounds_status_ptr());
    return e == cudaSuccess ? NM_OK : record_cuda_error(e, "quantised cache write launch");
}

int nm_mla_cache_read_q8(const void *cache, long n_cache_rows, const int64_t *rows, void *out, long out_stride, int n, int kv_lora, int rope,
                         nm_stream stream)
{
    if (!cache || !out || n < 1 || n > kMaxCall || n_cache_rows < 1 || out_stride < (long)kv_lora + rope) return NM_ERR_INVALID_ARG;
    if (!q8_dims_ok(kv_lora, rope)) return NM_ERR_UNSUPPORTED;
    if (((uintptr_t)cache & 15u) || ((uintptr_t)out & 15u) || out_stride % 8 || ((uintptr_t)rows & 7u)) return NM_ERR_ALIGNMENT;
    const cudaError_t e = launch_rows(cache_read_q8_kernel, n, (cudaStream_t)stream, static_cast<const unsigned char *>(cache), n_cache_rows, rows,
                                      static_cast<uint16_t *>(out), out_stride, n, kv_lora, rope, bounds_status_ptr());
    return e == cudaSuccess ? NM_OK : record_cuda_error(e, "quantised cache read launch");
}

#pragma GCC visibility pop
}  // extern "C"
