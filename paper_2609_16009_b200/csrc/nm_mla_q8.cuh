// Shared by the kernels on the quantised latent cache (nm_cache_q8.cu, nm_attn_q8.cu).
//
// Record of a cache row: kv_lora e4m3 codes | rope bf16 | one fp32 scale s = 2^e | 12 bytes of zeros;  row = s * (codes | bf16 part).
// One factor for both parts: dividing the bf16 part by a power of two is exact, and the scores of a row need one multiplication.
#pragma once

#include "nm_common.cuh"

namespace nm {

constexpr int kQ8MaxKv = 1024, kQ8MaxRope = 256;
constexpr int kQ8LeastExp = -32, kQ8MostExp = 32;  // of the scale: a latent beyond 448 * 2^32 saturates, zeros have s = 1
__host__ __device__ constexpr int q8_row_bytes(int kv_lora, int rope) { return kv_lora + 2 * rope + 16; }
inline bool q8_dims_ok(int kv_lora, int rope)
{
    return kv_lora >= 16 && kv_lora <= kQ8MaxKv && kv_lora % 16 == 0 && rope >= 0 && rope <= kQ8MaxRope && rope % 8 == 0;
}

}  // namespace nm
