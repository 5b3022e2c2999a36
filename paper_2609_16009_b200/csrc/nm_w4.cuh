// Shared by the kernels on 4-bit weights (nm_w4.cu, nm_w4_pack.cu).
//
// Storage.  The codes of 16 columns n x 64 k form a block of 512 bytes, one 16-byte vector per lane of a warp; the blocks of a
// 16-column strip lie behind each other along k.  Lane 4 g + t holds, in byte b of its word j, the codes of column g (low
// nibble) and column g + 8 (high nibble) at k = 32 (j >> 1) + 8 t + 4 (j & 1) + 2 (b & 1) + (b >> 1): with the mask
// 0x000f000f of the word shifted by 0, 4, 8 and 12 that is exactly the four registers of the weight operand of
// mma.m16n8k16 (rows g and g + 8, two pairs of k), and over the lanes t = 0..3 of a row eight consecutive k each - so the token
// operand is 16 consecutive bytes of a token row.  No shuffle, no shared memory between HBM and the matrix unit.
// Scales: [group of k][strip][g][2], the pair being columns g and g + 8 - one 4-byte load per lane.
#pragma once

#include "nm_common.cuh"

namespace nm {

constexpr int kW4Cols = 16, kW4Rows = 64;          // columns and k of a block
constexpr int kW4BlockBytes = kW4Cols * kW4Rows / 2;

inline bool w4_group_ok(int group) { return group == 32 || group == 64 || group == 128 || group == 256; }
inline bool w4_dtype_ok(int dtype) { return dtype == NM_BF16 || dtype == NM_BF16_F32OUT || dtype == NM_F16; }

}  // namespace nm
