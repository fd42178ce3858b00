// Device helpers of the decode-side kernels: 16-column MFMA and operands read straight from rows in memory.
#pragma once

#include "cosa_device.h"

namespace cosa {

typedef float f32x4_t __attribute__((ext_vector_type(4)));

// D (16 x 16, fp32) = A (16 x 32) B (32 x 16) + C, bf16: lane l supplies row / column l % 16 and k = 8 (l / 16)
// .. + 7; D row 4 (l / 16) + i, column l % 16 in register i.
__device__ __forceinline__ f32x4_t mfma16(const u32x4_t& a, const u32x4_t& b, const f32x4_t& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(a), as_bf16x8(b), c, 0, 0, 0);
}

// 16 bytes that a step reads once: not kept in the caches behind others that are read again. A kernel that only
// reads 4.3 GB: 6.13 TB/s with plain loads, 7.05 TB/s with these.
__device__ __forceinline__ u32x4_t ldg16_once(const void* p) {
  return __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(p));
}

// MFMA operands of 16 rows of 256 bf16 at `row(i)`, read once, for rows as lanes: operand c (32 columns) of lane (r, gq)
// is row r, columns 32 c + 8 gq .. + 7. Read that way, a load instruction would take half a line of 128 bytes of
// each row, and a line that is not kept would be fetched twice. So load (p, m) takes line m of rows 8 p + r % 8 (16
// bytes per lane, the third bit of the chunk in lane bit 3), and to_operands() exchanges lane bit 3 with p:
// two DPP moves for two registers.
struct RowOperands {
  static constexpr int kLines = 4;
  u32x4_t x[2 * kLines];

  template <class Row>
  __device__ __forceinline__ void load(int lane, Row&& row) {
    const int r = lane & 15, gq = lane >> 4;
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const uint16_t* a = row(8 * p + (r & 7)) + (r >> 3) * 32 + gq * 8;
#pragma unroll
      for (int m = 0; m < kLines; ++m) x[2 * m + p] = ldg16_once(a + m * 64);
    }
  }
  __device__ __forceinline__ void to_operands() {
#pragma unroll
    for (int m = 0; m < kLines; ++m)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int a = (int)x[2 * m][i], b = (int)x[2 * m + 1][i];
        // row_ror:8 within 16 lanes; lanes 8 .. 15 (banks 2, 3) of the first, 0 .. 7 of the second
        x[2 * m][i] = (uint32_t)__builtin_amdgcn_update_dpp(a, b, 0x128, 0xF, 0xC, false);
        x[2 * m + 1][i] = (uint32_t)__builtin_amdgcn_update_dpp(b, a, 0x128, 0xF, 0x3, false);
      }
  }
};

}  // namespace cosa
