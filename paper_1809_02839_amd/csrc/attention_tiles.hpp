// Matrix-instruction fragments of the attention kernels that keep scores in
// registers (attention_long.hip, attention_masked.hip).
#pragma once

#include "kernels.hpp"

namespace spx {
namespace {

typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4_t lds_s16x4_t;

__device__ __forceinline__ bf16x8_t gld8(const bf16_t* p) {
  return __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u16x8_t*>(p));
}
// 8 consecutive k of row `row` from an LDS tile [row][k] of pitch P.
template <int P>
__device__ __forceinline__ bf16x8_t frag_rows(const bf16_t* s, int row, int k) {
  return gld8(s + row * P + k);
}
// Operand for "row" m0 + lane % 32 from a tile stored [k][row], by two
// transposing reads (within a 16-lane group, lane i receives element i % 4 of
// the 8-byte chunk addressed by lane 4 q + i / 4, q < 4): the lanes of half h
// get k0 + 4 h + 0 .. 3 and k0 + 8 + 4 h + 0 .. 3, the k order of a score
// register group (see above).
template <int P>
__device__ __forceinline__ bf16x8_t frag_cols(const bf16_t* s, int m0, int k0, int lane) {
  const int g = lane >> 4, i = lane & 15;
  const bf16_t* p = s + (k0 + 4 * (g >> 1) + (i >> 2)) * P + m0 + 16 * (g & 1) + 4 * (i & 3);
  const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)(p));
  const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)(p + 8 * P));
  const u16x8_t v = {static_cast<uint16_t>(lo[0]), static_cast<uint16_t>(lo[1]), static_cast<uint16_t>(lo[2]),
                     static_cast<uint16_t>(lo[3]), static_cast<uint16_t>(hi[0]), static_cast<uint16_t>(hi[1]),
                     static_cast<uint16_t>(hi[2]), static_cast<uint16_t>(hi[3])};
  return __builtin_bit_cast(bf16x8_t, v);
}
__device__ __forceinline__ f32x16_t mfma(bf16x8_t b, bf16x8_t a, f32x16_t c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(b, a, c, 0, 0, 0);
}
template <int N>
__device__ __forceinline__ void zero(f32x16_t (&a)[N]) {
#pragma unroll
  for (int j = 0; j < N; ++j)
#pragma unroll
    for (int r = 0; r < 16; ++r) a[j][r] = 0.0f;
}
// Column of register r inside a 32-column group.
__device__ __forceinline__ int col_of(int r, int lane) { return 8 * (r >> 2) + 4 * (lane >> 5) + (r & 3); }

}  // namespace
}  // namespace spx
