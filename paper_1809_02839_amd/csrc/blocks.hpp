// e4m3 codes with a power-of-two scale, on the device: what the kernels that
// write tensors in blocks of 128 share.
#pragma once

#include <algorithm>

#include "common.hpp"

namespace spx {

__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float(static_cast<uint32_t>(e + 127) << 23); }

__device__ __forceinline__ uint32_t magnitude_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// Magnitude bits as the block's maximum takes them: values that are not finite are no part of it.
__device__ __forceinline__ uint32_t finite_bits(float v) {
  const uint32_t m = magnitude_bits(v);
  return m < 0x7f800000u ? m : 0u;
}

// Smallest e in [-117, 120] with max <= 448 * 2^e, 448 = 1.75 * 2^8, from the
// bits of a finite maximum.
__device__ __forceinline__ int block_exponent(uint32_t top) {
  return min(max(static_cast<int>(top >> 23) - 127 - 8 + ((top & 0x7fffffu) > 0x600000u), -117), 120);
}

// Largest of a value over aligned groups of 16 lanes, by exchanges inside the
// group's row of lanes (no LDS): pairs, quads, halves, mirrored halves.
__device__ __forceinline__ uint32_t max16(uint32_t v) {
#define SPX_STEP(ctrl) v = max(v, static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(v), ctrl, 0xf, 0xf, true)))
  SPX_STEP(0xb1);    // quad_perm 1 0 3 2
  SPX_STEP(0x4e);    // quad_perm 2 3 0 1
  SPX_STEP(0x141);   // row_half_mirror
  SPX_STEP(0x140);   // row_mirror
#undef SPX_STEP
  return v;
}

// What a value is scaled to: v / 2^e, rounded by the conversion afterwards.
// Finite values past 240 would become infinite at e = 120, where 256 * 2^120 is
// no float; they are held at 240. Others: NaN.
__device__ __forceinline__ float block_scaled(float v, float inv, float limit) {
  const float z = fminf(fmaxf(v * inv, -limit), limit);
  return magnitude_bits(v) < 0x7f800000u ? z : __uint_as_float(0x7fc00000u);
}
__device__ __forceinline__ float block_limit(int e) { return e == 120 ? 240.0f : 448.0f; }

// Four codes, rounded to nearest, ties to even; z within +-448 or NaN.
__device__ __forceinline__ uint32_t e4m3x4(float a, float b, float c, float d) {
  const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true));
}

// Bytes that a tile of `rows` rows takes of a line of `lines` scale bytes, from byte
// `first` on: its rows', and none behind the multiple of 16 that ends the line (what
// lies there, up to the next line, may be another tensor's).
__host__ __device__ constexpr long tile_scale_bytes(long rows, long first, long lines) {
  return std::min(rows, (lines + 15) / 16 * 16 - first);
}

// Vectors at any element's address: rows need not start at multiples of 16 bytes.
typedef float f32x4u_t __attribute__((ext_vector_type(4), aligned(4)));
typedef uint16_t u16x8u_t __attribute__((ext_vector_type(8), aligned(2)));

// Eight consecutive values of a row of bf16 or float32, n of them there (the others 0).
template <typename T>
__device__ __forceinline__ void load8(const T* p, int n, float (&v)[8]) {
  if (n >= 8) {
    if constexpr (sizeof(T) == 2) {
      const u16x8_t u = *reinterpret_cast<const u16x8u_t*>(p);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = bf16_to_f32(u[i]);
    } else {
      const f32x4_t u = *reinterpret_cast<const f32x4u_t*>(p), w = *reinterpret_cast<const f32x4u_t*>(p + 4);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = u[i], v[4 + i] = w[i];
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      v[i] = 0.0f;
      if (i < n) {
        if constexpr (sizeof(T) == 2) v[i] = bf16_to_f32(p[i]);
        else v[i] = p[i];
      }
    }
  }
}

template <typename T>
__device__ __forceinline__ void store8(T* p, int n, const float (&v)[8]) {
  if (n >= 8) {
    if constexpr (sizeof(T) == 2) {
      typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
      typedef uint32_t u32x4u_t __attribute__((ext_vector_type(4), aligned(2)));
      const u32x4_t u = {pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
      *reinterpret_cast<u32x4u_t*>(p) = u;
    } else {
      *reinterpret_cast<f32x4u_t*>(p) = f32x4_t{v[0], v[1], v[2], v[3]};
      *reinterpret_cast<f32x4u_t*>(p + 4) = f32x4_t{v[4], v[5], v[6], v[7]};
    }
  } else {
#pragma unroll
    for (int i = 0; i < 7; ++i)
      if (i < n) {
        if constexpr (sizeof(T) == 2) p[i] = f32_to_bf16(v[i]);
        else p[i] = v[i];
      }
  }
}

// Eight code bytes of a line, n of them there (lines start at multiples of 16).
__device__ __forceinline__ void store_codes8(uint8_t* p, int n, uint32_t lo, uint32_t hi) {
  if (n >= 8) {
    *reinterpret_cast<uint2*>(p) = make_uint2(lo, hi);
  } else {
#pragma unroll
    for (int i = 0; i < 7; ++i)
      if (i < n) p[i] = static_cast<uint8_t>((i < 4 ? lo : hi) >> (8 * (i % 4)));
  }
}

}  // namespace spx
