// Product of two tensors in blocks of 128.
//
// A bf16 out is summed by v_mfma_scale_f32_32x32x64_f8f6f4, whose operands carry an
// e8m0 scale for 32 values of a row: a block's byte serves four of them, so
// scaling costs no instruction. That instruction adds eight products of
// consecutive k in fixed point, cut (towards zero) 2^-13 below the largest of
// them, and the eights in float32: measured on normal values 1.5e-5 of the result's
// norm at any k, 9e-5 where a column in a hundred is 20 times the others; a bf16
// rounding is 1.7e-3. A float32 out is not given away to that: its codes are
// turned to bf16 (exact, scale included) for v_mfma_f32_32x32x16_bf16 at half the
// rate.
#include "blocks.hpp"
#include "kernels.hpp"

namespace spx {
namespace {

typedef int i32x8_t __attribute__((ext_vector_type(8)));
typedef int i32x4_t __attribute__((ext_vector_type(4)));

constexpr int NT = 256;

// 32 codes of a row at k .. k + 31, zeros behind kend (a line's bytes up to the next multiple of 16 may be read).
__device__ __forceinline__ i32x8_t codes32(const uint8_t* line, long k, long kend) {
  i32x8_t v;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const long at = k + 16 * h;
    uint4 u = make_uint4(0u, 0u, 0u, 0u);
    if (at < kend) u = *reinterpret_cast<const uint4*>(line + at);
    const int n = static_cast<int>(min(max(kend - at, 0L), 16L));
    uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int keep = min(max(n - 4 * q, 0), 4);
      v[4 * h + q] = static_cast<int>(keep == 4 ? w[q] : w[q] & ((1u << (8 * keep)) - 1u));
    }
  }
  return v;
}

// Codes 8 q .. 8 q + 7 of a lane's 32 as bf16, times their block's scale.
__device__ __forceinline__ bf16x8_t widened(const i32x8_t& v, int q, float scale) {
  bf16x8_t r;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint32_t w = static_cast<uint32_t>(v[2 * q + h]);
    const bf16x2_t lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false);
    const bf16x2_t hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true);
    r[4 * h] = lo[0], r[4 * h + 1] = lo[1], r[4 * h + 2] = hi[0], r[4 * h + 3] = hi[1];
  }
  return r;
}

__device__ __forceinline__ void store(const ProductArgs& a, long i, long j, float v) {
  if (a.bias) v += a.bias_dtype ? bf16_to_f32(static_cast<const bf16_t*>(a.bias)[j]) : static_cast<const float*>(a.bias)[j];
  if (a.relu && v < 0.0f) v = 0.0f;
  if (a.mask) {
    const long at = i * a.mask_ld + j;
    const float m = a.out_dtype ? bf16_to_f32(static_cast<const bf16_t*>(a.mask)[at]) : static_cast<const float*>(a.mask)[at];
    if (!(m > 0.0f)) v = 0.0f;
  }
  const long at = i * a.out_ld + j;
  if (a.out_dtype) static_cast<bf16_t*>(a.out)[at] = f32_to_bf16(v);
  else static_cast<float*>(a.out)[at] = a.accumulate ? static_cast<float*>(a.out)[at] + v : v;
}

// A wave: 32 x 32 of the output; four of them in a block of 64 x 64.
template <bool EXACT>
__global__ __launch_bounds__(NT) void product_kernel(ProductArgs a, uint32_t tiles_n) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t tm = blockIdx.x / tiles_n, tn = blockIdx.x - tm * tiles_n;
  const long i0 = 64L * tm + 32 * (wave >> 1), j0 = 64L * tn + 32 * (wave & 1);
  const long ra = min(i0 + (lane & 31), a.m - 1), rb = min(j0 + (lane & 31), a.n - 1);
  const uint8_t *la = a.a + ra * a.a_ld, *lb = a.b + rb * a.b_ld;
  f32x16_t acc = {};
  for (long k = 0; k < a.k; k += 64) {
    const long kk = k + 32 * (lane >> 5);
    const i32x8_t va = codes32(la, kk, a.k), vb = codes32(lb, kk, a.k);
    const int sa = a.a_scales[(k >> 7) * a.a_scales_ld + ra], sb = a.b_scales[(k >> 7) * a.b_scales_ld + rb];
    if constexpr (EXACT) {
      const float fa = __uint_as_float(static_cast<uint32_t>(sa) << 23), fb = __uint_as_float(static_cast<uint32_t>(sb) << 23);
#pragma unroll
      for (int q = 0; q < 4; ++q)
        acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widened(va, q, fa), widened(vb, q, fb), acc, 0, 0, 0);
    } else {
      acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(va, vb, acc, 0, 0, 0, sa, 0, sb);
    }
  }
#pragma unroll
  for (int v = 0; v < 16; ++v) {
    const long i = i0 + 8 * (v >> 2) + 4 * (lane >> 5) + (v & 3), j = j0 + (lane & 31);
    if (i < a.m && j < a.n) store(a, i, j, acc[v]);
  }
}

}  // namespace

size_t product_ws_bytes(long, long, long) { return 0; }

hipError_t product(const ProductArgs& a, hipStream_t s) {
  const long tm = (a.m + 63) / 64, tn = (a.n + 63) / 64;
  if (tm * tn > 1L << 23) return hipErrorInvalidValue;
  hipLaunchKernelGGL(a.out_dtype ? product_kernel<false> : product_kernel<true>, dim3(static_cast<unsigned>(tm * tn)), dim3(NT), 0, s, a, static_cast<uint32_t>(tn));
  return hipGetLastError();
}

}  // namespace spx
