// Activation checkpoints in 8 bits: e4m3 codes with a power-of-two scale for
// every 32 consecutive values of a row.
//
// Both directions are one pass bound by memory: 2 + 1 + 1/32 bytes a bf16 value.
// 409 million values are packed in 251 us and restored in 208, 4.9 and 5.9 TB/s
// (a copy of 1 GiB: 5.1); 16.8 million of a stage in 11 and 10 us.
// Four lanes hold a group, eight values each, so a group's largest magnitude
// takes two exchanges between lanes and no LDS. A power of two makes the scaling
// itself exact: the only rounding is the code's (four significant bits, half a
// step 2^-4 of the value).
#include "kernels.hpp"

namespace spx {
namespace {

constexpr int NT = 256, PER = 8, LANES = CHECKPOINT_GROUP / PER;

__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float(static_cast<uint32_t>(e + 127) << 23); }

struct Place {
  long row, col;   // first value of the lane's eight
  int n;           // of them inside the row
  bool live;
};

struct Job : CheckpointArgs {
  long total = 0;          // groups of the tensor
  FastDiv groups;          // of a row
  unsigned first = 0;      // its first block
};
struct Jobs {
  Job job[CHECKPOINT_MAX];
  int n = 0;
};

// The block's tensor: blocks are dealt to the tensors in order.
__device__ __forceinline__ const Job& my_job(const Jobs& jobs) {
  int j = 0;
  while (j + 1 < jobs.n && blockIdx.x >= jobs.job[j + 1].first) ++j;
  return jobs.job[j];
}

__device__ __forceinline__ Place place(const Job& a) {
  const long unit = static_cast<long>(blockIdx.x - a.first) * NT + threadIdx.x, g = unit / LANES;
  const bool live = g < a.total;
  const uint32_t gi = live ? static_cast<uint32_t>(g) : 0u, row = a.groups.div(gi);
  Place p;
  p.row = row;
  p.col = static_cast<long>(gi - row * a.groups.d) * CHECKPOINT_GROUP + (threadIdx.x % LANES) * PER;
  p.n = static_cast<int>(min(max(a.cols - p.col, 0L), static_cast<long>(PER)));
  p.live = live;
  return p;
}

template <typename T>
__device__ __forceinline__ float to_float(T v) {
  if constexpr (sizeof(T) == 2) return bf16_to_f32(v);
  else return v;
}

// WIDE: every lane's eight values are whole and 16-byte aligned.
template <typename T, bool WIDE>
__global__ __launch_bounds__(NT) void checkpoint_pack_kernel(Jobs jobs) {
  const Job& a = my_job(jobs);
  const Place p = place(a);
  const T* x = static_cast<const T*>(a.x) + p.row * a.ld + p.col;
  float v[PER];
  uint4 raw = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
  for (int i = 0; i < PER; ++i) v[i] = 0.0f;
  if (WIDE) {
    if (p.live && p.n) {
      if constexpr (sizeof(T) == 2) {
        raw = *reinterpret_cast<const uint4*>(x);
        const u16x8_t u = __builtin_bit_cast(u16x8_t, raw);
#pragma unroll
        for (int i = 0; i < PER; ++i) v[i] = bf16_to_f32(u[i]);
      } else {
        const float4 u = *reinterpret_cast<const float4*>(x), w = *reinterpret_cast<const float4*>(x + 4);
        v[0] = u.x, v[1] = u.y, v[2] = u.z, v[3] = u.w, v[4] = w.x, v[5] = w.y, v[6] = w.z, v[7] = w.w;
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (p.live && i < p.n) v[i] = to_float(x[i]);
  }
  // bits of the largest magnitude, ordered as the values are
  uint32_t top = 0;
  if constexpr (WIDE && sizeof(T) == 2) {
    typedef uint16_t u16x2_t __attribute__((ext_vector_type(2)));
    const auto pair = [&](uint32_t w) { return __builtin_bit_cast(u16x2_t, w & 0x7fff7fffu); };
    const u16x2_t m = __builtin_elementwise_max(__builtin_elementwise_max(pair(raw.x), pair(raw.y)),
                                                __builtin_elementwise_max(pair(raw.z), pair(raw.w)));
    top = static_cast<uint32_t>(max(m[0], m[1])) << 16;
  } else {
#pragma unroll
    for (int i = 0; i < PER; ++i) top = max(top, __float_as_uint(v[i]) & 0x7fffffffu);
  }
  top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 1)));
  top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 2)));
  // smallest e with top / 2^e <= 448 = 1.75 * 2^8
  const auto exponent = [](uint32_t t) {
    return min(max(static_cast<int>(t >> 23) - 127 - 8 + ((t & 0x7fffffu) > 0x600000u), -117), 120);
  };
  int e = exponent(top);
  uint32_t word[2] = {0u, 0u};
  const auto convert = [&](const float (&z)[PER]) {
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      int c = __builtin_amdgcn_cvt_pk_fp8_f32(z[4 * w], z[4 * w + 1], 0, false);
      word[w] = static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(z[4 * w + 2], z[4 * w + 3], c, true));
    }
  };
  float z[PER];
  constexpr float LEAST = 1.0f / 512.0f;   // 2^-9: what is not zero becomes at least this
  if (!__any(e == 120)) {
    // no value that is not finite (its bits would make e 120), and none that
    // needs a limit: a third fewer vector instructions, which bounded the pass
    const float inv = power_of_two(-e);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const float m = fmaxf(fabsf(v[i] * inv), LEAST);
      z[i] = copysignf(v[i] == 0.0f ? 0.0f : m, v[i]);
    }
  } else {
    uint32_t finite = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const uint32_t m = __float_as_uint(v[i]) & 0x7fffffffu;
      if (m < 0x7f800000u) finite = max(finite, m);
    }
    finite = max(finite, static_cast<uint32_t>(__shfl_xor(static_cast<int>(finite), 1)));
    finite = max(finite, static_cast<uint32_t>(__shfl_xor(static_cast<int>(finite), 2)));
    e = exponent(finite);
    const float inv = power_of_two(-e), limit = e == 120 ? 240.0f : 448.0f;   // 256 * 2^120 would be infinite
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const float m = fminf(fmaxf(fabsf(v[i] * inv), LEAST), limit);
      const float y = copysignf(v[i] == 0.0f ? 0.0f : m, v[i]);
      z[i] = (__float_as_uint(v[i]) & 0x7fffffffu) < 0x7f800000u ? y : __uint_as_float(0x7fc00000u);
    }
  }
  convert(z);
  if (!p.live) return;
  uint8_t* out = a.codes + p.row * a.cols + p.col;
  if (WIDE) {
    if (p.n) *reinterpret_cast<uint2*>(out) = make_uint2(word[0], word[1]);
  } else {
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (i < p.n) out[i] = static_cast<uint8_t>(word[i / 4] >> (8 * (i % 4)));
  }
  if (threadIdx.x % LANES == 0)
    a.scales[p.row * a.groups.d + p.col / CHECKPOINT_GROUP] = static_cast<uint8_t>(e + 127);
}

template <typename T, bool WIDE>
__global__ __launch_bounds__(NT) void checkpoint_restore_kernel(Jobs jobs) {
  const Job& a = my_job(jobs);
  const Place p = place(a);
  if (!p.live || p.n == 0) return;
  const uint8_t* codes = a.codes + p.row * a.cols + p.col;
  const float scale =
      __uint_as_float(static_cast<uint32_t>(a.scales[p.row * a.groups.d + p.col / CHECKPOINT_GROUP]) << 23);
  uint32_t word[2] = {0u, 0u};
  if (WIDE) {
    const uint2 u = *reinterpret_cast<const uint2*>(codes);
    word[0] = u.x, word[1] = u.y;
  } else {
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (i < p.n) word[i / 4] |= static_cast<uint32_t>(codes[i]) << (8 * (i % 4));
  }
  float v[PER];
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    const f32x2_t lo = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(word[w]), false);
    const f32x2_t hi = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(word[w]), true);
    v[4 * w] = lo[0] * scale;
    v[4 * w + 1] = lo[1] * scale;
    v[4 * w + 2] = hi[0] * scale;
    v[4 * w + 3] = hi[1] * scale;
  }
  T* out = static_cast<T*>(a.out) + p.row * a.ld + p.col;
  if (WIDE) {
    if constexpr (sizeof(T) == 2) {
      *reinterpret_cast<uint4*>(out) = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]),
                                                  pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
    } else {
      *reinterpret_cast<float4*>(out) = make_float4(v[0], v[1], v[2], v[3]);
      *reinterpret_cast<float4*>(out + 4) = make_float4(v[4], v[5], v[6], v[7]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      if (i >= p.n) continue;
      if constexpr (sizeof(T) == 2) out[i] = f32_to_bf16(v[i]);
      else out[i] = v[i];
    }
  }
}

bool wide(const CheckpointArgs& a, const void* t) {
  return a.cols % PER == 0 && a.ld % PER == 0 && reinterpret_cast<uintptr_t>(t) % 16 == 0 &&
         reinterpret_cast<uintptr_t>(a.codes) % 8 == 0;
}

// WIDE only where every tensor allows it.
template <typename K>
hipError_t launch(K* wide_kernel, K* plain_kernel, const CheckpointArgs* a, int n, hipStream_t s) {
  if (n < 1 || n > CHECKPOINT_MAX) return hipErrorInvalidValue;
  Jobs jobs;
  jobs.n = n;
  long blocks = 0;
  bool w = true;
  for (int i = 0; i < n; ++i) {
    Job& j = jobs.job[i];
    static_cast<CheckpointArgs&>(j) = a[i];
    j.groups = FastDiv(static_cast<uint32_t>((a[i].cols + CHECKPOINT_GROUP - 1) / CHECKPOINT_GROUP));
    j.total = a[i].rows * j.groups.d;
    j.first = static_cast<unsigned>(blocks);
    blocks += (j.total * LANES + NT - 1) / NT;
    w = w && wide(a[i], a[i].x ? a[i].x : a[i].out);
  }
  if (blocks >= 1L << 24) return hipErrorInvalidValue;   // grids of up to 2^32 - 1 threads
  hipLaunchKernelGGL(w ? wide_kernel : plain_kernel, dim3(static_cast<unsigned>(blocks)), dim3(NT), 0, s, jobs);
  return hipGetLastError();
}

}  // namespace

hipError_t checkpoint_pack(const CheckpointArgs* a, int n, int dtype, hipStream_t s) {
  if (dtype) return launch(checkpoint_pack_kernel<bf16_t, true>, checkpoint_pack_kernel<bf16_t, false>, a, n, s);
  return launch(checkpoint_pack_kernel<float, true>, checkpoint_pack_kernel<float, false>, a, n, s);
}

hipError_t checkpoint_restore(const CheckpointArgs* a, int n, int dtype, hipStream_t s) {
  if (dtype) return launch(checkpoint_restore_kernel<bf16_t, true>, checkpoint_restore_kernel<bf16_t, false>, a, n, s);
  return launch(checkpoint_restore_kernel<float, true>, checkpoint_restore_kernel<float, false>, a, n, s);
}

}  // namespace spx
