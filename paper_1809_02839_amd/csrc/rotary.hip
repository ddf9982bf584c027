// Rotary positions: each pair (a, b) of a head turned by position * frequency.
//
// Bound by reading and writing x once. The turn of a (token, pair) is shared by
// every head, so a block first forms the cosines and sines of its few tokens in
// LDS and then streams the heads. The angle is position * turns of a full turn
// in float64, reduced to its fraction before it becomes a float: in float32 a
// position of a million would be off by 0.06 radians. Forming it per head
// instead would take 500 instructions for every 32 bytes moved. 671 MB of float32
// heads take 123 us, 5.4 TB/s (a copy of 1 GiB: 5.1); the queries and keys of 8192
// tokens inside their packed projection, 34 MB, 7.7 us.
#include "kernels.hpp"

namespace spx {
namespace {

constexpr int NT = 256, MAX_TOKENS = 8;   // a block's tokens; their turns fit 8 KB of LDS

template <typename T, int VEC>
struct Pack {
  float v[VEC];
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (sizeof(T) == 4) {
      if constexpr (VEC == 4) {
        const float4 u = *reinterpret_cast<const float4*>(p);
        v[0] = u.x, v[1] = u.y, v[2] = u.z, v[3] = u.w;
      } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[i] = p[i];
      }
    } else if constexpr (VEC == 8) {
      const u16x8_t u = *reinterpret_cast<const u16x8_t*>(p);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = bf16_to_f32(u[i]);
    } else {
#pragma unroll
      for (int i = 0; i < VEC; ++i) v[i] = bf16_to_f32(p[i]);
    }
  }
  __device__ __forceinline__ void store(T* p) const {
    if constexpr (sizeof(T) == 4) {
      if constexpr (VEC == 4) {
        *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
      } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i) p[i] = v[i];
      }
    } else if constexpr (VEC == 8) {
      *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]),
                                                pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
    } else {
#pragma unroll
      for (int i = 0; i < VEC; ++i) p[i] = f32_to_bf16(v[i]);
    }
  }
};

// VEC: values of one access (16 bytes, or single values where a stride, an
// address or the pair count does not allow that). Interleaved, VEC values are
// VEC / 2 whole pairs (VEC == 1: one pair, two single accesses).
template <typename T, int VEC, bool INTERLEAVED>
__global__ __launch_bounds__(NT) void rotary_kernel(RotaryArgs a, int per_block, FastDiv units, FastDiv per_head,
                                                    int turned, int heads_per_block) {
  __shared__ __attribute__((aligned(16))) float cs[MAX_TOKENS * 128], sn[MAX_TOKENS * 128];
  const int half = a.rot / 2, row0 = blockIdx.x * per_block, rows = min(per_block, a.rows - row0);
  for (int e = threadIdx.x; e < rows * half; e += NT) {
    const int t = e / half, i = e - t * half, row = row0 + t;
    const int pos = a.positions ? a.positions[row] : row % a.tokens;
    double turn = (pos + a.first) * a.turns[i];   // the sum may pass 32 bits
    turn -= rint(turn);
    float s, c;
    sincospif(2.0f * static_cast<float>(turn), &s, &c);
    cs[e] = c * a.magnitude;
    sn[e] = s * a.magnitude * a.sign;
  }
  __syncthreads();
  // a unit: one access of one head of one token, turned ones first
  const int h0 = blockIdx.y * heads_per_block, heads = min(heads_per_block, a.heads - h0);
  const int total = rows * heads * static_cast<int>(per_head.d);
  const bool full = heads == heads_per_block;
  for (int u = threadIdx.x; u < total; u += NT) {
    const int t = full ? units.div(u) : u / (heads * static_cast<int>(per_head.d));
    const int w = u - t * heads * static_cast<int>(per_head.d);
    const int hh = per_head.div(w), j = w - hh * static_cast<int>(per_head.d), h = h0 + hh, row = row0 + t;
    const int b = row / a.tokens, tok = row - b * a.tokens;
    const T* x = static_cast<const T*>(a.x) + b * a.xb + tok * a.xt + h * a.xh;
    T* o = static_cast<T*>(a.out) + b * a.ob + tok * a.ot + h * a.oh;
    const float *c = cs + t * half, *s = sn + t * half;
    if (j >= turned) {   // past the turned part: copied
      Pack<T, VEC> v;
      const int at = a.rot + (j - turned) * VEC;
      v.load(x + at);
      v.store(o + at);
    } else if constexpr (!INTERLEAVED) {
      Pack<T, VEC> p, q;
      const int i = j * VEC;
      p.load(x + i);
      q.load(x + half + i);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const float u0 = p.v[e], u1 = q.v[e];
        p.v[e] = u0 * c[i + e] - u1 * s[i + e];
        q.v[e] = u0 * s[i + e] + u1 * c[i + e];
      }
      p.store(o + i);
      q.store(o + half + i);
    } else {
      constexpr int W = VEC < 2 ? 2 : VEC;
      Pack<T, W> p;
      const int i = j * (W / 2);
      p.load(x + 2 * i);
#pragma unroll
      for (int e = 0; e < W / 2; ++e) {
        const float u0 = p.v[2 * e], u1 = p.v[2 * e + 1];
        p.v[2 * e] = u0 * c[i + e] - u1 * s[i + e];
        p.v[2 * e + 1] = u0 * s[i + e] + u1 * c[i + e];
      }
      p.store(o + 2 * i);
    }
  }
}

template <typename T, int WIDE>
hipError_t launch(const RotaryArgs& a, hipStream_t s) {
  const auto by = [](long v) { return v % WIDE == 0; };
  bool wide = by(a.xb) && by(a.xt) && by(a.xh) && by(a.ob) && by(a.ot) && by(a.oh) && by(a.dim) && by(a.rot) &&
              reinterpret_cast<uintptr_t>(a.x) % 16 == 0 && reinterpret_cast<uintptr_t>(a.out) % 16 == 0;
  if (!a.interleaved) wide = wide && by(a.rot / 2);
  const int vec = wide ? WIDE : 1;
  const int turned = a.interleaved ? a.rot / (wide ? WIDE : 2) : a.rot / 2 / vec;
  const int copied = a.x == a.out ? 0 : (a.dim - a.rot) / vec;
  // About a thousand accesses a block: enough to cover the turns' cost and the
  // load latency; few tokens of many heads are spread over blocks by heads.
  int per_block = 1, heads_per_block = a.heads;
  while (per_block < MAX_TOKENS && 2L * per_block * a.heads * (turned + copied) <= 4 * NT) per_block *= 2;
  while (heads_per_block > 1 && static_cast<long>(heads_per_block) * (turned + copied) > 4 * NT)
    heads_per_block = (heads_per_block + 1) / 2;
  const dim3 grid((a.rows + per_block - 1) / per_block, (a.heads + heads_per_block - 1) / heads_per_block);
  const FastDiv per_head(turned + copied), units(heads_per_block * (turned + copied));
  auto* kernel = a.interleaved ? (wide ? rotary_kernel<T, WIDE, true> : rotary_kernel<T, 1, true>)
                               : (wide ? rotary_kernel<T, WIDE, false> : rotary_kernel<T, 1, false>);
  hipLaunchKernelGGL(kernel, grid, dim3(NT), 0, s, a, per_block, units, per_head, turned, heads_per_block);
  return hipGetLastError();
}

}  // namespace

hipError_t rotary(const RotaryArgs& a, int dtype, hipStream_t s) {
  return dtype ? launch<bf16_t, 8>(a, s) : launch<float, 4>(a, s);
}

}  // namespace spx
