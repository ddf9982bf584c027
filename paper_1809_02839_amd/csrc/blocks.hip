// Tensors in blocks of 128: e4m3 codes with a power-of-two scale for 128 values
// of a row, or for a tile of 128 x 128, packed as they lie, transposed, or both.
//
// One pass, bound by memory: a thread block takes a tile of 128 x 128, which
// holds whole scales of every kind (rows, columns, the tile), so x is read once
// for both orientations. Thread (g, c) of 16 x 16 holds rows 8 g .. 8 g + 7 at
// columns 8 c .. 8 c + 7: a row's scale needs the 16 lanes of a row group, a
// column's the 16 threads of equal c, over LDS. The transposed codes turn in LDS
// (8 rows of a column are 8 consecutive bytes of a transposed line). Codes come from
// the conversions that scale (two values an instruction, straight from bf16) and
// maxima of bf16 pairs: with float arithmetic for each value the pass was bound by
// vector instructions (134 million values in both orientations 205 us, now 118, 4.5
// TB/s, as they lie alone 77, 5.3, transposed alone 97, 4.2; 409 million restored from
// either in 289, 4.2). A tensor of few tiles leaves CUs idle: 2048 x 512 is 64 blocks, 7 us.
// Transposed codes meet bank conflicts on their way into LDS, 11 to 32% of the busy cycles.
#include "blocks.hpp"
#include "kernels.hpp"

namespace spx {
namespace {

constexpr int NT = 256, TILE = BLOCK_COLS;
constexpr int PITCH = TILE + 16;   // bytes between transposed lines in LDS
constexpr uint32_t LIMITED = 0x7f600000u;   // bits of 448 * 2^119: past it a scale's codes are limited, or a value is not finite

typedef uint16_t u16x2_t __attribute__((ext_vector_type(2)));
typedef int16_t i16x2_t __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t max_pairs(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2_t, a), __builtin_bit_cast(u16x2_t, b)));
}

// Two values over 2^e (scale = 2^e) as codes, rounded to nearest, ties to even, into half `hi` of a word.
__device__ __forceinline__ uint32_t codes_of(uint32_t word, uint32_t pair, float scale, bool hi) {   // of bf16
  const i16x2_t old = __builtin_bit_cast(i16x2_t, word);
  const bf16x2_t v = __builtin_bit_cast(bf16x2_t, pair);
  return __builtin_bit_cast(uint32_t, hi ? __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(old, v, scale, true)
                                         : __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(old, v, scale, false));
}
__device__ __forceinline__ uint32_t codes_of(uint32_t word, float a, float b, float scale, bool hi) {
  const i16x2_t old = __builtin_bit_cast(i16x2_t, word);
  return __builtin_bit_cast(uint32_t, hi ? __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(old, a, b, scale, true)
                                         : __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(old, a, b, scale, false));
}

// A thread's 8 x 8 values of the tile, as they lie in memory.
template <typename T>
struct Values;
template <>
struct Values<bf16_t> {
  uint32_t w[8][4];
  __device__ __forceinline__ float at(int i, int j) const { return bf16_to_f32(static_cast<bf16_t>(w[i][j / 2] >> (16 * (j % 2)))); }
  __device__ __forceinline__ void load(int i, const bf16_t* p) {
    const u16x8_t u = *reinterpret_cast<const u16x8u_t*>(p);
    const uint4 q = __builtin_bit_cast(uint4, u);
    w[i][0] = q.x, w[i][1] = q.y, w[i][2] = q.z, w[i][3] = q.w;
  }
  __device__ __forceinline__ void load_part(int i, const bf16_t* p, int n) {
#pragma unroll
    for (int j = 0; j < 8; j += 2)
      w[i][j / 2] = (j < n ? p[j] : 0u) | ((j + 1 < n ? static_cast<uint32_t>(p[j + 1]) : 0u) << 16);
  }
  // bits of the largest magnitude of row i; of each column
  __device__ __forceinline__ uint32_t row_top(int i) const {
    uint32_t m = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q) m = max_pairs(m, w[i][q] & 0x7fff7fffu);
    return max(m << 16, m & 0xffff0000u);
  }
  __device__ __forceinline__ void col_tops(uint32_t (&top)[8]) const {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      uint32_t m = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) m = max_pairs(m, w[i][q] & 0x7fff7fffu);
      top[2 * q] = m << 16, top[2 * q + 1] = m & 0xffff0000u;
    }
  }
  __device__ __forceinline__ uint2 row_codes(int i, float scale) const {
    return make_uint2(codes_of(codes_of(0u, w[i][0], scale, false), w[i][1], scale, true),
                      codes_of(codes_of(0u, w[i][2], scale, false), w[i][3], scale, true));
  }
  __device__ __forceinline__ uint2 col_codes(int j, float scale) const {
    uint32_t r[2] = {0u, 0u};
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      const uint32_t pair = __builtin_amdgcn_perm(w[i + 1][j / 2], w[i][j / 2], j % 2 ? 0x07060302u : 0x05040100u);
      r[i / 4] = codes_of(r[i / 4], pair, scale, i % 4 != 0);
    }
    return make_uint2(r[0], r[1]);
  }
};
template <>
struct Values<float> {
  float v[8][8];
  __device__ __forceinline__ float at(int i, int j) const { return v[i][j]; }
  __device__ __forceinline__ void load(int i, const float* p) { load8(p, 8, v[i]); }
  __device__ __forceinline__ void load_part(int i, const float* p, int n) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[i][j] = j < n ? p[j] : 0.0f;
  }
  __device__ __forceinline__ uint32_t row_top(int i) const {
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) m = max(m, magnitude_bits(v[i][j]));
    return m;
  }
  __device__ __forceinline__ void col_tops(uint32_t (&top)[8]) const {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      top[j] = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) top[j] = max(top[j], magnitude_bits(v[i][j]));
    }
  }
  __device__ __forceinline__ uint2 row_codes(int i, float scale) const {
    return make_uint2(codes_of(codes_of(0u, v[i][0], v[i][1], scale, false), v[i][2], v[i][3], scale, true),
                      codes_of(codes_of(0u, v[i][4], v[i][5], scale, false), v[i][6], v[i][7], scale, true));
  }
  __device__ __forceinline__ uint2 col_codes(int j, float scale) const {
    return make_uint2(codes_of(codes_of(0u, v[0][j], v[1][j], scale, false), v[2][j], v[3][j], scale, true),
                      codes_of(codes_of(0u, v[4][j], v[5][j], scale, false), v[6][j], v[7][j], scale, true));
  }
};

// A block's tile: row by row of tiles; or (runs) each XCD, which blocks go round,
// takes a run of the order strip of eight tile rows, column, row, so that lines of
// memory which neighbours share, where a tensor's lines do not start at multiples of
// 128 bytes, meet in one L2. 50001 x 8184 bf16 packed in both orientations and
// restored from one: by rows 508 and 375 us, by runs 416 and 289; 16384 x 4096, where
// nothing is shared and the XCDs' runs start on the same memory channels, 55 and 33
// against 70 and 36.
struct Grid {
  uint32_t tiles_m, tiles_n;
  int runs;
};
__device__ __forceinline__ bool my_tile(const Grid& g, uint32_t& tm, uint32_t& tn) {
  const uint32_t total = g.tiles_m * g.tiles_n;
  if (!g.runs) {
    tm = blockIdx.x / g.tiles_n;
    tn = blockIdx.x - tm * g.tiles_n;
    return blockIdx.x < total;
  }
  const uint32_t each = (total + 7) >> 3, ord = (blockIdx.x & 7) * each + (blockIdx.x >> 3);
  if ((blockIdx.x >> 3) >= each || ord >= total) return false;
  const uint32_t strip = ord / (8 * g.tiles_n), in = ord - strip * 8 * g.tiles_n, high = min(8u, g.tiles_m - 8 * strip);
  tn = in / high;
  tm = 8 * strip + in - tn * high;
  return true;
}

template <typename T>
__global__ __launch_bounds__(NT) void blocks_pack_kernel(BlocksArgs a, Grid grid) {
  // the columns' largest by row group, then the transposed codes
  __shared__ __attribute__((aligned(16))) uint8_t room[TILE * PITCH];
  __shared__ int col_e[TILE];
  __shared__ uint32_t group_top[16];
  uint32_t(*const tops)[TILE] = reinterpret_cast<uint32_t(*)[TILE]>(room);
  static_assert(sizeof(room) >= 16 * TILE * 4, "the largest fit");
  const int t = threadIdx.x, c = t & 15, g = t >> 4;
  uint32_t tm, tn;
  if (!my_tile(grid, tm, tn)) return;
  const long row0 = static_cast<long>(tm) * TILE, col0 = static_cast<long>(tn) * TILE;
  const int rows = static_cast<int>(min(a.rows - row0, static_cast<long>(TILE)));
  const int cols = static_cast<int>(min(a.cols - col0, static_cast<long>(TILE)));
  const int nc = min(max(cols - 8 * c, 0), 8);   // of the thread's columns
  const T* x = static_cast<const T*>(a.x) + (row0 + 8 * g) * a.ld + col0 + 8 * c;
  Values<T> v;
  if (rows == TILE && cols == TILE) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v.load(i, x + i * a.ld);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v.load_part(i, x + i * a.ld, 8 * g + i < rows ? nc : 0);
  }

  uint32_t row_top[8], any = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) any = max(any, row_top[i] = v.row_top(i));
  // a block of values that are all finite, none that needs a limit, takes the short way
  const bool limited = __syncthreads_or(any > LIMITED);
  if (limited) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      row_top[i] = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) row_top[i] = max(row_top[i], finite_bits(v.at(i, j)));
    }
  }
  int e_row[8], e_col[8];
  if (a.tiles) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, row_top[i]);
    m = max16(m);
    if (c == 0) group_top[g] = m;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 16; ++i) m = max(m, group_top[i]);
    const int e = block_exponent(m);
#pragma unroll
    for (int i = 0; i < 8; ++i) e_row[i] = e_col[i] = e;
    if (t < TILE) col_e[t] = e;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) e_row[i] = block_exponent(max16(row_top[i]));
    if (a.t_codes) {
      uint32_t top[8];
      v.col_tops(top);
      if (limited) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          top[j] = 0;
#pragma unroll
          for (int i = 0; i < 8; ++i) top[j] = max(top[j], finite_bits(v.at(i, j)));
        }
      }
      *reinterpret_cast<uint4*>(&tops[g][8 * c]) = make_uint4(top[0], top[1], top[2], top[3]);
      *reinterpret_cast<uint4*>(&tops[g][8 * c + 4]) = make_uint4(top[4], top[5], top[6], top[7]);
      __syncthreads();
      if (t < TILE) {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) m = max(m, tops[i][t]);
        col_e[t] = block_exponent(m);
      }
      __syncthreads();
#pragma unroll
      for (int j = 0; j < 8; ++j) e_col[j] = col_e[8 * c + j];
    }
  }

  const auto slow_codes = [&](int e, auto&& value) {
    const float inv = power_of_two(-e), limit = block_limit(e);
    float z[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) z[q] = block_scaled(value(q), inv, limit);
    return make_uint2(e4m3x4(z[0], z[1], z[2], z[3]), e4m3x4(z[4], z[5], z[6], z[7]));
  };
  if (a.codes) {
    uint8_t* out = a.codes + (row0 + 8 * g) * a.codes_ld + col0 + 8 * c;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      uint2 u;
      if (limited) u = slow_codes(e_row[i], [&](int j) { return v.at(i, j); });
      else u = v.row_codes(i, power_of_two(e_row[i]));
      if (8 * g + i < rows) store_codes8(out + i * a.codes_ld, nc, u.x, u.y);
    }
    if (c == 0) {
      uint32_t lo = 0, hi = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        lo |= static_cast<uint32_t>(e_row[i] + 127) << (8 * i);
        hi |= static_cast<uint32_t>(e_row[4 + i] + 127) << (8 * i);
      }
      if (8 * g < rows) store_codes8(a.scales + static_cast<long>(tn) * a.scales_ld + row0 + 8 * g, min(rows - 8 * g, 8), lo, hi);
    }
  }
  if (!a.t_codes) return;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    uint2 u;
    if (limited) u = slow_codes(e_col[j], [&](int i) { return v.at(i, j); });
    else u = v.col_codes(j, power_of_two(e_col[j]));
    *reinterpret_cast<uint2*>(room + (8 * c + j) * PITCH + 8 * g) = u;
  }
  __syncthreads();
#pragma unroll
  for (int q = 0; q < TILE / 32; ++q) {
    const int line = 32 * q + (t >> 3), at = 16 * (t & 7);
    if (line >= cols || at >= rows) continue;
    uint8_t* out = a.t_codes + (col0 + line) * a.t_ld + row0 + at;
    const uint4 u = *reinterpret_cast<const uint4*>(room + line * PITCH + at);
    if (at + 16 <= rows) {
      *reinterpret_cast<uint4*>(out) = u;
    } else {
      store_codes8(out, rows - at, u.x, u.y);
      store_codes8(out + 8, rows - at - 8, u.z, u.w);
    }
  }
  if (t < cols) a.t_scales[static_cast<long>(tm) * a.t_scales_ld + col0 + t] = static_cast<uint8_t>(col_e[t] + 127);
}

// Thread (g, c) of 16 x 16: rows 8 g .. 8 g + 7 (whose scale bytes lie together) at columns 8 c .. 8 c + 7.
template <typename T>
__global__ __launch_bounds__(NT) void blocks_restore_kernel(BlocksArgs a, Grid grid) {
  const int t = threadIdx.x, c = t & 15, g = t >> 4;
  uint32_t tm, tn;
  if (!my_tile(grid, tm, tn)) return;
  const long row0 = static_cast<long>(tm) * TILE + 8 * g, col = static_cast<long>(tn) * TILE + 8 * c;
  const int n = static_cast<int>(min(max(a.cols - col, 0L), 8L)), rows = static_cast<int>(min(max(a.rows - row0, 0L), 8L));
  if (n == 0 || rows == 0) return;
  const uint8_t* p = a.codes + row0 * a.codes_ld + col;
  const uint8_t* s = a.scales + tn * a.scales_ld + row0;
  T* out = static_cast<T*>(a.out) + row0 * a.ld + col;
  const auto restore = [&](uint32_t lo, uint32_t hi, uint32_t byte, T* to) {
    const float scale = __uint_as_float(byte << 23);
    float v[8];
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const uint32_t w = q ? hi : lo;
      const f32x2_t a0 = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w), false);
      const f32x2_t a1 = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w), true);
      v[4 * q] = a0[0] * scale, v[4 * q + 1] = a0[1] * scale, v[4 * q + 2] = a1[0] * scale, v[4 * q + 3] = a1[1] * scale;
    }
    store8<T>(to, n, v);
  };
  if (n == 8 && rows == 8) {
    uint2 w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = *reinterpret_cast<const uint2*>(p + i * a.codes_ld);
    const uint2 e = *reinterpret_cast<const uint2*>(s);
#pragma unroll
    for (int i = 0; i < 8; ++i) restore(w[i].x, w[i].y, ((i < 4 ? e.x : e.y) >> (8 * (i % 4))) & 0xffu, out + i * a.ld);
    return;
  }
  for (int i = 0; i < rows; ++i) {
    uint32_t w[2] = {0u, 0u};
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < n) w[j / 4] |= static_cast<uint32_t>(p[i * a.codes_ld + j]) << (8 * (j % 4));
    restore(w[0], w[1], s[i], out + i * a.ld);
  }
}

// t: x or out
template <typename K>
hipError_t launch(K* kernel, const BlocksArgs& a, const void* t, int dtype, hipStream_t s) {
  const long tm = (a.rows + TILE - 1) / TILE, tn = (a.cols + TILE - 1) / TILE;
  if (tm * tn > 1L << 23) return hipErrorInvalidValue;   // grids of up to 2^32 - 1 threads
  Grid grid{static_cast<uint32_t>(tm), static_cast<uint32_t>(tn), 0};
  const auto shares = [](const void* p, long ld) { return p && (ld % 128 || reinterpret_cast<uintptr_t>(p) % 128); };
  grid.runs = shares(t, a.ld * (dtype ? 2 : 4)) || shares(a.codes, a.codes_ld) || shares(a.t_codes, a.t_ld);
  hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>((tm * tn + 7) / 8 * 8)), dim3(NT), 0, s, a, grid);
  return hipGetLastError();
}

}  // namespace

hipError_t blocks_pack(const BlocksArgs& a, int dtype, hipStream_t s) {
  return dtype ? launch(blocks_pack_kernel<bf16_t>, a, a.x, dtype, s) : launch(blocks_pack_kernel<float>, a, a.x, dtype, s);
}

hipError_t blocks_restore(const BlocksArgs& a, int dtype, hipStream_t s) {
  return dtype ? launch(blocks_restore_kernel<bf16_t>, a, a.out, dtype, s)
               : launch(blocks_restore_kernel<float>, a, a.out, dtype, s);
}

}  // namespace spx
