// Tensors in blocks of 128: e4m3 codes with a power-of-two scale for 128 values
// of a row, or for a tile of 128 x 128, packed as they lie, transposed, or both.
//
// One pass, bound by memory: a thread block takes a tile of 128 x 128, which
// holds whole scales of every kind (rows, columns, the tile), so x is read once
// for both orientations. Thread (g, c) of 16 x 16 holds rows 8 g .. 8 g + 7 at
// columns 8 c .. 8 c + 7: a row's scale needs the 16 lanes of a row group, a
// column's the 16 threads of equal c, over LDS. The transposed codes turn in LDS
// (8 rows of a column are 8 consecutive bytes of a transposed line).
#include "blocks.hpp"
#include "kernels.hpp"

namespace spx {
namespace {

constexpr int NT = 256, TILE = BLOCK_COLS;
constexpr int PITCH = TILE + 16;   // bytes between transposed lines in LDS

template <typename T>
__global__ __launch_bounds__(NT) void blocks_pack_kernel(BlocksArgs a, uint32_t tiles_n) {
  __shared__ uint32_t tops[16][TILE];          // per row group: the columns' largest
  __shared__ uint8_t turned[TILE * PITCH];
  __shared__ int col_e[TILE];
  __shared__ uint32_t group_top[16];
  const int t = threadIdx.x, c = t & 15, g = t >> 4;
  const uint32_t tm = blockIdx.x / tiles_n, tn = blockIdx.x - tm * tiles_n;
  const long row0 = static_cast<long>(tm) * TILE, col0 = static_cast<long>(tn) * TILE;
  const int rows = static_cast<int>(min(a.rows - row0, static_cast<long>(TILE)));
  const int cols = static_cast<int>(min(a.cols - col0, static_cast<long>(TILE)));
  const int nc = min(max(cols - 8 * c, 0), 8);   // of the thread's columns
  const T* x = static_cast<const T*>(a.x) + (row0 + 8 * g) * a.ld + col0 + 8 * c;
  float v[8][8];
#pragma unroll
  for (int i = 0; i < 8; ++i) load8<T>(x + i * a.ld, 8 * g + i < rows ? nc : 0, v[i]);

  uint32_t row_top[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) m = max(m, finite_bits(v[i][j]));
    row_top[i] = max16(m);
  }
  int e_row[8], e_col[8];
  if (a.tiles) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, row_top[i]);
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
    for (int i = 0; i < 8; ++i) e_row[i] = block_exponent(row_top[i]);
    if (a.t_codes) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = max(m, finite_bits(v[i][j]));
        tops[g][8 * c + j] = m;
      }
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

  if (a.codes) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int r = 8 * g + i;
      if (r >= rows) break;
      const float inv = power_of_two(-e_row[i]), limit = block_limit(e_row[i]);
      float z[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) z[j] = block_scaled(v[i][j], inv, limit);
      store_codes8(a.codes + (row0 + r) * a.codes_ld + col0 + 8 * c, nc, e4m3x4(z[0], z[1], z[2], z[3]),
                   e4m3x4(z[4], z[5], z[6], z[7]));
      if (c == 0) a.scales[static_cast<long>(tn) * a.scales_ld + row0 + r] = static_cast<uint8_t>(e_row[i] + 127);
    }
  }
  if (!a.t_codes) return;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float inv = power_of_two(-e_col[j]), limit = block_limit(e_col[j]);
    float z[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) z[i] = block_scaled(v[i][j], inv, limit);
    *reinterpret_cast<uint2*>(turned + (8 * c + j) * PITCH + 8 * g) =
        make_uint2(e4m3x4(z[0], z[1], z[2], z[3]), e4m3x4(z[4], z[5], z[6], z[7]));
  }
  __syncthreads();
#pragma unroll
  for (int q = 0; q < TILE / 32; ++q) {
    const int line = 32 * q + (t >> 3), at = 16 * (t & 7);
    if (line >= cols || at >= rows) continue;
    uint8_t* out = a.t_codes + (col0 + line) * a.t_ld + row0 + at;
    const uint4 u = *reinterpret_cast<const uint4*>(turned + line * PITCH + at);
    if (at + 16 <= rows) {
      *reinterpret_cast<uint4*>(out) = u;
    } else {
      store_codes8(out, rows - at, u.x, u.y);
      store_codes8(out + 8, rows - at - 8, u.z, u.w);
    }
  }
  if (t < cols) a.t_scales[static_cast<long>(tm) * a.t_scales_ld + col0 + t] = static_cast<uint8_t>(col_e[t] + 127);
}

template <typename T>
__global__ __launch_bounds__(NT) void blocks_restore_kernel(BlocksArgs a, uint32_t tiles_n) {
  const int t = threadIdx.x, c = t & 15, g = t >> 4;
  const uint32_t tm = blockIdx.x / tiles_n, tn = blockIdx.x - tm * tiles_n;
  const long row0 = static_cast<long>(tm) * TILE + 8 * g, col = static_cast<long>(tn) * TILE + 8 * c;
  const int n = static_cast<int>(min(max(a.cols - col, 0L), 8L));
  if (n == 0) return;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const long r = row0 + i;
    if (r >= a.rows) break;
    const uint8_t* p = a.codes + r * a.codes_ld + col;
    uint32_t w[2] = {0u, 0u};
    if (n == 8) {
      const uint2 u = *reinterpret_cast<const uint2*>(p);
      w[0] = u.x, w[1] = u.y;
    } else {
#pragma unroll
      for (int j = 0; j < 7; ++j)
        if (j < n) w[j / 4] |= static_cast<uint32_t>(p[j]) << (8 * (j % 4));
    }
    const float scale = __uint_as_float(static_cast<uint32_t>(a.scales[tn * a.scales_ld + r]) << 23);
    float v[8];
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const f32x2_t lo = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w[q]), false);
      const f32x2_t hi = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w[q]), true);
      v[4 * q] = lo[0] * scale, v[4 * q + 1] = lo[1] * scale, v[4 * q + 2] = hi[0] * scale, v[4 * q + 3] = hi[1] * scale;
    }
    store8<T>(static_cast<T*>(a.out) + r * a.ld + col, n, v);
  }
}

template <typename K>
hipError_t launch(K* kernel, const BlocksArgs& a, hipStream_t s) {
  const long tm = (a.rows + TILE - 1) / TILE, tn = (a.cols + TILE - 1) / TILE;
  if (tm * tn > 1L << 23) return hipErrorInvalidValue;   // grids of up to 2^32 - 1 threads
  hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(tm * tn)), dim3(NT), 0, s, a, static_cast<uint32_t>(tn));
  return hipGetLastError();
}

}  // namespace

hipError_t blocks_pack(const BlocksArgs& a, int dtype, hipStream_t s) {
  return dtype ? launch(blocks_pack_kernel<bf16_t>, a, s) : launch(blocks_pack_kernel<float>, a, s);
}

hipError_t blocks_restore(const BlocksArgs& a, int dtype, hipStream_t s) {
  return dtype ? launch(blocks_restore_kernel<bf16_t>, a, s) : launch(blocks_restore_kernel<float>, a, s);
}

}  // namespace spx
