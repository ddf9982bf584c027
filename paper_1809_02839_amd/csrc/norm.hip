// Root-mean-square norm of rows with the addition of a residual, an output in
// 16 or 32 bits, in 8-bit blocks of 128, or both, and its gradients.
//
// Bound by memory: a row is read once, stays in the registers of the TPR threads
// that share it (V times eight columns each), and is written from there. The
// backward's rows do the same with dy and h, the next row's loads under way
// meanwhile; the weight gradient is summed by every thread for its own columns
// over the rows of its block, and the blocks' partial rows are added in order by a
// second launch (no atomics).
//
// The sum of squares, rstd and y before its rounding are formed in 64 bits: an
// 8-bit code steps by an eighth of the value, so a y that is off by a last bit of
// float32 next to such a border would show; memory hides the arithmetic.
//
// 16384 x 8192 bf16 with a residual: forward 199 us, backward 201, 5.4 and 5.3 TB/s
// (a copy of 1 GiB: 5.1); 8192 x 512 to 8 bits 9.4. The backward of rows
// past 8192 columns has no registers for them and the next and reads them a second
// time, from L2: 3.9 TB/s at 16384 columns, 1.9 at 32768, where what is left spills.
// Forwards of such rows: 4.5 TB/s at 16384 columns, 3.9 at 32768, which spill too.
#include <algorithm>
#include <type_traits>

#include "blocks.hpp"
#include "kernels.hpp"

namespace spx {
namespace {

constexpr int NT = 256;

typedef float f32x8_t __attribute__((ext_vector_type(8)));

// Sum over the TPR threads of a row, the same bits in each of them. part: LDS for one value a wave.
template <int TPR, typename F>
__device__ __forceinline__ F row_sum(F v, F* part) {
#pragma unroll
  for (int m = 1; m < 64; m *= 2) v += __shfl_xor(v, m);
  if constexpr (TPR > 64) {
    __syncthreads();   // the last sum's readers are done
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = part[0];
#pragma unroll
    for (int w = 1; w < TPR / 64; ++w) v += part[w];
  }
  return v;
}

__device__ __forceinline__ void load_weight(const RmsNormArgs& a, uint32_t col, int n, float (&w)[8]) {
  if (a.weight_dtype) load8<bf16_t>(static_cast<const bf16_t*>(a.weight) + col, n, w);
  else load8<float>(static_cast<const float*>(a.weight) + col, n, w);
}

template <typename T>
__device__ __forceinline__ float rounded(float v) {
  if constexpr (sizeof(T) == 2) return bf16_to_f32(f32_to_bf16(v));
  else return v;
}

// Eight values of a row as they lie in memory.
template <typename T>
struct Raw {
  typename std::conditional<sizeof(T) == 2, u16x8_t, f32x8_t>::type v;
  __device__ __forceinline__ void load(const T* p, int n) {
    if (n >= 8) {
      if constexpr (sizeof(T) == 2) {
        v = *reinterpret_cast<const u16x8u_t*>(p);
      } else {
        v = __builtin_shufflevector(f32x4_t(*reinterpret_cast<const f32x4u_t*>(p)), f32x4_t(*reinterpret_cast<const f32x4u_t*>(p + 4)),
                                    0, 1, 2, 3, 4, 5, 6, 7);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = i < n ? p[i] : T(0);
    }
  }
  __device__ __forceinline__ float operator[](int i) const {
    if constexpr (sizeof(T) == 2) return bf16_to_f32(v[i]);
    else return v[i];
  }
};

// 1 / sqrt(m): float32's, and one step of Newton's iteration in 64 bits. 0 where m passes
// float32. Below its normal numbers m loses bits in float32, more than one step
// brings back (1e-44: 1.4e-4): there 2^128 m is taken, and 2^64 put back.
__device__ __forceinline__ double inverse_root(double m) {
  const bool small = m < 0x1p-126;
  const double s = small ? m * 0x1p128 : m;
  const double r = 1.0f / sqrtf(static_cast<float>(s));
  const double q = r * (1.5 - 0.5 * s * r * r);
  return r == 0.0 ? 0.0 : small ? q * 0x1p64 : q;
}

constexpr int threads_of(int tpr) { return tpr > NT ? tpr : NT; }

template <typename T, typename Y, int TPR, int V>
__global__ __launch_bounds__(threads_of(TPR)) void rms_norm_fwd_kernel(RmsNormArgs a) {
  __shared__ double part[16];
  constexpr int ROWS = threads_of(TPR) / TPR;   // of a block
  const uint32_t t = threadIdx.x % TPR;
  const int group = __builtin_amdgcn_readfirstlane(threadIdx.x / TPR);   // a wave's row is one: its addresses stay scalar
  for (long row = static_cast<long>(blockIdx.x) * ROWS + group; row < a.rows;
       row += static_cast<long>(gridDim.x) * ROWS) {
    float h[V][8];
    Raw<T> x[V], res[V];
    const auto left = [&](int v) { return min(max(static_cast<int>(a.cols) - 8 * static_cast<int>(v * TPR + t), 0), 8); };
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const uint32_t col = 8u * (v * TPR + t);
      x[v].load(static_cast<const T*>(a.x) + row * a.x_ld + col, left(v));
      if (a.residual) res[v].load(static_cast<const T*>(a.residual) + row * a.residual_ld + col, left(v));
    }
    double sum = 0.0;
#pragma unroll
    for (int v = 0; v < V; ++v) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        h[v][i] = a.residual ? rounded<T>(x[v][i] + res[v][i]) : x[v][i];
        sum = fma(static_cast<double>(h[v][i]), static_cast<double>(h[v][i]), sum);
      }
      if (a.sum) store8<T>(static_cast<T*>(a.sum) + row * a.sum_ld + 8u * (v * TPR + t), left(v), h[v]);
    }
    sum = row_sum<TPR>(sum, part);
    const double r = inverse_root(sum / static_cast<double>(a.cols) + static_cast<double>(a.eps));
    if (a.rstd && t == 0) a.rstd[row] = static_cast<float>(r);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const uint32_t col = 8u * (v * TPR + t);
      const int n = left(v);
      float w[8];
      load_weight(a, col, n, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) h[v][i] = static_cast<float>(static_cast<double>(h[v][i]) * r * static_cast<double>(w[i]));
      if (a.y) store8<Y>(static_cast<Y*>(a.y) + row * a.y_ld + col, n, h[v]);
      if (a.codes) {   // 16 threads hold a block
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) top = max(top, i < n ? finite_bits(h[v][i]) : 0u);
        const int e = block_exponent(max16(top));
        const float inv = power_of_two(-e), limit = block_limit(e);
        float z[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] = block_scaled(h[v][i], inv, limit);
        store_codes8(a.codes + row * a.codes_ld + col, n, e4m3x4(z[0], z[1], z[2], z[3]), e4m3x4(z[4], z[5], z[6], z[7]));
        if (t % 16 == 0 && n > 0) a.scales[col / BLOCK_COLS * a.scales_ld + row] = static_cast<uint8_t>(e + 127);
      }
    }
  }
}

template <typename T, typename Y, int TPR, int V>
__global__ __launch_bounds__(threads_of(TPR)) void rms_norm_bwd_kernel(RmsNormArgs a) {
  __shared__ float part[16];
  constexpr int ROWS = threads_of(TPR) / TPR;
  const uint32_t t = threadIdx.x % TPR;
  const int group = __builtin_amdgcn_readfirstlane(threadIdx.x / TPR);
  const long step = static_cast<long>(gridDim.x) * ROWS;
  const auto left = [&](int v) { return min(max(static_cast<int>(a.cols) - 8 * static_cast<int>(v * TPR + t), 0), 8); };
  constexpr bool KEEP = TPR < 1024;   // the row, the next one and the weight in registers; else read twice, from L2 the second time
  float dw[V][8] = {}, kept[KEEP ? V : 1][8];
  if constexpr (KEEP) {
#pragma unroll
    for (int v = 0; v < V; ++v) load_weight(a, 8u * (v * TPR + t), left(v), kept[v]);
  }
  const auto weight = [&](int v, float (&w)[8]) {
    if constexpr (KEEP) {
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = kept[v][i];
    } else {
      load_weight(a, 8u * (v * TPR + t), left(v), w);
    }
  };
  struct Part {
    Raw<T> h, more;
    Raw<Y> dy;
  };
  const auto load = [&](Part& q, long row, int v, bool more) {
    const uint32_t col = 8u * (v * TPR + t);
    q.h.load(static_cast<const T*>(a.x) + row * a.sum_ld + col, left(v));
    q.dy.load(static_cast<const Y*>(a.dy) + row * a.dy_ld + col, left(v));
    if (more && a.dsum) q.more.load(static_cast<const T*>(a.dsum) + row * a.dsum_ld + col, left(v));
  };
  const auto load_row = [&](Part (&q)[KEEP ? V : 1], float& r, long row) {
    r = a.rstd[row];
#pragma unroll
    for (int v = 0; v < (KEEP ? V : 0); ++v) load(q[v], row, v, true);
  };
  const float count = static_cast<float>(a.cols);
  Part now[KEEP ? V : 1], next[KEEP ? V : 1];
  float r = 0.0f, r_next = 0.0f;
  long row = static_cast<long>(blockIdx.x) * ROWS + group;
  if (row < a.rows) load_row(now, r, row);
  for (; row < a.rows; row += step) {
    if (row + step < a.rows) load_row(next, r_next, row + step);
    float dot = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      Part& q = now[KEEP ? v : 0];
      if constexpr (!KEEP) load(q, row, v, false);
      float w[8];
      weight(v, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float z = q.h[i] * r, d = q.dy[i];
        dw[v][i] = fmaf(d, z, dw[v][i]);
        dot = fmaf(d * w[i], z, dot);
      }
    }
    const float mean = row_sum<TPR>(dot, part) / count;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      Part& q = now[KEEP ? v : 0];
      if constexpr (!KEEP) load(q, row, v, true);
      float d[8], w[8];
      weight(v, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float z = q.h[i] * r, u = q.dy[i] * w[i];
        d[i] = fmaf(r, fmaf(-z, mean, u), a.dsum ? q.more[i] : 0.0f);
      }
      store8<T>(static_cast<T*>(a.dx) + row * a.dx_ld + 8u * (v * TPR + t), left(v), d);
    }
#pragma unroll
    for (int v = 0; v < (KEEP ? V : 0); ++v) now[v] = next[v];
    r = r_next;
  }
  // a partial row of the block: [block][cols]; of several row groups first their sum, in order
  if constexpr (ROWS > 1) {
    __shared__ float groups[ROWS][V][TPR * 8];
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int i = 0; i < 8; ++i) groups[threadIdx.x / TPR][v][8 * t + i] = dw[v][i];
    __syncthreads();
    if (threadIdx.x >= TPR) return;
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float s = groups[0][v][8 * t + i];
#pragma unroll
        for (int g = 1; g < ROWS; ++g) s += groups[g][v][8 * t + i];
        dw[v][i] = s;
      }
  }
  float* ws = a.ws + blockIdx.x * a.cols;
#pragma unroll
  for (int v = 0; v < V; ++v) store8<float>(ws + 8u * (v * TPR + t), left(v), dw[v]);
}

// dweight[c] = the partial rows' sum, in order: 32 runs of rows, then those.
constexpr int SUM_COLS = 32, SUM_RUNS = 32;
__global__ __launch_bounds__(SUM_COLS * SUM_RUNS) void rms_norm_sum_kernel(const float* ws, float* out, long cols, int rows) {
  __shared__ float part[SUM_RUNS][SUM_COLS];
  const int c = threadIdx.x % SUM_COLS, run = threadIdx.x / SUM_COLS;
  const long col = static_cast<long>(blockIdx.x) * SUM_COLS + c;
  const int each = (rows + SUM_RUNS - 1) / SUM_RUNS, r1 = min((run + 1) * each, rows);
  float s = 0.0f;
  if (col < cols) {
#pragma unroll 8
    for (int r = run * each; r < r1; ++r) s += ws[r * cols + col];
  }
  part[run][c] = s;
  __syncthreads();
  if (run || col >= cols) return;
  s = part[0][c];
#pragma unroll
  for (int i = 1; i < SUM_RUNS; ++i) s += part[i][c];
  out[col] = s;
}

// Threads of a row and vectors of a thread. A wave to a row up to 1024 columns (16384
// rows of 1024: 24 us, with 256 threads 34), more threads past them (8192 of 2048: 24,
// with a wave 25; 256 of 2048: 3.4 and 5.1), and further on as few threads as hold the
// row: 8192 of 8192 in 512 threads 100 us, in 1024 161; of 4096 in 256 54, in 512 77. The
// backward holds five times a vector's registers for each and takes more threads:
// 4096 of 16384 in 1024 137, in 512 181.
struct Shape {
  int tpr, v;
};
Shape fwd_shape(long cols) {
  const long n = (cols + 7) / 8;
  if (n <= 64) return {64, 1};
  if (n <= 128) return {64, 2};
  if (n <= 256) return {256, 1};
  if (n <= 512) return {256, 2};
  if (n <= 1024) return {512, 2};
  if (n <= 2048) return {512, 4};
  return {1024, 4};
}
Shape bwd_shape(long cols) {
  const long n = (cols + 7) / 8;
  if (n <= 64) return {64, 1};
  if (n <= 128) return {64, 2};
  if (n <= 256) return {256, 1};
  if (n <= 512) return {256, 2};
  if (n <= 1024) return {512, 2};
  if (n <= 2048) return {1024, 2};
  return {1024, 4};
}
int rows_of_block(const Shape& s) { return s.tpr < NT ? NT / s.tpr : 1; }

// Blocks of a backward at most, each of which leaves a partial row: 65536 x 512 takes 53 us
// with 512, 83 with 256 and 56 with 1024; 8192 x 8192 109, 104 and 116; 8192 x 2048 30, 40 and 27.
constexpr long BWD_BLOCKS = 512;
long bwd_blocks(long rows, const Shape& s) {
  return std::max(1L, std::min((rows + 2 * rows_of_block(s) - 1) / (2 * rows_of_block(s)), BWD_BLOCKS));
}

template <typename T, typename Y>
hipError_t launch_fwd(const RmsNormArgs& a, hipStream_t s) {
  const Shape sh = fwd_shape(a.cols);
  const unsigned blocks = static_cast<unsigned>(std::min((a.rows + rows_of_block(sh) - 1) / rows_of_block(sh), 1L << 16));
#define SPX_CASE(TPR, V)                                                                                           \
  if (sh.tpr == TPR && sh.v == V) {                                                                                \
    hipLaunchKernelGGL((rms_norm_fwd_kernel<T, Y, TPR, V>), dim3(blocks), dim3(threads_of(TPR)), 0, s, a);         \
    return hipGetLastError();                                                                                      \
  }
  SPX_CASE(64, 1)
  SPX_CASE(64, 2)
  SPX_CASE(256, 1)
  SPX_CASE(256, 2)
  SPX_CASE(512, 2)
  SPX_CASE(512, 4)
  SPX_CASE(1024, 4)
#undef SPX_CASE
  return hipErrorInvalidValue;
}

template <typename T, typename Y>
hipError_t launch_bwd(const RmsNormArgs& a, hipStream_t s) {
  const Shape sh = bwd_shape(a.cols);
  const unsigned blocks = static_cast<unsigned>(bwd_blocks(a.rows, sh));
#define SPX_CASE(TPR, V)                                                                                           \
  if (sh.tpr == TPR && sh.v == V) {                                                                                \
    hipLaunchKernelGGL((rms_norm_bwd_kernel<T, Y, TPR, V>), dim3(blocks), dim3(threads_of(TPR)), 0, s, a);         \
    return hipGetLastError();                                                                                      \
  }
  SPX_CASE(64, 1)
  SPX_CASE(64, 2)
  SPX_CASE(256, 1)
  SPX_CASE(256, 2)
  SPX_CASE(512, 2)
  SPX_CASE(1024, 2)
  SPX_CASE(1024, 4)
#undef SPX_CASE
  return hipErrorInvalidValue;
}

}  // namespace

size_t rms_norm_ws_bytes(long rows, long cols) {
  return static_cast<size_t>(bwd_blocks(rows, bwd_shape(cols))) * cols * sizeof(float);
}

hipError_t rms_norm_fwd(const RmsNormArgs& a, hipStream_t s) {
  if (a.dtype) return launch_fwd<bf16_t, bf16_t>(a, s);
  return a.out_dtype ? launch_fwd<float, bf16_t>(a, s) : launch_fwd<float, float>(a, s);
}

hipError_t rms_norm_bwd(const RmsNormArgs& a, hipStream_t s) {
  if (a.rows) {   // of no rows no tensor is touched, and dweight is their sum, 0
    const hipError_t e = a.dtype       ? launch_bwd<bf16_t, bf16_t>(a, s)
                         : a.out_dtype ? launch_bwd<float, bf16_t>(a, s)
                                       : launch_bwd<float, float>(a, s);
    if (e != hipSuccess) return e;
  }
  const unsigned sums = static_cast<unsigned>((a.cols + SUM_COLS - 1) / SUM_COLS);
  hipLaunchKernelGGL(rms_norm_sum_kernel, dim3(sums), dim3(SUM_COLS * SUM_RUNS), 0, s, a.ws, a.dweight, a.cols,
                     a.rows ? static_cast<int>(bwd_blocks(a.rows, bwd_shape(a.cols))) : 0);
  return hipGetLastError();
}

}  // namespace spx
