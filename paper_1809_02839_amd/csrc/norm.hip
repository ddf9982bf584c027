// Root-mean-square norm of rows with the addition of a residual, an output in
// 16 or 32 bits, in 8-bit blocks of 128, or both, and its gradients.
//
// Bound by memory: a row is read once, stays in the registers of the TPR threads
// that share it (V times eight columns each), and is written from there. The
// backward's rows do the same with dy and h; the weight gradient is summed by
// every thread for its own columns over the rows of its block, and the blocks'
// partial rows are added in order by a second launch (no atomics).
#include <algorithm>

#include "blocks.hpp"
#include "kernels.hpp"

namespace spx {
namespace {

constexpr int NT = 256;

// Sum over the TPR threads of a row, the same bits in each of them. part: LDS for one value a wave.
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float* part) {
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

__device__ __forceinline__ void load_weight(const RmsNormArgs& a, long col, int n, float (&w)[8]) {
  if (a.weight_dtype) load8<bf16_t>(static_cast<const bf16_t*>(a.weight) + col, n, w);
  else load8<float>(static_cast<const float*>(a.weight) + col, n, w);
}

template <typename T>
__device__ __forceinline__ float rounded(float v) {
  if constexpr (sizeof(T) == 2) return bf16_to_f32(f32_to_bf16(v));
  else return v;
}

template <typename T, typename Y, int TPR, int V>
__global__ __launch_bounds__(TPR > NT ? TPR : NT) void rms_norm_fwd_kernel(RmsNormArgs a) {
  __shared__ float part[16];
  constexpr int ROWS = TPR < NT ? NT / TPR : 1;   // of a block
  const int t = threadIdx.x % TPR;
  for (long row = static_cast<long>(blockIdx.x) * ROWS + threadIdx.x / TPR; row < a.rows;
       row += static_cast<long>(gridDim.x) * ROWS) {
    float h[V][8];
    float sum = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const long col = 8L * (v * TPR + t);
      const int n = static_cast<int>(min(max(a.cols - col, 0L), 8L));
      load8<T>(static_cast<const T*>(a.x) + row * a.x_ld + col, n, h[v]);
      if (a.residual) {
        float r[8];
        load8<T>(static_cast<const T*>(a.residual) + row * a.residual_ld + col, n, r);
#pragma unroll
        for (int i = 0; i < 8; ++i) h[v][i] = rounded<T>(h[v][i] + r[i]);
        if (a.sum) store8<T>(static_cast<T*>(a.sum) + row * a.sum_ld + col, n, h[v]);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) sum = fmaf(h[v][i], h[v][i], sum);
    }
    sum = row_sum<TPR>(sum, part);
    const float r = 1.0f / sqrtf(sum / static_cast<float>(a.cols) + a.eps);
    if (a.rstd && t == 0) a.rstd[row] = r;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const long col = 8L * (v * TPR + t);
      const int n = static_cast<int>(min(max(a.cols - col, 0L), 8L));
      float w[8];
      load_weight(a, col, n, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) h[v][i] = h[v][i] * r * w[i];
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
__global__ __launch_bounds__(TPR > NT ? TPR : NT) void rms_norm_bwd_kernel(RmsNormArgs a) {
  __shared__ float part[16];
  constexpr int ROWS = TPR < NT ? NT / TPR : 1;
  const int t = threadIdx.x % TPR;
  float dw[V][8];
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int i = 0; i < 8; ++i) dw[v][i] = 0.0f;
  const float count = static_cast<float>(a.cols);
  for (long row = static_cast<long>(blockIdx.x) * ROWS + threadIdx.x / TPR; row < a.rows;
       row += static_cast<long>(gridDim.x) * ROWS) {
    const float r = a.rstd[row];
    float u[V][8], z[V][8];
    float dot = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const long col = 8L * (v * TPR + t);
      const int n = static_cast<int>(min(max(a.cols - col, 0L), 8L));
      float w[8];
      load8<T>(static_cast<const T*>(a.x) + row * a.sum_ld + col, n, z[v]);
      load8<Y>(static_cast<const Y*>(a.dy) + row * a.dy_ld + col, n, u[v]);
      load_weight(a, col, n, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        z[v][i] *= r;
        dw[v][i] = fmaf(u[v][i], z[v][i], dw[v][i]);
        u[v][i] *= w[i];
        dot = fmaf(u[v][i], z[v][i], dot);
      }
    }
    const float mean = row_sum<TPR>(dot, part) / count;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const long col = 8L * (v * TPR + t);
      const int n = static_cast<int>(min(max(a.cols - col, 0L), 8L));
      float d[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) d[i] = 0.0f;
      if (a.dsum) load8<T>(static_cast<const T*>(a.dsum) + row * a.dsum_ld + col, n, d);
#pragma unroll
      for (int i = 0; i < 8; ++i) d[i] = fmaf(r, fmaf(-z[v][i], mean, u[v][i]), d[i]);
      store8<T>(static_cast<T*>(a.dx) + row * a.dx_ld + col, n, d);
    }
  }
  // partial row of this row group: [block * ROWS + group][cols]
  float* ws = a.ws + (static_cast<long>(blockIdx.x) * ROWS + threadIdx.x / TPR) * a.cols;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const long col = 8L * (v * TPR + t);
    const int n = static_cast<int>(min(max(a.cols - col, 0L), 8L));
    store8<float>(ws + col, n, dw[v]);
  }
}

// dweight[c] = the partial rows' sum, in order: eight runs of rows, then those.
constexpr int SUM_COLS = 32, SUM_RUNS = NT / SUM_COLS;
__global__ __launch_bounds__(NT) void rms_norm_sum_kernel(const float* ws, float* out, long cols, int rows) {
  __shared__ float part[SUM_RUNS][SUM_COLS];
  const int c = threadIdx.x % SUM_COLS, run = threadIdx.x / SUM_COLS;
  const long col = static_cast<long>(blockIdx.x) * SUM_COLS + c;
  const int each = (rows + SUM_RUNS - 1) / SUM_RUNS, r1 = min((run + 1) * each, rows);
  float s = 0.0f;
  if (col < cols)
    for (int r = run * each; r < r1; ++r) s += ws[r * cols + col];
  part[run][c] = s;
  __syncthreads();
  if (run || col >= cols) return;
  s = part[0][c];
#pragma unroll
  for (int i = 1; i < SUM_RUNS; ++i) s += part[i][c];
  out[col] = s;
}

// Threads of a row and vectors of a thread: one of 64 x {1, 2, 4}, 256 x {2, 4, 8}, 1024 x {4, 8}.
struct Shape {
  int tpr, v;
};
Shape shape_of(long cols) {
  const long n = (cols + 7) / 8;
  if (n <= 64) return {64, 1};
  if (n <= 128) return {64, 2};
  if (n <= 256) return {64, 4};
  if (n <= 512) return {256, 2};
  if (n <= 1024) return {256, 4};
  if (n <= 2048) return {256, 8};
  if (n <= 4096) return {1024, 4};
  return {1024, 8};
}
int rows_of_block(const Shape& s) { return s.tpr < NT ? NT / s.tpr : 1; }

constexpr long BWD_BLOCKS = 1024;
long bwd_blocks(long rows, const Shape& s) {
  const long need = (rows + rows_of_block(s) - 1) / rows_of_block(s);
  return std::max(1L, std::min(need, BWD_BLOCKS / rows_of_block(s)));
}

template <typename T, typename Y, bool BWD>
hipError_t launch(const RmsNormArgs& a, const Shape& sh, unsigned blocks, hipStream_t s) {
#define SPX_CASE(TPR, V)                                                                                          \
  if (sh.tpr == TPR && sh.v == V) {                                                                               \
    if (BWD) hipLaunchKernelGGL((rms_norm_bwd_kernel<T, Y, TPR, V>), dim3(blocks), dim3(TPR > NT ? TPR : NT), 0, s, a); \
    else hipLaunchKernelGGL((rms_norm_fwd_kernel<T, Y, TPR, V>), dim3(blocks), dim3(TPR > NT ? TPR : NT), 0, s, a);     \
    return hipGetLastError();                                                                                     \
  }
  SPX_CASE(64, 1)
  SPX_CASE(64, 2)
  SPX_CASE(64, 4)
  SPX_CASE(256, 2)
  SPX_CASE(256, 4)
  SPX_CASE(256, 8)
  SPX_CASE(1024, 4)
  SPX_CASE(1024, 8)
#undef SPX_CASE
  return hipErrorInvalidValue;
}

template <bool BWD>
hipError_t dispatch(const RmsNormArgs& a, const Shape& sh, unsigned blocks, hipStream_t s) {
  if (a.dtype) return launch<bf16_t, bf16_t, BWD>(a, sh, blocks, s);
  return a.out_dtype ? launch<float, bf16_t, BWD>(a, sh, blocks, s) : launch<float, float, BWD>(a, sh, blocks, s);
}

}  // namespace

size_t rms_norm_ws_bytes(long rows, long cols) {
  const Shape sh = shape_of(cols);
  return static_cast<size_t>(bwd_blocks(rows, sh)) * rows_of_block(sh) * cols * sizeof(float);
}

hipError_t rms_norm_fwd(const RmsNormArgs& a, hipStream_t s) {
  const Shape sh = shape_of(a.cols);
  const long blocks = std::min((a.rows + rows_of_block(sh) - 1) / rows_of_block(sh), 1L << 16);
  return dispatch<false>(a, sh, static_cast<unsigned>(blocks), s);
}

hipError_t rms_norm_bwd(const RmsNormArgs& a, hipStream_t s) {
  const Shape sh = shape_of(a.cols);
  const long blocks = bwd_blocks(a.rows, sh);
  if (hipError_t e = dispatch<true>(a, sh, static_cast<unsigned>(blocks), s); e != hipSuccess) return e;
  const unsigned sums = static_cast<unsigned>((a.cols + SUM_COLS - 1) / SUM_COLS);
  hipLaunchKernelGGL(rms_norm_sum_kernel, dim3(sums), dim3(NT), 0, s, a.ws, a.dweight, a.cols,
                     static_cast<int>(blocks * rows_of_block(sh)));
  return hipGetLastError();
}

}  // namespace spx
