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
#include <algorithm>
#include <type_traits>
#include <utility>

#include "blocks.hpp"
#include "kernels.hpp"

namespace spx {
namespace {

typedef int i32x8_t __attribute__((ext_vector_type(8)));
typedef int i32x4_t __attribute__((ext_vector_type(4)));

constexpr int NT = 256;
constexpr int BUF_FLAGS = 0x00020000;   // raw buffer resource word 3
constexpr int OOB = 0x40000000;         // past every resource, also with a tile's offset added: the load writes zeros
constexpr int BK = BLOCK_COLS;

// f(integral_constant<int, 0>) .. f(integral_constant<int, N - 1>): matrix
// instructions take the byte of a scale register as a constant.
template <class F, int... I>
__device__ __forceinline__ void each(std::integer_sequence<int, I...>, F&& f) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, class F>
__device__ __forceinline__ void each(F&& f) {
  each(std::make_integer_sequence<int, N>{}, std::forward<F>(f));
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t make_rsrc(const uint8_t* p, long bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(p), static_cast<short>(0),
                                           static_cast<int>(std::min(std::max(bytes, 0L), 0x7fffffe0L)), BUF_FLAGS);
}

// Direct loads into LDS: 16 (4) bytes of lane l land at lds + 16 l (4 l). A wait
// state lies between the write of M0 and the load that reads it; what is loaded
// is waited for by dma_wait, since the compiler does not see these loads.
__device__ __forceinline__ void dma16(__amdgpu_buffer_rsrc_t r, uint32_t lds, int off) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds), "v"(off), "s"(r)
               : "memory", "m0");
}
__device__ __forceinline__ void dma4(__amdgpu_buffer_rsrc_t r, uint32_t lds, int off) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(lds), "v"(off), "s"(r)
               : "memory", "m0");
}
template <int N>
__device__ __forceinline__ void dma_wait() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
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

struct TileArgs : ProductArgs {
  uint32_t tiles_m = 0, tiles_n = 0, total = 0;   // total: tiles by slices of k
  int k_blocks = 0, per_split = 0, splits = 1;    // blocks of 128, and of a slice
  float* partial = nullptr;                       // splits > 1: [slice][m][n]
  int wide = 0;                                   // rows of out and mask allow a thread's columns at once
};

template <int W>
__device__ __forceinline__ void store_whole(const ProductArgs& a, long at, const float (&v)[W]) {
  typedef float fW __attribute__((ext_vector_type(W)));
  typedef uint16_t hW __attribute__((ext_vector_type(W)));
  if (a.out_dtype) {
    if constexpr (W == 4) {
      *reinterpret_cast<uint2*>(static_cast<bf16_t*>(a.out) + at) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
    } else if constexpr (W == 2) {
      *reinterpret_cast<uint32_t*>(static_cast<bf16_t*>(a.out) + at) = pack_bf16x2(v[0], v[1]);
    } else {
      static_cast<bf16_t*>(a.out)[at] = f32_to_bf16(v[0]);
    }
  } else {
    fW u;
#pragma unroll
    for (int q = 0; q < W; ++q) u[q] = v[q];
    *reinterpret_cast<fW*>(static_cast<float*>(a.out) + at) = u;
  }
}

// What becomes of W consecutive columns j .. j + W - 1 of row i, n of them there.
template <int W>
__device__ __forceinline__ void finish(const ProductArgs& a, bool wide, long i, long j, int n, float (&v)[W]) {
  if (n <= 0) return;
  const bool all = wide && n >= W;
  typedef float fW __attribute__((ext_vector_type(W)));
  typedef bf16_t hW __attribute__((ext_vector_type(W)));
  const auto load = [&](const void* base, int dtype, long at, bool whole, float (&x)[W]) {
#pragma unroll
    for (int q = 0; q < W; ++q) x[q] = 0.0f;
    if (dtype) {
      const bf16_t* p = static_cast<const bf16_t*>(base) + at;
      if (whole) {
        const hW u = *reinterpret_cast<const hW*>(p);
#pragma unroll
        for (int q = 0; q < W; ++q) x[q] = bf16_to_f32(u[q]);
      } else {
#pragma unroll
        for (int q = 0; q < W; ++q)
          if (q < n) x[q] = bf16_to_f32(p[q]);
      }
    } else {
      const float* p = static_cast<const float*>(base) + at;
      if (whole) {
        const fW u = *reinterpret_cast<const fW*>(p);
#pragma unroll
        for (int q = 0; q < W; ++q) x[q] = u[q];
      } else {
#pragma unroll
        for (int q = 0; q < W; ++q)
          if (q < n) x[q] = p[q];
      }
    }
  };
  float x[W];
  if (a.bias) {
    load(a.bias, a.bias_dtype, j, false, x);
#pragma unroll
    for (int q = 0; q < W; ++q) v[q] += x[q];
  }
  if (a.relu) {
#pragma unroll
    for (int q = 0; q < W; ++q) v[q] = v[q] < 0.0f ? 0.0f : v[q];
  }
  if (a.mask) {
    load(a.mask, a.out_dtype, i * a.mask_ld + j, all, x);
#pragma unroll
    for (int q = 0; q < W; ++q) v[q] = x[q] > 0.0f ? v[q] : 0.0f;
  }
  const long at = i * a.out_ld + j;
  if (a.accumulate) {
    load(a.out, 0, at, all, x);
#pragma unroll
    for (int q = 0; q < W; ++q) v[q] += x[q];
  }
  if (all) {
    store_whole<W>(a, at, v);
    return;
  }
#pragma unroll
  for (int q = 0; q < W; ++q)
    if (q < n) {
      if (a.out_dtype) static_cast<bf16_t*>(a.out)[at + q] = f32_to_bf16(v[q]);
      else static_cast<float*>(a.out)[at + q] = v[q];
    }
}

// One operand's part of a block tile: T * 64 rows, of which wave half w takes
// T * 32 as T matrix-instruction tiles; tile i holds the half's rows T r + i, r <
// 32, so a lane's T scales (and, for B, its T columns of the result) lie side by
// side. In LDS row s = (w T + i) 32 + r has the 128 codes of a k block in eight
// chunks of 16, chunk c at c ^ (s / 2 % 8): sixteen lanes that read one chunk of
// consecutive rows then touch every bank once.
template <int T>
struct Side {
  static constexpr int ROWS = 64 * T, LOADS = 2 * T, CODES = ROWS * BK, BYTES = CODES + 256;   // scales: one load
  __amdgpu_buffer_rsrc_t codes, scales;
  int off;          // of the first direct load's row, and the lane's chunk in it
  int chunk;        // byte of that chunk in the k block
  int ld;

  __device__ void init(const uint8_t* c, const uint8_t* s, long ld, long s_ld, long row0, long rows, long k, int k_blocks,
                       int wave, int lane) {
    const int here = static_cast<int>(min(rows - row0, static_cast<long>(ROWS)));
    const long line = (k + 15) / 16 * 16;   // a line's bytes that are there
    codes = make_rsrc(c + row0 * ld, (here - 1) * ld + line);
    chunk = ((lane & 7) ^ ((4 * (wave & 1) + (lane >> 4)) & 7)) * 16;
    off = (8 * wave + (lane >> 3)) * T * static_cast<int>(ld) + chunk;
    this->ld = static_cast<int>(ld);
    scales = make_rsrc(s + row0, (k_blocks - 1) * s_ld + (rows + 15) / 16 * 16 - row0);
  }
  // Load q of a k block into the stage at `lds`; from: off in that block. Rows behind the last become zeros.
  __device__ __forceinline__ void load(int q, uint32_t lds, int from, int wave) {
    dma16(codes, lds + 1024u * (wave + 4 * q), from + ((q / T) * 32 * T + q % T) * ld);
  }
};

// 64 TI x 64 TJ of the output by four waves of 32 TI x 32 TJ.
//
// k goes by blocks of 128, two of them in LDS, filled by direct loads; a wave
// multiplies one half of a block from registers while the next half comes from
// LDS. The barrier in the middle of a block stands for both: its second half has
// been read, so the block after next may be loaded over it, and the next block has
// arrived.
template <int TI, int TJ, bool EXACT, int BLOCKS>
__global__ __launch_bounds__(NT, BLOCKS) void product_tile_kernel(TileArgs a) {
  typedef Side<TI> SA;
  typedef Side<TJ> SB;
  constexpr int STAGE = SA::BYTES + SB::BYTES;
  __shared__ __attribute__((aligned(16))) uint8_t lds[2 * STAGE];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave >> 1, wn = wave & 1, r = lane & 31, half = lane >> 5;

  // each XCD (blocks go round them) takes a run of the order slice, strip of four tile rows, column, row
  const uint32_t each_xcd = (a.total + 7) >> 3, ord = (blockIdx.x & 7) * each_xcd + (blockIdx.x >> 3);
  if ((blockIdx.x >> 3) >= each_xcd || ord >= a.total) return;
  const uint32_t tiles = a.tiles_m * a.tiles_n, split = ord / tiles, t = ord - split * tiles;
  const uint32_t strip = t / (4 * a.tiles_n), in = t - strip * 4 * a.tiles_n, high = min(4u, a.tiles_m - 4 * strip);
  const uint32_t tn = in / high, tm = 4 * strip + in - tn * high;
  const long row0 = static_cast<long>(tm) * SA::ROWS, col0 = static_cast<long>(tn) * SB::ROWS;
  const int kb0 = split * a.per_split, kb1 = min(kb0 + a.per_split, a.k_blocks);

  SA sa;
  SB sb;
  sa.init(a.a, a.a_scales, a.a_ld, a.a_scales_ld, row0, a.m, a.k, a.k_blocks, wave, lane);
  sb.init(a.b, a.b_scales, a.b_ld, a.b_scales_ld, col0, a.n, a.k, a.k_blocks, wave, lane);
  const uint32_t base = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) uint8_t*)&lds[0]));
  const int line = static_cast<int>((a.k + 15) / 16 * 16);
  const auto from = [&](int off, int chunk, int kb) { return off + (kb < kb1 && kb * BK + chunk < line ? kb * BK : OOB); };
  // waves of even number load A's scale bytes, the others B's: twice the same bytes, and no branch in the loop
  const __amdgpu_buffer_rsrc_t scales = wave & 1 ? sb.scales : sa.scales;
  const int scales_ld = static_cast<int>(wave & 1 ? a.b_scales_ld : a.a_scales_ld);
  const uint32_t scales_at = wave & 1 ? SA::BYTES + SB::CODES : SA::CODES;
  const auto load_scales = [&](int kb, uint32_t stage) {
    dma4(scales, stage + scales_at, kb < kb1 ? 4 * lane + kb * scales_ld : 0x7ffffff0);
  };
  const auto load_block = [&](int kb) {
    const uint32_t stage = base + static_cast<uint32_t>(kb & 1) * STAGE;
    load_scales(kb, stage);
    const int fa0 = from(sa.off, sa.chunk, kb), fb0 = from(sb.off, sb.chunk, kb);
#pragma unroll
    for (int q = 0; q < SA::LOADS; ++q) sa.load(q, stage, fa0, wave);
#pragma unroll
    for (int q = 0; q < SB::LOADS; ++q) sb.load(q, stage + SA::BYTES, fb0, wave);
  };
  f32x16_t acc[TI][TJ] = {};
  i32x8_t fa[2][TI], fb[2][TJ];   // by half of a k block
  // lane r of 32 reads chunks 4 h + 2 half, + 1 of row r of its tiles
  const int low = r * BK + (((2 * half) ^ ((r >> 1) & 7)) << 4);
  const auto read = [&](int tile_row, const uint8_t* s, int h) {
    const uint8_t* p = s + tile_row * (32 * BK);
    const i32x4_t lo = *reinterpret_cast<const i32x4_t*>(p + (low ^ (h << 6)));
    const i32x4_t hi = *reinterpret_cast<const i32x4_t*>(p + (low ^ (h << 6) ^ 16));
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  };
  const auto read_a = [&](int i, int kb, int h) { fa[h][i] = read(wm * TI + i, lds + (kb & 1) * STAGE, h); };
  const auto read_b = [&](int j, int kb, int h) { fb[h][j] = read(wn * TJ + j, lds + (kb & 1) * STAGE + SA::BYTES, h); };
  // a lane's T scale bytes side by side
  const auto scale_bytes = [&](const uint8_t* s, auto width) {
    if constexpr (decltype(width)::value == 4) return *reinterpret_cast<const uint32_t*>(s);
    else if constexpr (decltype(width)::value == 2) return static_cast<uint32_t>(*reinterpret_cast<const uint16_t*>(s));
    else return static_cast<uint32_t>(*s);
  };
  uint32_t ea = 0, eb = 0;
  const auto read_scales = [&](int kb, uint32_t& na, uint32_t& nb) {
    const uint8_t* s = lds + (kb & 1) * STAGE;
    na = scale_bytes(s + SA::CODES + wm * 32 * TI + r * TI, std::integral_constant<int, TI>{});
    nb = scale_bytes(s + SA::BYTES + SB::CODES + wn * 32 * TJ + r * TJ, std::integral_constant<int, TJ>{});
  };

  // Bytes of the last block's lines behind k are not the tensor's: zeros in half h.
  const auto cut = [&](int n, int h) {   // n: codes of the block that count
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      const int keep = min(max(n - 64 * h - 32 * half - 4 * q, 0), 4);
      const int mask = static_cast<int>(keep == 4 ? 0xffffffffu : (1u << (8 * keep)) - 1u);
#pragma unroll
      for (int i = 0; i < TI; ++i) fa[h][i][q] &= mask;
#pragma unroll
      for (int j = 0; j < TJ; ++j) fb[h][j][q] &= mask;
    }
  };

  // Products of half h with what else the step does before each of them: todo(index).
  const auto multiply = [&](auto hc, auto&& todo) {
    constexpr int h = decltype(hc)::value;
    if constexpr (EXACT) {
      float va[TI], vb[TJ];
#pragma unroll
      for (int i = 0; i < TI; ++i) va[i] = __uint_as_float(((ea >> (8 * i)) & 0xffu) << 23);
#pragma unroll
      for (int j = 0; j < TJ; ++j) vb[j] = __uint_as_float(((eb >> (8 * j)) & 0xffu) << 23);
      each<4>([&](auto qc) {
        constexpr int q = decltype(qc)::value;
        bf16x8_t wb[TJ];
#pragma unroll
        for (int j = 0; j < TJ; ++j) wb[j] = widened(fb[h][j], q, vb[j]);
        each<TI>([&](auto ic) {
          constexpr int i = decltype(ic)::value;
          const bf16x8_t w = widened(fa[h][i], q, va[i]);
#pragma unroll
          for (int j = 0; j < TJ; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(w, wb[j], acc[i][j], 0, 0, 0);
          if constexpr (q % 2 == 0) todo(std::integral_constant<int, (q / 2) * TI + i>{}, std::integral_constant<int, 2 * TI>{});
        });
      });
    } else {
      each<TI>([&](auto ic) {
        each<TJ>([&](auto jc) {
          constexpr int i = decltype(ic)::value, j = decltype(jc)::value;
          acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fa[h][i], fb[h][j], acc[i][j], 0, 0, i, ea, j, eb);
          todo(std::integral_constant<int, i * TJ + j>{}, std::integral_constant<int, TI * TJ>{});
        });
      });
    }
  };
  // item w of the reads of a half: B's tiles first, as every product of the next step's first row needs them
  const auto read_item = [&](auto wc, int kb, int h) {
    constexpr int w = decltype(wc)::value;
    if constexpr (w == 0) read_a(0, kb, h);
    else if constexpr (w <= TJ) read_b(w - 1, kb, h);
    else if constexpr (w < TI + TJ) read_a(w - TJ, kb, h);
  };

  constexpr int READS = TI + TJ, LOADS = SA::LOADS + SB::LOADS;
  const auto read_some = [&](auto wc, auto total, int kb, int h) {
    constexpr int w = decltype(wc)::value, n = decltype(total)::value, per = (READS + n - 1) / n;
    each<per>([&](auto u) { read_item(std::integral_constant<int, w * per + decltype(u)::value>{}, kb, h); });
  };
  if (kb0 < kb1) {
    load_block(kb0);
    load_block(kb0 + 1);
    dma_wait<LOADS>();
    __syncthreads();
    each<READS>([&](auto w) { read_item(w, kb0, 0); });
    read_scales(kb0, ea, eb);
    for (int kb = kb0; kb + 1 < kb1; ++kb) {
      multiply(std::integral_constant<int, 0>{}, [&](auto w, auto total) {
        read_some(w, total, kb, 1);
        __builtin_amdgcn_sched_barrier(0);
      });
      dma_wait<0>();
      __syncthreads();
      const uint32_t stage = base + static_cast<uint32_t>(kb & 1) * STAGE;
      load_scales(kb + 2, stage);
      uint32_t na, nb;
      read_scales(kb + 1, na, nb);
      const int fa0 = from(sa.off, sa.chunk, kb + 2), fb0 = from(sb.off, sb.chunk, kb + 2);
      multiply(std::integral_constant<int, 1>{}, [&](auto wc, auto total) {
        constexpr int w = decltype(wc)::value, n = decltype(total)::value, per = (LOADS + n - 1) / n;
        read_some(wc, total, kb + 1, 0);
        each<per>([&](auto u) {
          constexpr int item = w * per + decltype(u)::value;
          if constexpr (item < SA::LOADS) sa.load(item, stage, fa0, wave);
          else if constexpr (item < LOADS) sb.load(item - SA::LOADS, stage + SA::BYTES, fb0, wave);
        });
        __builtin_amdgcn_sched_barrier(0);
      });
      ea = na;
      eb = nb;
    }
    const int n = static_cast<int>(min(a.k - (kb1 - 1L) * BK, static_cast<long>(BK)));
    each<READS>([&](auto w) { read_item(w, kb1 - 1, 1); });
    if (n < BK) {
      cut(n, 0);
      cut(n, 1);
    }
    multiply(std::integral_constant<int, 0>{}, [](auto, auto) {});
    multiply(std::integral_constant<int, 1>{}, [](auto, auto) {});
  }
  dma_wait<0>();   // the block's LDS may be another's when it ends

  ProductArgs e = a;   // a slice's sums go to its plane as they are
  if (a.partial) {
    e.out = a.partial + split * a.m * a.n;
    e.out_ld = a.n;
    e.out_dtype = e.relu = e.accumulate = 0;
    e.bias = e.mask = nullptr;
  }
  const long j = col0 + wn * 32 * TJ + r * TJ;
  const int n = static_cast<int>(min(a.n - j, static_cast<long>(TJ)));
  const long row_first = row0 + wm * 32 * TI + 4 * half * TI;
  if (a.wide && col0 + SB::ROWS <= a.n && !e.mask && !e.accumulate) {   // straight stores of whole columns
    float bias[TJ];
#pragma unroll
    for (int q = 0; q < TJ; ++q)
      bias[q] = !e.bias ? 0.0f : e.bias_dtype ? bf16_to_f32(static_cast<const bf16_t*>(e.bias)[j + q])
                                               : static_cast<const float*>(e.bias)[j + q];
    const float least = e.relu ? 0.0f : -INFINITY;
#pragma unroll
    for (int i = 0; i < TI; ++i) {
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const long row = row_first + (8 * (v >> 2) + (v & 3)) * TI + i;
        float x[TJ];
#pragma unroll
        for (int q = 0; q < TJ; ++q) {
          x[q] = acc[i][q][v] + bias[q];
          x[q] = x[q] < least ? least : x[q];
        }
        if (row < a.m) store_whole<TJ>(e, row * e.out_ld + j, x);
      }
    }
    return;
  }
  // the general epilogue is long: a loop over rows, which pass through LDS for an index of their own
  __syncthreads();
  float* own = reinterpret_cast<float*>(lds) + wave * (16 * 64 * TJ) + lane * TJ;
  static_assert(4 * 16 * 64 * TJ * 4 <= 2 * STAGE, "a tile row of every wave fits");
  each<TI>([&](auto ic) {
    constexpr int i = decltype(ic)::value;
#pragma unroll
    for (int v = 0; v < 16; ++v)
#pragma unroll
      for (int q = 0; q < TJ; ++q) own[v * 64 * TJ + q] = acc[i][q][v];
#pragma unroll 1
    for (int v = 0; v < 16; ++v) {
      const long row = row_first + (8 * (v >> 2) + (v & 3)) * TI + i;
      float x[TJ];
#pragma unroll
      for (int q = 0; q < TJ; ++q) x[q] = own[v * 64 * TJ + q];
      if (row < a.m) finish<TJ>(e, a.wide, row, j, n, x);
    }
  });
}

// The slices' partial sums, added in order.
__global__ __launch_bounds__(NT) void product_join_kernel(TileArgs a) {
  const long cols = (a.n + 3) / 4, at = static_cast<long>(blockIdx.x) * NT + threadIdx.x;
  const long i = at / cols, j = 4 * (at - i * cols);
  if (i >= a.m) return;
  const int n = static_cast<int>(min(a.n - j, 4L));
  float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
  const float* p = a.partial + i * a.n + j;
  for (int s = 0; s < a.splits; ++s)
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (q < n) v[q] += p[static_cast<long>(s) * a.m * a.n + q];
  finish<4>(a, a.wide, i, j, n, v);
}

struct Plan {
  int ti, tj, splits, per;
};

Plan plan_of(long m, long n, long k, bool exact) {
  const auto tiles = [&](int ti, int tj) { return ((m + 64 * ti - 1) / (64 * ti)) * ((n + 64 * tj - 1) / (64 * tj)); };
  const int blocks = static_cast<int>((k + BK - 1) / BK);
  Plan p{2, 2, 1, std::max(blocks, 1)};
  if (!exact && tiles(4, 4) >= 192) p.ti = p.tj = 4;
  else if (tiles(2, 2) < 256) p.ti = p.tj = 1;
  return p;
}

bool wide(const void* p, long ld, int dtype, int w) {
  return !p || (ld % w == 0 && reinterpret_cast<uintptr_t>(p) % ((dtype ? 2 : 4) * w) == 0);
}

template <int TI, int TJ, bool EXACT, int BLOCKS>
hipError_t launch(TileArgs a, hipStream_t s) {
  a.tiles_m = static_cast<uint32_t>((a.m + 64 * TI - 1) / (64 * TI));
  a.tiles_n = static_cast<uint32_t>((a.n + 64 * TJ - 1) / (64 * TJ));
  a.total = a.tiles_m * a.tiles_n * a.splits;
  const int w = a.splits > 1 ? 4 : TJ;
  a.wide = wide(a.out, a.out_ld, a.out_dtype, w) && wide(a.mask, a.mask_ld, a.out_dtype, w);
  hipLaunchKernelGGL((product_tile_kernel<TI, TJ, EXACT, BLOCKS>), dim3((a.total + 7) / 8 * 8), dim3(NT), 0, s, a);
  return hipGetLastError();
}

}  // namespace

size_t product_ws_bytes(long, long, long) { return 0; }

hipError_t product(const ProductArgs& args, hipStream_t s) {
  const bool exact = args.out_dtype == 0;
  const Plan p = plan_of(args.m, args.n, args.k, exact);
  TileArgs a;
  static_cast<ProductArgs&>(a) = args;
  a.k_blocks = static_cast<int>((args.k + BK - 1) / BK);
  a.splits = p.splits;
  a.per_split = p.per;
  if (exact) return p.ti == 2 ? launch<2, 2, true, 2>(a, s) : launch<1, 1, true, 4>(a, s);
  if (p.ti == 4) return launch<4, 4, false, 1>(a, s);
  return p.ti == 2 ? launch<2, 2, false, 2>(a, s) : launch<1, 1, false, 4>(a, s);
}

}  // namespace spx
