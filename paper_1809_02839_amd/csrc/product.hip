// Product of two tensors in blocks of 128.
//
// A bf16 out is summed by v_mfma_scale_f32_32x32x64_f8f6f4, whose operands carry an
// e8m0 scale for 32 values of a row: a block's byte serves four of them, so
// scaling costs no instruction. That instruction adds eight products of
// consecutive k in fixed point, cut (towards zero) 2^-13 below the largest of
// them, and the eights in float32: measured on normal values 1.5e-5 of the result's
// norm at any k, 9e-5 where a few columns are far larger than the others; a bf16
// rounding is 1.7e-3. A float32 out is not given away to that: its codes are
// turned to bf16 (exact, scale included) for v_mfma_f32_32x32x16_bf16 at half the
// rate (1e-7 of the norm).
//
// 8192 cubed: 400 us, 2750 TFLOP/s, matrix instructions busy 79% of the time; float32
// out 745 us, 1475 TFLOP/s, busy 80%. The vendor library multiplies such codes without
// block scales in 376 us, and bf16 at 1574 TFLOP/s (16384 x 16384 x 8192).
#include <algorithm>
#include <iterator>
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
  int k_blocks = 0, per_split = 0, splits = 1;    // blocks of 128 (1 at least), and of a slice
  float* partial = nullptr;                       // splits > 1: [slice][m][n]
};

// W values of a row, stored at any element's address.
template <int W>
using Floats = float __attribute__((ext_vector_type(W), aligned(4)));

template <int W>
__device__ __forceinline__ void store_whole(float* p, const float (&v)[W]) {
  Floats<W> u;
#pragma unroll
  for (int q = 0; q < W; ++q) u[q] = v[q];
  *reinterpret_cast<Floats<W>*>(p) = u;
}
template <int W>
__device__ __forceinline__ void store_whole(bf16_t* p, const float (&v)[W]) {
  if constexpr (W == 4) {
    typedef uint32_t pair_t __attribute__((ext_vector_type(2), aligned(2)));
    *reinterpret_cast<pair_t*>(p) = pair_t{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
  } else if constexpr (W == 2) {
    typedef uint32_t word_t __attribute__((aligned(2)));
    *reinterpret_cast<word_t*>(p) = pack_bf16x2(v[0], v[1]);
  } else {
    *p = f32_to_bf16(v[0]);
  }
}
__device__ __forceinline__ float value(float v) { return v; }
__device__ __forceinline__ float value(bf16_t v) { return bf16_to_f32(v); }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(bf16_t* p, float v) { *p = f32_to_bf16(v); }

// n (of W) values of a row, the others 0.
template <int W, typename T>
__device__ __forceinline__ void load_part(const T* p, int n, float (&v)[W]) {
  if (n >= W) {
    typedef T vec_t __attribute__((ext_vector_type(W), aligned(sizeof(T))));
    const vec_t u = *reinterpret_cast<const vec_t*>(p);
#pragma unroll
    for (int q = 0; q < W; ++q) v[q] = value(u[q]);
  } else {
#pragma unroll
    for (int q = 0; q < W; ++q) v[q] = q < n ? value(p[q]) : 0.0f;
  }
}

template <int W>
__device__ __forceinline__ void load_bias(const ProductArgs& a, long j, int n, float (&v)[W]) {
#pragma unroll
  for (int q = 0; q < W; ++q) v[q] = 0.0f;
  if (!a.bias) return;
  if (a.bias_dtype) load_part<W>(static_cast<const bf16_t*>(a.bias) + j, n, v);
  else load_part<W>(static_cast<const float*>(a.bias) + j, n, v);
}

// What becomes of the sums v of n (of W) columns, at p in out and at gate in the mask.
template <int W, typename T>
__device__ __forceinline__ void finish(const ProductArgs& a, const float (&bias)[W], T* p, const T* gate, int n, float (&v)[W]) {
  const float least = a.relu ? 0.0f : -INFINITY;   // a NaN stays
#pragma unroll
  for (int q = 0; q < W; ++q) {
    v[q] += bias[q];
    v[q] = v[q] < least ? least : v[q];
  }
  float x[W];
  if (a.mask) {
    load_part<W>(gate, n, x);
#pragma unroll
    for (int q = 0; q < W; ++q) v[q] = x[q] > 0.0f ? v[q] : 0.0f;
  }
  if (a.accumulate) {
    load_part<W>(p, n, x);
#pragma unroll
    for (int q = 0; q < W; ++q) v[q] += x[q];
  }
  if (n >= W) {
    store_whole<W>(p, v);
  } else {
#pragma unroll
    for (int q = 0; q < W; ++q)
      if (q < n) put(p + q, v[q]);
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
  __amdgpu_buffer_rsrc_t codes;
  int off;          // of the first direct load's row, and the lane's chunk in it
  int chunk;        // byte of that chunk in the k block
  int ld;

  __device__ __forceinline__ void init(const uint8_t* c, long ld, long row0, long rows, long k, int wave, int lane) {
    const int here = static_cast<int>(min(rows - row0, static_cast<long>(ROWS)));
    const long line = (k + 15) / 16 * 16;   // a line's bytes that are there
    codes = make_rsrc(c + row0 * ld, k ? (here - 1) * ld + line : 0);
    chunk = ((lane & 7) ^ ((4 * (wave & 1) + (lane >> 4)) & 7)) * 16;
    off = (8 * wave + (lane >> 3)) * T * static_cast<int>(ld) + chunk;
    this->ld = static_cast<int>(ld);
  }
  // Load q of a k block into the stage at `lds`; from: off in that block. Rows behind the last become zeros.
  __device__ __forceinline__ void load(int q, uint32_t lds, int from, int wave) {
    dma16(codes, lds + 1024u * (wave + 4 * q), from + ((q / T) * 32 * T + q % T) * ld);
  }
};

// Blocks that share a CU's LDS, 160 KiB.
constexpr int blocks_of_cu(int ti, int tj, int stages) {
  return 160 * 1024 / (stages * (64 * (ti + tj) * BK + 512));
}

// 64 TI x 64 TJ of the output by four waves of 32 TI x 32 TJ.
//
// k goes by blocks of 128, STAGES of them in LDS, filled by direct loads; a wave
// multiplies one half of a block from registers while the next half comes from
// LDS. After the barrier in the middle of a block, its second half read by every
// wave, a later block is loaded over it; where a half has four groups of products or
// more, the next block is waited for, by a second barrier, amid the second half's
// (8192 cubed 418 -> 400 us: loads have half as long again to arrive). Steps of 64 k
// in twice the stages, for longer waits still, lost (458: half lines of memory).
enum Epilogue : int {
  EPI_PLAIN,   // bias and ReLU
  EPI_READS,   // also a mask, or sums to add to
  EPI_SLICE    // a slice's sums, as they are, to its plane
};
template <int TI, int TJ, bool EXACT, int STAGES, int EPILOGUE>
__global__ __launch_bounds__(NT, blocks_of_cu(TI, TJ, STAGES)) void product_tile_kernel(TileArgs a) {
  typedef Side<TI> SA;
  typedef Side<TJ> SB;
  constexpr int STAGE = SA::BYTES + SB::BYTES;
  __shared__ __attribute__((aligned(16))) uint8_t lds[STAGES * STAGE];
  static_assert((STAGES & (STAGES - 1)) == 0 && (STAGES - 1) * (SA::LOADS + SB::LOADS + 1) < 64, "counted by vmcnt");
  const auto stage_of = [](int kb) { return (kb & (STAGES - 1)) * STAGE; };
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
  sa.init(a.a, a.a_ld, row0, a.m, a.k, wave, lane);
  sb.init(a.b, a.b_ld, col0, a.n, a.k, wave, lane);
  const uint32_t base = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) uint8_t*)&lds[0]));
  const int line = static_cast<int>((a.k + 15) / 16 * 16);
  const auto from = [&](int off, int chunk, int kb) { return off + (kb < kb1 && kb * BK + chunk < line ? kb * BK : OOB); };
  // waves of even number load A's scale bytes, the others B's: twice the same bytes, and no branch in the loop
  const bool second = wave & 1;
  const int scales_ld = static_cast<int>(second ? a.b_scales_ld : a.a_scales_ld);
  const uint32_t scales_at = second ? SA::BYTES + SB::CODES : SA::CODES;
  const long line0 = second ? col0 : row0, lines = second ? a.n : a.m;
  const __amdgpu_buffer_rsrc_t scales =
      make_rsrc((second ? a.b_scales : a.a_scales) + line0,
                a.k ? (a.k_blocks - 1L) * scales_ld + (lines + 15) / 16 * 16 - line0 : 0);
  // lanes that have no byte of the tile's part of a line load its last four again
  const int scales_off = static_cast<int>(std::min(4L * lane, tile_scale_bytes(second ? SB::ROWS : SA::ROWS, line0, lines) - 4));
  const auto load_scales = [&](int kb, uint32_t stage) {
    dma4(scales, stage + scales_at, kb < kb1 ? scales_off + kb * scales_ld : 0x7ffffff0);
  };
  const auto load_block = [&](int kb) {
    const uint32_t stage = base + static_cast<uint32_t>(stage_of(kb));
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
  const auto read_a = [&](int i, int kb, int h) { fa[h][i] = read(wm * TI + i, lds + stage_of(kb), h); };
  const auto read_b = [&](int j, int kb, int h) { fb[h][j] = read(wn * TJ + j, lds + stage_of(kb) + SA::BYTES, h); };
  // a lane's T scale bytes side by side
  const auto scale_bytes = [&](const uint8_t* s, auto width) {
    if constexpr (decltype(width)::value == 4) return *reinterpret_cast<const uint32_t*>(s);
    else if constexpr (decltype(width)::value == 2) return static_cast<uint32_t>(*reinterpret_cast<const uint16_t*>(s));
    else return static_cast<uint32_t>(*s);
  };
  uint32_t ea = 0, eb = 0;
  const auto read_scales = [&](int kb, uint32_t& na, uint32_t& nb) {
    const uint8_t* s = lds + stage_of(kb);
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
  constexpr bool LATE = (EXACT ? 2 * TI : TI * TJ) >= 4;   // groups of products: the next block is waited for amid the second half's
  const auto read_some = [&](auto wc, auto total, int kb, int h) {
    constexpr int w = decltype(wc)::value, n = decltype(total)::value, per = (READS + n - 1) / n;
    each<per>([&](auto u) { read_item(std::integral_constant<int, w * per + decltype(u)::value>{}, kb, h); });
  };
#pragma unroll
  for (int q = 0; q < STAGES; ++q) load_block(kb0 + q);
  dma_wait<(STAGES - 1) * (LOADS + 1)>();
  __syncthreads();
  each<READS>([&](auto w) { read_item(w, kb0, 0); });
  read_scales(kb0, ea, eb);
  for (int kb = kb0; kb + 1 < kb1; ++kb) {
    multiply(std::integral_constant<int, 0>{}, [&](auto w, auto total) {
      read_some(w, total, kb, 1);
      __builtin_amdgcn_sched_barrier(0);
    });
    if constexpr (!LATE) dma_wait<(STAGES - 2) * (LOADS + 1)>();
    __syncthreads();
    const uint32_t stage = base + static_cast<uint32_t>(stage_of(kb));
    load_scales(kb + STAGES, stage);
    uint32_t na, nb;
    if constexpr (!LATE) read_scales(kb + 1, na, nb);
    const int fa0 = from(sa.off, sa.chunk, kb + STAGES), fb0 = from(sb.off, sb.chunk, kb + STAGES);
    multiply(std::integral_constant<int, 1>{}, [&](auto wc, auto total) {
      constexpr int w = decltype(wc)::value, n = decltype(total)::value, per = (LOADS + n - 1) / n;
      if constexpr (!LATE) read_some(wc, total, kb + 1, 0);
      else if constexpr (w >= n / 2) read_some(std::integral_constant<int, w - n / 2>{}, std::integral_constant<int, n - n / 2>{}, kb + 1, 0);
      each<per>([&](auto u) {
        constexpr int item = w * per + decltype(u)::value;
        if constexpr (item < SA::LOADS) sa.load(item, stage, fa0, wave);
        else if constexpr (item < LOADS) sb.load(item - SA::LOADS, stage + SA::BYTES, fb0, wave);
      });
      if constexpr (LATE && w == n / 2 - 1) {
        dma_wait<(STAGES - 2) * (LOADS + 1) + 1 + ((w + 1) * per < LOADS ? (w + 1) * per : LOADS)>();
        __syncthreads();
        read_scales(kb + 1, na, nb);
      }
      __builtin_amdgcn_sched_barrier(0);
    });
    ea = na;
    eb = nb;
  }
  const int left = static_cast<int>(min(a.k - (kb1 - 1L) * BK, static_cast<long>(BK)));
  each<READS>([&](auto w) { read_item(w, kb1 - 1, 1); });
  if (left < BK) {
    cut(left, 0);
    cut(left, 1);
  }
  multiply(std::integral_constant<int, 0>{}, [](auto, auto) {});
  multiply(std::integral_constant<int, 1>{}, [](auto, auto) {});
  dma_wait<0>();   // the block's LDS may be another's when it ends
  // lane: columns j .. of the rows first + (8 (v / 4) + v % 4) TI + i, `rows` of them there
  const long j = col0 + wn * 32 * TJ + r * TJ, first = row0 + wm * 32 * TI + 4 * half * TI;
  const int n = static_cast<int>(min(a.n - j, static_cast<long>(TJ)));
  const int rows = static_cast<int>(min(a.m - first, 64L * TI));
  if (n <= 0 || rows <= 0) return;
  typedef typename std::conditional<EXACT || EPILOGUE == EPI_SLICE, float, bf16_t>::type T;
  const long ld = EPILOGUE == EPI_SLICE ? a.n : a.out_ld;
  T* const out = (EPILOGUE == EPI_SLICE ? reinterpret_cast<T*>(a.partial) + split * a.m * a.n : static_cast<T*>(a.out)) + first * ld + j;
  const T* const gates = static_cast<const T*>(a.mask) + first * a.mask_ld + j;
  float bias[TJ];
  if constexpr (EPILOGUE != EPI_SLICE) load_bias<TJ>(a, j, n, bias);
  const float least = a.relu ? 0.0f : -INFINITY;   // a NaN stays
  const auto row_at = [](int i, int v) { return (8 * (v >> 2) + (v & 3)) * TI + i; };   // row v of tile i, from first
  if (EPILOGUE != EPI_READS || n < TJ) {
    each<TI>([&](auto ic) {
      constexpr int i = decltype(ic)::value;
#pragma unroll
      for (int v0 = 0; v0 < 16; v0 += 4) {   // four rows, TI apart
        const int d0 = row_at(i, v0);
        T* const p = out + d0 * ld;
        const T* const g = gates + d0 * a.mask_ld;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          if (d0 + v * TI >= rows) continue;
          T* const at = p + v * TI * ld;
          float x[TJ];
#pragma unroll
          for (int q = 0; q < TJ; ++q) {
            x[q] = acc[i][q][v0 + v];
            if constexpr (EPILOGUE != EPI_SLICE) {
              x[q] += bias[q];
              x[q] = x[q] < least ? least : x[q];
            }
            if constexpr (EPILOGUE == EPI_READS) {   // columns at the edge
              if (q >= n) continue;
              if (a.mask) x[q] = value(g[v * TI * a.mask_ld + q]) > 0.0f ? x[q] : 0.0f;
              if (EXACT && a.accumulate) x[q] += value(at[q]);
            }
          }
          if (n >= TJ) {
            store_whole<TJ>(at, x);
          } else {
#pragma unroll
            for (int q = 0; q < TJ; ++q)
              if (q < n) put(at + q, x[q]);
          }
        }
      }
    });
    return;
  }
  if constexpr (EPILOGUE == EPI_READS) {   // what a group of rows reads is asked for a group before
    constexpr int GROUP = EXACT ? 8 : 16, GROUPS = TI * 16 / GROUP;
    typedef T vec_t __attribute__((ext_vector_type(TJ), aligned(sizeof(T))));
    vec_t gate[2][GROUP], old[2][EXACT ? GROUP : 1];
    const auto ask = [&](auto gc) {
      constexpr int g = decltype(gc)::value;
#pragma unroll
      for (int v = 0; v < GROUP; ++v) {
        const long d = min(row_at(g * GROUP / 16, g * GROUP % 16 + v), rows - 1);
        if (a.mask) gate[g & 1][v] = *reinterpret_cast<const vec_t*>(gates + d * a.mask_ld);
        if constexpr (EXACT) {
          if (a.accumulate) old[g & 1][v] = *reinterpret_cast<const vec_t*>(out + d * ld);
        }
      }
    };
    ask(std::integral_constant<int, 0>{});
    each<GROUPS>([&](auto gc) {
      constexpr int g = decltype(gc)::value, i = g * GROUP / 16;
      if constexpr (g + 1 < GROUPS) ask(std::integral_constant<int, g + 1>{});
#pragma unroll
      for (int v = 0; v < GROUP; ++v) {
        const int d = row_at(i, g * GROUP % 16 + v);
        if (d >= rows) continue;
        float x[TJ];
#pragma unroll
        for (int q = 0; q < TJ; ++q) {
          x[q] = acc[i][q][g * GROUP % 16 + v] + bias[q];
          x[q] = x[q] < least ? least : x[q];
          if (a.mask) x[q] = value(gate[g & 1][v][q]) > 0.0f ? x[q] : 0.0f;
          if constexpr (EXACT) {
            if (a.accumulate) x[q] += value(old[g & 1][v][q]);
          }
        }
        store_whole<TJ>(out + d * ld, x);
      }
    });
  }
}

// The slices' partial sums, added in order.
__global__ __launch_bounds__(NT) void product_join_kernel(TileArgs a) {
  const long cols = (a.n + 3) / 4, at = static_cast<long>(blockIdx.x) * NT + threadIdx.x;
  const long i = at / cols, j = 4 * (at - i * cols);
  if (i >= a.m) return;
  const int n = static_cast<int>(min(a.n - j, 4L));
  float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
  const float* p = a.partial + i * a.n + j;
  const long plane = a.m * a.n;
  if (a.n % 4 == 0) {
#pragma unroll 4
    for (int s = 0; s < a.splits; ++s) {
      const float4 u = *reinterpret_cast<const float4*>(p + s * plane);
      v[0] += u.x, v[1] += u.y, v[2] += u.z, v[3] += u.w;
    }
  } else {
    for (int s = 0; s < a.splits; ++s)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (q < n) v[q] += p[s * plane + q];
  }
  float bias[4];
  load_bias<4>(a, j, n, bias);
  const long o = i * a.out_ld + j, gate = i * a.mask_ld + j;
  if (a.out_dtype) finish<4>(a, bias, static_cast<bf16_t*>(a.out) + o, static_cast<const bf16_t*>(a.mask) + gate, n, v);
  else finish<4>(a, bias, static_cast<float*>(a.out) + o, static_cast<const float*>(a.mask) + gate, n, v);
}

// Few rows of A (tokens): B, the weight, is read once and bounds the time. A wave
// takes 16 RT rows of B and every W-th block of k, its codes straight from memory
// into the registers of v_mfma_scale_f32_16x16x128_f8f6f4 (lane 16 c + r: 32
// codes of row r), the next block's under way while it multiplies; the waves'
// sums are added in order over LDS. 16 x 16384 x 8192: 28 us, 4.8 TB/s (in
// tiles of 64 32); half the waves' time is waiting for memory.
struct Fragment {
  i32x8_t codes;
  int scale;
};

template <int RT, int MT, bool EXACT>
__global__ __launch_bounds__(RT == 1 ? 1024 : 512) void product_rows_kernel(ProductArgs a, int k_blocks) {
  extern __shared__ __attribute__((aligned(16))) float sums[];   // [wave][RT][MT][lane][4]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
  const int r = lane & 15, c = lane >> 4;
  const long j0 = static_cast<long>(blockIdx.x) * 16 * RT;
  const uint8_t *pb[RT], *pa[MT];
  long rb[RT], ra[MT];
#pragma unroll
  for (int i = 0; i < RT; ++i) {
    rb[i] = min(j0 + 16 * i + r, a.n - 1);
    pb[i] = a.b + rb[i] * a.b_ld + 32 * c;
  }
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    ra[i] = min(16L * i + r, a.m - 1);
    pa[i] = a.a + ra[i] * a.a_ld + 32 * c;
  }
  struct Block {
    Fragment b[RT], a[MT];
  };
  const auto load = [&](Block& f, int kb) {
    const long at = static_cast<long>(kb) * BK, left = a.k - at - 32 * c;   // codes from the lane's first on
#pragma unroll
    for (int i = 0; i < RT + MT; ++i) {
      Fragment& t = i < RT ? f.b[i] : f.a[i - RT];
      const uint8_t* p = (i < RT ? pb[i] : pa[i - RT]) + at;
      i32x4_t h[2] = {};
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        if (left > 16 * q) h[q] = *reinterpret_cast<const i32x4_t*>(p + 16 * q);
      }
      t.codes = __builtin_shufflevector(h[0], h[1], 0, 1, 2, 3, 4, 5, 6, 7);
      t.scale = i < RT ? a.b_scales[kb * a.b_scales_ld + rb[i]] : a.a_scales[kb * a.a_scales_ld + ra[i - RT]];
    }
  };
  const auto cut = [&](Block& f, int kb) {   // bytes behind k are not the tensor's
    const long left = a.k - static_cast<long>(kb) * BK - 32 * c;
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      const int keep = static_cast<int>(min(max(left - 4 * q, 0L), 4L));
      const int mask = static_cast<int>(keep == 4 ? 0xffffffffu : (1u << (8 * keep)) - 1u);
#pragma unroll
      for (int i = 0; i < RT; ++i) f.b[i].codes[q] &= mask;
#pragma unroll
      for (int i = 0; i < MT; ++i) f.a[i].codes[q] &= mask;
    }
  };
  f32x4_t acc[RT][MT] = {};
  const auto multiply = [&](const Block& f) {
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        if constexpr (EXACT) {
          const float sb = __uint_as_float(static_cast<uint32_t>(f.b[i].scale) << 23);
          const float sa = __uint_as_float(static_cast<uint32_t>(f.a[m].scale) << 23);
#pragma unroll
          for (int q = 0; q < 4; ++q)
            acc[i][m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widened(f.b[i].codes, q, sb), widened(f.a[m].codes, q, sa),
                                                                acc[i][m], 0, 0, 0);
        } else {
          acc[i][m] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(f.b[i].codes, f.a[m].codes, acc[i][m], 0, 0, 0,
                                                                       f.b[i].scale, 0, f.a[m].scale);
        }
      }
  };
  Block now, next;
  if (wave < k_blocks) load(now, wave);
  for (int kb = wave; kb < k_blocks; kb += waves) {
    if (kb + waves < k_blocks) load(next, kb + waves);
    if ((kb + 1L) * BK > a.k) cut(now, kb);
    multiply(now);
    now = next;
  }
#pragma unroll
  for (int i = 0; i < RT; ++i)
#pragma unroll
    for (int m = 0; m < MT; ++m) *reinterpret_cast<f32x4_t*>(sums + (((wave * RT + i) * MT + m) * 64 + lane) * 4) = acc[i][m];
  __syncthreads();
  // lane 16 c + r of tile (i, m) holds columns j0 + 16 i + 4 c .. + 3 of row 16 m + r
  for (int t = threadIdx.x; t < RT * MT * 64; t += blockDim.x) {
    const int l = t & 63, m = (t >> 6) % MT, i = (t >> 6) / MT;
    const long row = 16 * m + (l & 15), j = j0 + 16 * i + 4 * (l >> 4);
    float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int w = 0; w < waves; ++w) {
      const f32x4_t u = *reinterpret_cast<const f32x4_t*>(sums + (w * RT * MT * 64 + t) * 4);
#pragma unroll
      for (int q = 0; q < 4; ++q) v[q] += u[q];
    }
    const int n = static_cast<int>(min(a.n - j, 4L));
    if (row >= a.m || n <= 0) continue;
    float bias[4];
    load_bias<4>(a, j, n, bias);
    typedef typename std::conditional<EXACT, float, bf16_t>::type T;
    finish<4>(a, bias, static_cast<T*>(a.out) + row * a.out_ld + j, static_cast<const T*>(a.mask) + row * a.mask_ld + j, n, v);
  }
}

// Rows of A that this kernel takes. 32 x 8192 x 4096 takes 10.7 us in it, in tiles of 64
// 10.3, in float32 11.3 and 12.3; 64 x 4096 x 4096, 64 rows a wave, would take 14.7, in tiles
// 9.0.
constexpr long ROWS_MAX = 32;

template <int MT, bool EXACT>
hipError_t launch_rows(const ProductArgs& a, hipStream_t s) {
  const int k_blocks = static_cast<int>((a.k + BK - 1) / BK);
  // 16 RT rows a block: a block for each CU at least where there are so many rows (16 x 8192 x
  // 4096: 32 rows 9.3 us, 16 11.5, 64 12.0; 16 x 16384 x 8192: 64 rows 28.3, 32 35.2). Waves: four
  // where k has no blocks for more (the same times as eight), sixteen for 16 rows and a long k,
  // which a few rows of A gain by and 32 lose by (1 x 2048 x 8192 7.3 us, with eight 8.1; 16 x
  // 2048 x 8192 10.5 and 9.8; 32 x 8176 x 2048 9.7 and 8.7)
  const int rt = a.n >= 256 * 64 ? 4 : a.n >= 256 * 32 ? 2 : 1;
  const int waves = k_blocks <= 4 ? 4 : rt == 1 && k_blocks > 8 ? 16 : 8;
  const unsigned blocks = static_cast<unsigned>((a.n + 16 * rt - 1) / (16 * rt));
  const size_t lds = static_cast<size_t>(waves) * rt * MT * 1024;
  if (rt == 4) hipLaunchKernelGGL((product_rows_kernel<4, MT, EXACT>), dim3(blocks), dim3(64 * waves), lds, s, a, k_blocks);
  else if (rt == 2) hipLaunchKernelGGL((product_rows_kernel<2, MT, EXACT>), dim3(blocks), dim3(64 * waves), lds, s, a, k_blocks);
  else hipLaunchKernelGGL((product_rows_kernel<1, MT, EXACT>), dim3(blocks), dim3(64 * waves), lds, s, a, k_blocks);
  return hipGetLastError();
}

// Kernels of square block tiles: 64 t rows and columns, stages of k in LDS, and
// what they cost by measurement (us): fixed for a block's start and end, a k
// block with one, or as many as fit, blocks of the kind on a CU, and a block's mask or
// sums to add to (8192 x 2048 x 2048 in float32 that is added to: tiles of 128 70 us, of
// 256 80; written only 62 and 59).
struct Variant {
  int t, stages, per_cu;
  double fixed, step_alone, step_full, reads;
};
constexpr Variant VARIANTS[] = {{4, 2, 1, 10.3, 1.40, 1.40, 3.0}, {2, 2, 2, 4.5, 0.44, 0.91, 1.0}, {1, 4, 2, 2.2, 0.22, 0.375, 0.5}};
constexpr Variant VARIANTS_EXACT[] = {{4, 2, 1, 12.5, 2.70, 2.70, 20.0}, {2, 2, 2, 4.6, 0.84, 1.54, 6.0}, {1, 4, 2, 2.5, 0.385, 0.62, 2.0}};

struct Plan {
  int variant = 0, splits = 1, per_split = 1;
};

constexpr int MAX_SPLITS = 16;

// The kernel and the slices of k of the least modelled time: rounds of blocks over
// the 256 CUs, and for slices a second launch that reads their planes. In us: 8192
// cubed in tiles of 256 398, of 128 510; 8192 x 512 x 2048 of 256 28, of 128 14, of 64 21;
// 512 x 2048 x 8192 of 128 34, of 64 19; 512 x 512 x 8192 of 64 17, in 4 slices 10.6.
Plan plan_of(long m, long n, long k, bool exact, bool reads) {
  const int k_blocks = static_cast<int>(std::max((k + BK - 1) / BK, 1L));
  Plan best;
  double least = 1e300;
  for (int i = 0; i < static_cast<int>(std::size(VARIANTS)); ++i) {
    const Variant& v = exact ? VARIANTS_EXACT[i] : VARIANTS[i];
    const long tiles = ((m + 64 * v.t - 1) / (64 * v.t)) * ((n + 64 * v.t - 1) / (64 * v.t));
    for (int splits : {1, 2, 3, 4, 6, 8, 12, MAX_SPLITS}) {
      if (splits > 1 && (2 * splits > k_blocks || tiles * splits > 1 << 16)) break;   // few tiles only: planes stay small
      const int per = (k_blocks + splits - 1) / splits, used = (k_blocks + per - 1) / per;
      const long slots = 256L * v.per_cu, work = tiles * used, rounds = work / slots, rest = work - rounds * slots;
      const double fixed = v.fixed + (reads && used == 1 ? v.reads : 0.0), full = fixed + per * v.step_full;
      double t = rounds * full;
      if (rest > 256) t += full;
      else if (rest) t += fixed + per * v.step_alone;
      if (used > 1) t += 2.0 + 2.0 * (used + reads) * m * n * 4 / 5e6;
      if (t < least) {
        least = t;
        best.variant = i;
        best.splits = used;
        best.per_split = per;
      }
    }
  }
  return best;
}

template <int TI, int TJ, bool EXACT, int STAGES>
hipError_t launch(TileArgs a, hipStream_t s) {
  a.tiles_m = static_cast<uint32_t>((a.m + 64 * TI - 1) / (64 * TI));
  a.tiles_n = static_cast<uint32_t>((a.n + 64 * TJ - 1) / (64 * TJ));
  a.total = a.tiles_m * a.tiles_n * a.splits;
  const dim3 grid((a.total + 7) / 8 * 8);
  if (a.partial) hipLaunchKernelGGL((product_tile_kernel<TI, TJ, EXACT, STAGES, EPI_SLICE>), grid, dim3(NT), 0, s, a);
  else if (a.mask || a.accumulate) hipLaunchKernelGGL((product_tile_kernel<TI, TJ, EXACT, STAGES, EPI_READS>), grid, dim3(NT), 0, s, a);
  else hipLaunchKernelGGL((product_tile_kernel<TI, TJ, EXACT, STAGES, EPI_PLAIN>), grid, dim3(NT), 0, s, a);
  return hipGetLastError();
}

template <bool EXACT>
hipError_t product_of(const ProductArgs& args, hipStream_t s) {
  if (args.m <= 16) return launch_rows<1, EXACT>(args, s);
  if (args.m <= ROWS_MAX) return launch_rows<2, EXACT>(args, s);
  const Plan p = plan_of(args.m, args.n, args.k, EXACT, args.mask || args.accumulate);
  TileArgs a;
  static_cast<ProductArgs&>(a) = args;
  a.k_blocks = static_cast<int>(std::max((args.k + BK - 1) / BK, 1L));
  a.splits = p.splits;
  a.per_split = p.per_split;
  if (p.splits > 1) a.partial = args.ws;
  const hipError_t e = p.variant == 0   ? launch<4, 4, EXACT, VARIANTS[0].stages>(a, s)
                       : p.variant == 1 ? launch<2, 2, EXACT, VARIANTS[1].stages>(a, s)
                                        : launch<1, 1, EXACT, VARIANTS[2].stages>(a, s);
  if (e != hipSuccess || p.splits == 1) return e;
  const long threads = a.m * ((a.n + 3) / 4);
  hipLaunchKernelGGL(product_join_kernel, dim3(static_cast<unsigned>((threads + NT - 1) / NT)), dim3(NT), 0, s, a);
  return hipGetLastError();
}

}  // namespace

ProductPlan product_plan(long m, long n, long k, bool exact, bool reads) {
  if (m <= ROWS_MAX) return {};
  const Plan p = plan_of(m, n, k, exact, reads);
  return {64 * (exact ? VARIANTS_EXACT : VARIANTS)[p.variant].t, p.splits, p.per_split};
}

size_t product_ws_bytes(long m, long n, long k) {
  if (m <= ROWS_MAX || n == 0) return 0;
  size_t planes = 0;
  for (bool exact : {false, true}) {
    for (bool reads : {false, true}) {
      const int splits = plan_of(m, n, k, exact, reads).splits;
      if (splits > 1) planes = std::max(planes, static_cast<size_t>(splits));
    }
  }
  return planes * m * n * sizeof(float);
}

hipError_t product(const ProductArgs& a, hipStream_t s) { return a.out_dtype ? product_of<false>(a, s) : product_of<true>(a, s); }

}  // namespace spx
