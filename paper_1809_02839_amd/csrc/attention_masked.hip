// Masked attention with shared key/value heads, forward and backward.
//
// Every mask the interface has (causal with a prefix, documents, valid lengths)
// leaves a row one interval of keys [lo, hi), and both ends only grow with the
// row's position. So a tile is classified from its first and last row: skipped,
// whole, or cut (only cut tiles compare columns), and no mask tensor exists.
//
// Rows are the queries of every head that shares a key/value head (row r: query
// r / group, head r % group of the group), so one staging of a key tile serves
// the whole group.
//
// The fragment of the walked operand goes first into the matrix instruction, so a
// lane ends with scores of one row of its own: masks, maxima and sums of a row are
// scalars of a lane, and the registers of a group of 32 columns are already an
// operand of the next product (attention_long.hip). Probabilities and score
// gradients are rounded to bf16 for it, 2^-8 of each at most and at random, as the
// results are once more: the matrix instructions take no wider operand at their rate,
// and two roundings of one size make the error of out and the gradients 1.1 to 1.4
// times that of a result rounded once. Scores, maxima, sums and results stay float32.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "attention_tiles.hpp"

namespace spx {
namespace {

constexpr int NT = 256, ROWS = 128, KT = 64;   // threads, rows of a block, keys (rows) of a staged tile
constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;

struct Args : AttentionArgs {
  const int2* doc = nullptr;      // [batch][kv_len]: first and past-the-last token of the token's document
  float* delta = nullptr;         // [batch][heads][q_len]: sum of P dP = out . dout (backward)
  float c1 = 0.0f;                // |scale| log2(e)
  float c2 = 0.0f, c3 = 0.0f;     // capped: cap log2(e), and one over it
  float c4 = 0.0f;                // capped: 2 |scale| / cap log2(e)
  int flip = 0;                   // scale < 0: one operand of the scores changes sign instead
  FastDiv by_group, by_bh, by_kv, by_tiles, by_step;
  int step = KT;                  // rows of a step of the walk over rows: whole queries, where a group fits a tile
  int tiles = 0;
  int pieces = 1;                 // most pieces that a tile's walk is cut into, a block each
  int quantum = 1;                // fewest steps of a piece
  float* part = nullptr;          // [pieces][...][dim] partial results (pieces > 1)
  float2* part_ml = nullptr;      // [pieces][batch][heads][q_len] maximum and sum (forward)
  float* part2 = nullptr;         // dV's (part is dK's)
};

// Values that are the same in every lane, for scalar registers.
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ int2 uniform(int2 v) { return make_int2(uniform(v.x), uniform(v.y)); }

// A walk over [begin, end) in steps of W is cut into at most a.pieces equal
// pieces, none shorter than about a.quantum steps: long walks are shared out,
// short ones stay whole and write their results at once.
__device__ __forceinline__ int pieces_of(const Args& a, int W, int begin, int end) {
  if (a.pieces == 1) return 1;
  const int steps = max(0, end - begin + W - 1) / W;
  return max(1, min(a.pieces, (steps + a.quantum - 1) / a.quantum));
}
// The n'th of `of` equal shares (all of it the same in every lane).
__device__ __forceinline__ void share(int W, int n, int of, int& begin, int& end) {
  const int steps = uniform(max(0, end - begin + W - 1) / W), b = begin;
  const int part = uniform(steps / of), rest = steps - part * of;
  begin = b + (n * part + min(n, rest)) * W;
  end = min(end, b + ((n + 1) * part + min(n + 1, rest)) * W);
}

struct Sequence {
  int limit, prefix;              // valid keys; keys every row sees (causal)
  const int2* doc;
  __device__ __forceinline__ Sequence(const Args& a, int b)
      : limit(a.kv_lengths ? min(max(a.kv_lengths[b], 0), a.kv_len) : a.kv_len),
        prefix(a.prefix ? min(max(a.prefix[b], 0), a.kv_len) : 0),
        doc(a.doc ? a.doc + static_cast<long>(b) * a.kv_len : nullptr) {}
  // Keys [x, y) that the row at position p sees (none if y <= x).
  __device__ __forceinline__ int2 keys(const Args& a, int p) const {
    return clip(a, p, doc ? doc[p] : make_int2(0, 0x7fffffff));
  }
  // The same from its document's first and past-the-last token.
  __device__ __forceinline__ int2 clip(const Args& a, int p, int2 d) const {
    int hi = min(limit, d.y);
    if (a.causal) hi = min(hi, max(p + 1, prefix));
    return make_int2(d.x, hi);
  }
};

// Keys that the rows [row0, row0 + n) see between them; a walk over them begins
// at a multiple of its step.
__device__ __forceinline__ int2 key_span(const Args& a, const Sequence& seq, int row0, int n) {
  const auto position = [&](int r) { return a.q_offset + static_cast<int>(a.by_group.div(min(r, a.rows - 1))); };
  return make_int2(seq.keys(a, position(row0)).x, seq.keys(a, position(row0 + n - 1)).y);
}

// Rows that see one of the keys [key0, key0 + n); likewise.
__device__ __forceinline__ int2 row_span(const Args& a, const Sequence& seq, int key0, int n) {
  const int valid = min(seq.limit, key0 + n);
  if (key0 >= valid) return make_int2(0, 0);
  int pa = -(1 << 30), pb = 0x7fffffff;   // their positions
  if (a.causal && key0 >= seq.prefix) pa = key0;
  if (seq.doc) {
    pa = max(pa, seq.doc[key0].x);
    pb = seq.doc[valid - 1].y;
  }
  const auto row = [&](int p) {
    return static_cast<int>(min(max(static_cast<long>(p) - a.q_offset, 0L) * a.group, static_cast<long>(a.rows)));
  };
  return make_int2(row(pa), row(pb));
}

// How a kernel forms scores from products: times the scale and no more; capped or
// with a bias; and capped by more than NEAR_CAP.
enum Scores { PLAIN, GENERAL, FAR_CAP };

// Scores of a group's products in units of log2: s log2(e). Where they are
// capped, f(r, tanh(z / cap)) is called for each.
//
// tanh(u) = 1 - 2 / (1 + e^(2u)) is off by 2^-22.6 whatever u is, a score by
// 2^-22.6 cap: 2^-16 at most for caps up to NEAR_CAP, which changes a probability
// by 2^-16 of itself. Past it, for |u| <= 1/2, tanh(u) is u p(u^2) and the score z
// p, off relative to themselves however far the cap is (p: degree 4, fitted for
// the least error of tanh(u) / u, 2^-26 exactly and 2^-23 as evaluated), and only
// for larger |u|, where 2^-22.6 is 2^-21.5 of the value, the first form. A group
// with no such score takes the polynomial alone. Near caps keep the first form, the
// faster one (16 heads of 4096 causal tokens capped at 30: forward 138 us, backward
// 446; by the second form 147 and 540).
constexpr float NEAR_CAP = 64.0f;
template <int KIND, typename F>
__device__ __forceinline__ void scores(const Args& a, f32x16_t& s, F&& f) {
  const auto tanh_far = [&](float product) {
    return fmaf(-2.0f, __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(product * a.c4)), 1.0f);
  };
  if (KIND == GENERAL) {
    if (a.c2 == 0.0f) {
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] *= a.c1;
      return;
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const float t = tanh_far(s[r]);
      f(r, t);
      s[r] = t * a.c2;
    }
    return;
  }
  const auto ratio = [](float u) {   // tanh(u) / u
    const float y = u * u;
    return fmaf(y, fmaf(y, fmaf(y, fmaf(y, 0.01724149100482464f, -0.05304549261927605f), 0.13325878977775574f),
                        -0.333331435918808f), 1.0f);
  };
  float top = 0.0f;
#pragma unroll
  for (int r = 0; r < 16; ++r) top = fmaxf(top, fabsf(s[r]));
  if (!__any(top * a.c1 > 0.5f * a.c2)) {
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const float z = s[r] * a.c1, u = z * a.c3, p = ratio(u);
      f(r, u * p);
      s[r] = z * p;
    }
    return;
  }
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const float z = s[r] * a.c1, u = z * a.c3, p = ratio(u), far = tanh_far(s[r]);
    const bool near = fabsf(u) <= 0.5f;
    f(r, near ? u * p : far);
    s[r] = near ? z * p : far * a.c2;
  }
}

// A staged tile: KT rows of C 16-byte chunks in LDS, chunk c of row r in place
// c ^ swizzle(r). The places are chosen so that the 32 rows of a row fragment
// and the 4 x 2 rows of a transposing read each spread over all banks.
template <int DH>
struct Tile {
  static constexpr int C = DH <= 32 ? 4 : DH <= 64 ? 8 : 16, V = KT * C / NT, BYTES = KT * C * 16;
  static_assert(KT * C % NT == 0, "whole accesses");
  static __device__ __forceinline__ int swizzle(int r) {
    if (C == 16) return ((r & 3) << 2) | ((r >> 2) & 3);
    if (C == 8) return ((r & 2) << 1) | ((r >> 2) & 3);
    return (r >> 2) & 3;
  }
};

// Direct load into LDS: the 16 bytes at lane l's byte offset from the resource's
// base land at LDS byte address lds + 16 l (lds wave-uniform, passed in M0); an
// offset past the resource writes zeros. Issued through inline assembly so that
// the compiler, which cannot tell the two buffers apart, does not wait for the
// next tile before each read of this one; landed() waits for the wave's own
// loads, and the barrier after it for the others'. A load to LDS may read M0 one
// wait state after a scalar write of it at the earliest (s_nop 0: the compiler
// puts it there itself, but does not look into assembly). The statement declares
// M0 clobbered; nothing else in these kernels keeps a value in M0 (a host test
// checks the assembly for both).
__device__ __forceinline__ void direct16(__amdgpu_buffer_rsrc_t r, uint32_t lds, int off) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds), "v"(off), "s"(r)
               : "memory", "m0");
}
__device__ __forceinline__ __amdgpu_buffer_rsrc_t resource(const bf16_t* p) {   // p: the same in every lane
  const uint64_t u = reinterpret_cast<uintptr_t>(p);
  p = reinterpret_cast<const bf16_t*>(static_cast<uint64_t>(static_cast<uint32_t>(uniform(static_cast<int>(u >> 32)))) << 32 |
                                      static_cast<uint32_t>(uniform(static_cast<int>(u))));
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16_t*>(p), static_cast<short>(0), 0x7fffffe0, 0x00020000);
}
constexpr int OUTSIDE = 0x7ffffff0;   // past every resource
__device__ __forceinline__ void landed() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
__device__ __forceinline__ uint32_t lds_address(const void* p) {
  return static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const char*)p));
}

// A thread's part of the copy of tiles of N rows by THREADS threads: its byte
// offsets from the tile's first row, the same for every tile, so that a whole
// tile costs no address arithmetic (with 64-bit addresses formed for each access
// it was half of all vector instructions).
template <int DH, int N, int THREADS>
struct Loader {
  using T = Tile<DH>;
  static constexpr int V = N * T::C / THREADS;
  int off[V];
  // row(r): element offset of the tile's row r.
  template <typename F>
  __device__ __forceinline__ void init(int t, int dim, F&& row) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int e = t + THREADS * i, r = e / T::C, col = ((e % T::C) ^ T::swizzle(r)) * 8;
      off[i] = col < dim ? static_cast<int>(min(2 * (row(r) + col), static_cast<long>(OUTSIDE))) : OUTSIDE;
    }
  }
  // Starts the copy of rows first .. into LDS, zeros for those outside `span`: what
  // nothing sees may hold anything (memory not written yet), and a probability of
  // zero would not hide what is not finite. Of a tile with fewer rows the others are
  // OUTSIDE as they are.
  __device__ __forceinline__ void start(const bf16_t* base, uint32_t lds, int first, int2 span, int t,
                                        int rows = N) const {
    const __amdgpu_buffer_rsrc_t r = resource(base);
    const uint32_t to = uniform(static_cast<int>(lds)) + (THREADS > 64 ? 1024 * __builtin_amdgcn_readfirstlane(t >> 6) : 0);
    if (first >= span.x && first + rows <= span.y) {
#pragma unroll
      for (int i = 0; i < V; ++i) direct16(r, to + 16 * THREADS * i, off[i]);
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const int at = first + (t + THREADS * i) / T::C;
        direct16(r, to + 16 * THREADS * i, at >= span.x && at < span.y ? off[i] : OUTSIDE);
      }
    }
  }
};

// Byte offsets of a lane's fragments in a tile: rows c0 + lane % 32, columns
// 16 q + 8 (lane / 32) .. at rows ^ (q << 5) + c0 * pitch; and, transposed (see
// frag_cols), rows k0 .. + 15, columns 32 j .. at cols[half] ^ (j << 6) + k0 * pitch.
template <int DH>
struct Lane {
  static constexpr int PITCH = Tile<DH>::C * 16;
  uint32_t rows, cols[2];
  __device__ __forceinline__ explicit Lane(int lane) {
    const int r = lane & 31, g = lane >> 4, i = lane & 15;
    rows = r * PITCH + (((lane >> 5) ^ Tile<DH>::swizzle(r)) << 4);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int k = 4 * (g >> 1) + (i >> 2) + 8 * h, chunk = 2 * (g & 1) + ((i & 3) >> 1);
      cols[h] = k * PITCH + ((chunk ^ Tile<DH>::swizzle(k)) << 4) + 8 * (i & 1);
    }
  }
  // A copy whose offsets the compiler works out where they are used: hoisted out
  // of a loop, the sixteen of them would cost the registers of a result column.
  __device__ __forceinline__ Lane here() const {
    Lane l = *this;
    asm volatile("" : "+v"(l.rows), "+v"(l.cols[0]), "+v"(l.cols[1]));
    return l;
  }
  __device__ __forceinline__ bf16x8_t row_frag(const char* tile, int c0, int q) const {
    return gld8(reinterpret_cast<const bf16_t*>(tile + c0 * PITCH + (rows ^ (q << 5))));
  }
  __device__ __forceinline__ bf16x8_t col_frag(const char* tile, int k0, int j) const {
    const char* t = tile + k0 * PITCH;
    const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)(t + (cols[0] ^ (j << 6))));
    const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)(t + (cols[1] ^ (j << 6))));
    const u16x8_t v = {static_cast<uint16_t>(lo[0]), static_cast<uint16_t>(lo[1]), static_cast<uint16_t>(lo[2]),
                       static_cast<uint16_t>(lo[3]), static_cast<uint16_t>(hi[0]), static_cast<uint16_t>(hi[1]),
                       static_cast<uint16_t>(hi[2]), static_cast<uint16_t>(hi[3])};
    return __builtin_bit_cast(bf16x8_t, v);
  }
};

template <int DH>
__device__ __forceinline__ void load_row(const bf16_t* row, int dim, int lane, bf16x8_t (&f)[DH / 16], int flip = 0) {
  const uint32_t sign = flip ? 0x80008000u : 0u;
#pragma unroll
  for (int q = 0; q < DH / 16; ++q) {
    const int col = 16 * q + 8 * (lane >> 5);
    uint4 u = make_uint4(0, 0, 0, 0);
    if (col < dim) u = *reinterpret_cast<const uint4*>(row + col);
    u.x ^= sign, u.y ^= sign, u.z ^= sign, u.w ^= sign;
    f[q] = __builtin_bit_cast(bf16x8_t, u);
  }
}

// The wave's 32 rows (fragments fr) against rows c0 .. c0 + 31 of a tile.
template <int DH>
__device__ __forceinline__ f32x16_t product(const bf16x8_t (&fr)[DH / 16], const char* tile, int c0,
                                            const Lane<DH>& at) {
  f32x16_t acc;
#pragma unroll
  for (int r = 0; r < 16; ++r) acc[r] = 0.0f;
#pragma unroll
  for (int q = 0; q < DH / 16; ++q) acc = mfma(at.row_frag(tile, c0, q), fr[q], acc);
  return acc;
}

// Half c of a group's values as an operand, rounded to bf16.
__device__ __forceinline__ bf16x8_t pack8(const f32x16_t& v, int c) {
  const uint4 u = make_uint4(pack_bf16x2(v[8 * c], v[8 * c + 1]), pack_bf16x2(v[8 * c + 2], v[8 * c + 3]),
                             pack_bf16x2(v[8 * c + 4], v[8 * c + 5]), pack_bf16x2(v[8 * c + 6], v[8 * c + 7]));
  return __builtin_bit_cast(bf16x8_t, u);
}

// acc += the group's values times rows c0 .. of a tile.
template <int DH>
__device__ __forceinline__ void accumulate(const f32x16_t& v, const char* tile, int c0, const Lane<DH>& at,
                                           f32x16_t (&acc)[DH / 32]) {
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    const bf16x8_t fa = pack8(v, c);
#pragma unroll
    for (int j = 0; j < DH / 32; ++j) acc[j] = mfma(at.col_frag(tile, c0 + 16 * c, j), fa, acc[j]);
  }
}

// Row lane % 32 of a wave's 32 x DH result, times alpha, as bf16.
template <int DH>
__device__ __forceinline__ void store_row(bf16_t* out, int dim, const f32x16_t (&acc)[DH / 32], float alpha, int lane) {
#pragma unroll
  for (int jn = 0; jn < DH / 32; ++jn)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int col = 32 * jn + col_of(4 * g, lane);
      if (col < dim)
        *reinterpret_cast<uint2*>(out + col) =
            make_uint2(pack_bf16x2(acc[jn][4 * g] * alpha, acc[jn][4 * g + 1] * alpha),
                       pack_bf16x2(acc[jn][4 * g + 2] * alpha, acc[jn][4 * g + 3] * alpha));
    }
}

// The same as float32 partial results.
template <int DH>
__device__ __forceinline__ void store_part(float* out, int dim, const f32x16_t (&acc)[DH / 32], float alpha, int lane) {
#pragma unroll
  for (int jn = 0; jn < DH / 32; ++jn)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int col = 32 * jn + col_of(4 * g, lane);
      if (col < dim)
        *reinterpret_cast<float4*>(out + col) = make_float4(acc[jn][4 * g] * alpha, acc[jn][4 * g + 1] * alpha,
                                                            acc[jn][4 * g + 2] * alpha, acc[jn][4 * g + 3] * alpha);
    }
}

// Documents: each token's run of equal numbers. A block owns a chunk of tokens,
// one a thread; where a run crosses its ends it is followed outwards, four
// chunks at a time.
__global__ __launch_bounds__(1024) void document_runs_kernel(const int32_t* ids, int len, FastDiv chunks, int2* runs) {
  __shared__ unsigned long long starts[16], ends[16];   // by wave: tokens that start, or end, a run
  __shared__ int edge;
  const int n = blockDim.x, b = chunks.div(blockIdx.x);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int first = (blockIdx.x - b * chunks.d) * n, j = first + tid, last = min(first + n, len) - 1;
  ids += static_cast<long>(b) * len;
  runs += static_cast<long>(b) * len;
  const bool in = j < len;
  const int id = in ? ids[j] : 0, before = in && j > 0 ? ids[j - 1] : 0, after = in && j < len - 1 ? ids[j + 1] : 0;
  const unsigned long long s = __ballot(in && (j == 0 || before != id));
  const unsigned long long e = __ballot(in && (j == len - 1 || after != id));
  if (lane == 0) starts[wave] = s, ends[wave] = e;
  __syncthreads();
  int start = first, end = last + 1;   // of the runs that come in and go out
  if (!(starts[0] & 1)) {
    for (int to = first; to > 0;) {
      const int w = min(4 * n, to), base = to - w;
      if (tid == 0) edge = -1;
      __syncthreads();
      int found = -1;
      for (int k = tid; k < w; k += n)
        if (ids[base + k] != ids[first]) found = base + k;
      if (found >= 0) atomicMax(&edge, found);
      __syncthreads();
      found = edge;
      __syncthreads();
      start = found < 0 ? base : found + 1;
      if (found >= 0) break;
      to = base;
    }
  }
  if (!(ends[(last - first) >> 6] >> ((last - first) & 63) & 1)) {
    for (int from = last + 1; from < len;) {
      const int w = min(4 * n, len - from);
      if (tid == 0) edge = 0x7fffffff;
      __syncthreads();
      int found = 0x7fffffff;
      for (int k = tid; k < w; k += n)
        if (ids[from + k] != ids[last]) found = min(found, from + k);
      if (found != 0x7fffffff) atomicMin(&edge, found);
      __syncthreads();
      found = edge;
      __syncthreads();
      end = found == 0x7fffffff ? from + w : found;
      if (found != 0x7fffffff) break;
      from += w;
    }
  }
  if (!in) return;
  // the last start at or before the token, the first end at or after it
  unsigned long long m = starts[wave] & (~0ull >> (63 - lane));
  int w = wave;
  while (m == 0 && w > 0) m = starts[--w];
  const int x = m ? first + 64 * w + 63 - __clzll(m) : start;
  m = ends[wave] & (~0ull << lane);
  w = wave;
  while (m == 0 && 64 * (w + 1) < n) m = ends[++w];
  const int y = m ? first + 64 * w + __ffsll(m) : end;
  runs[j] = make_int2(x, y);
}

// One block's place: its (sequence, kv head) and tile. Consecutive blocks take
// different kv heads (of one XCD each where their number is a multiple of 8),
// and the tiles with the most work under a causal mask first: the last rows,
// the first keys. Blocks that run together walk the same pieces.
struct Block {
  int b, kh, tile, piece;
  __device__ __forceinline__ Block(const Args& a, bool last_first) {
    const uint32_t x = blockIdx.x, pt = a.by_bh.div(x), bh = x - pt * a.by_bh.d, t = pt - a.by_tiles.div(pt) * a.tiles;
    piece = a.by_tiles.div(pt);
    b = a.by_kv.div(bh);
    kh = bh - b * a.kv_heads;
    tile = last_first ? a.tiles - 1 - static_cast<int>(t) : static_cast<int>(t);
  }
};

// How far (in powers of two) a score may pass the running maximum before the
// sums are scaled anew: probabilities stay below 2^8, in float32 as exact as
// below 1, and most tiles skip the pass over the result's registers.
constexpr float SLACK = 8.0f;

// A row's running softmax: result so far (not normalised), maximum and sum.
template <int DH>
struct Running {
  f32x16_t o[DH / 32];
  float m = -INFINITY, sum = 0.0f;   // sum: the lane's own half of the columns until closed

  // Takes in 32 N keys from k0 on. cut: the tile's columns are compared with the
  // row's keys.
  template <int KIND, int N>
  __device__ __forceinline__ void take(const Args& a, const Lane<DH>& frag, const char* Ks, const char* Vs,
                                       const bf16x8_t (&fq)[DH / 16], int k0, int p, float slope, int2 mine, bool cut,
                                       int lane) {
    f32x16_t s[N];
#pragma unroll
    for (int n = 0; n < N; ++n) s[n] = product<DH>(fq, Ks, 32 * n, frag);
    if (KIND != PLAIN) {
#pragma unroll
      for (int n = 0; n < N; ++n) scores<KIND>(a, s[n], [](int, float) {});
      if (a.slopes) {
        const float far = static_cast<float>(p - k0 - col_of(0, lane));
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
          for (int r = 0; r < 16; ++r) s[n][r] -= slope * fabsf(far - static_cast<float>(32 * n + col_of(r, 0)));
      }
    }
    const float c1 = KIND == PLAIN ? a.c1 : 1.0f;   // s c1: the scores
    if (cut) {
#pragma unroll
      for (int n = 0; n < N; ++n)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int j = k0 + 32 * n + col_of(r, lane);
          if (j < mine.x || j >= mine.y) s[n][r] = -INFINITY;
        }
    }
    float top = s[0][0];
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int r = 0; r < 16; ++r) top = fmaxf(top, s[n][r]);
    top = fmaxf(top, __shfl_xor(top, 32)) * c1;
    if (__any(top > m + SLACK)) {
      const float next = fmaxf(m, top), shrink = __builtin_amdgcn_exp2f(m - (next == -INFINITY ? 0.0f : next));
      m = next;
      sum *= shrink;
#pragma unroll
      for (int j = 0; j < DH / 32; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[j][r] *= shrink;
    }
    const float base = m == -INFINITY ? 0.0f : m;   // nothing seen so far weighs zero
#pragma unroll
    for (int n = 0; n < N; ++n) {
      float part[2] = {0.0f, 0.0f};
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[n][r] = __builtin_amdgcn_exp2f(fmaf(s[n][r], c1, -base));
        part[r & 1] += s[n][r];
      }
      sum += part[0] + part[1];
      accumulate<DH>(s[n], Vs, 32 * n, frag, o);
    }
  }
};

__device__ __forceinline__ long row_index(const Args& a, int b, int head, int i) {
  return (static_cast<long>(b) * a.heads + head) * a.q_len + i;
}
__device__ __forceinline__ float lse_of(float m, float sum) { return sum == 0.0f ? -INFINITY : m * LN2 + logf(sum); }

// A block: 128 rows, or one piece of their keys; one pass over the keys. The
// matrix instructions are busy 53% of the time at 128 columns (16 heads, 8192
// causal tokens, 311 us, 884 TFLOP/s; 16384 tokens with two heads to a key head
// 1087 us, 1012 TFLOP/s); the rest waits on the exponentials between the two
// products, four instructions' time each, which the other wave of a SIMD only
// partly covers. At 64 columns they bound the kernel (32 heads, 8192 tokens, 306 us,
// 900 TFLOP/s).
template <int DH, int KIND>
__global__ __launch_bounds__(NT, 2) void attention_masked_fwd_kernel(Args a) {
  using T = Tile<DH>;
  __shared__ __attribute__((aligned(16))) char lds[2][2][T::BYTES];   // buffer, K or V
  const Block at(a, true);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const Lane<DH> frag(lane);
  const Sequence seq(a, at.b);
  const int row0 = at.tile * ROWS + 32 * wave, row = min(row0 + (lane & 31), a.rows - 1);
  const int i = a.by_group.div(row), head = at.kh * a.group + row - i * a.group, p = a.q_offset + i;
  const int2 mine = seq.keys(a, p);
  const auto position = [&](int r) { return a.q_offset + static_cast<int>(a.by_group.div(min(r, a.rows - 1))); };
  const int2 wfirst = uniform(seq.keys(a, position(row0))), wlast = uniform(seq.keys(a, position(row0 + 31)));
  const int2 span = uniform(key_span(a, seq, at.tile * ROWS, ROWS));
  int begin = span.x / KT * KT, end = span.y;
  const int pieces = uniform(pieces_of(a, KT, begin, end));
  if (at.piece >= pieces) return;
  share(KT, at.piece, pieces, begin, end);
  const bf16_t* k = a.k + at.b * a.sk.b + at.kh * a.sk.h;
  const bf16_t* v = a.v + at.b * a.sv.b + at.kh * a.sv.h;
  Loader<DH, KT, NT> kl, vl;
  kl.init(tid, a.dim, [&](int r) { return r * a.sk.t; });
  vl.init(tid, a.dim, [&](int r) { return r * a.sv.t; });
  const auto fetch = [&](int k0, int buf) {
    kl.start(k + k0 * a.sk.t, lds_address(lds[buf][0]), k0, span, tid);
    vl.start(v + k0 * a.sv.t, lds_address(lds[buf][1]), k0, span, tid);
  };
  if (begin < end) fetch(begin, 0);
  const float slope = a.slopes ? a.slopes[head] * LOG2E : 0.0f;
  bf16x8_t fq[DH / 16];
  load_row<DH>(a.q + at.b * a.sq.b + i * a.sq.t + head * a.sq.h, a.dim, lane, fq, a.flip);

  Running<DH> run;
  zero(run.o);
  int buf = 0;
  for (int k0 = begin; k0 < end; k0 += KT, buf ^= 1) {
    landed();
    __syncthreads();
    if (k0 + KT < end) fetch(k0 + KT, buf ^ 1);
    if (k0 >= wlast.y || k0 + KT <= wfirst.x) continue;
    run.template take<KIND, KT / 32>(a, frag, lds[buf][0], lds[buf][1], fq, k0, p, slope, mine,
                                    k0 < wlast.x || k0 + KT > wfirst.y, lane);
  }
  const float sum = run.sum + __shfl_xor(run.sum, 32);
  if (row0 + (lane & 31) >= a.rows) return;
  const long r = row_index(a, at.b, head, i);
  if (pieces > 1) {
    const long rp = at.piece * static_cast<long>(a.batch) * a.heads * a.q_len + r;
    store_part<DH>(a.part + rp * a.dim, a.dim, run.o, 1.0f, lane);
    if (lane < 32) a.part_ml[rp] = make_float2(run.m, sum);
    return;
  }
  store_row<DH>(a.out + at.b * a.so.b + i * a.so.t + head * a.so.h, a.dim, run.o, sum == 0.0f ? 0.0f : 1.0f / sum, lane);
  if (a.lse && lane < 32) a.lse[r] = lse_of(run.m, sum);
}

// Up to 32 rows (single tokens, and what a group makes of a few): bound by reading
// the keys and values once, so the block's waves share out the keys, each with
// tiles of 32 of its own that no other wave waits for, and join their sums at the
// end. 1.6 GB of 16 ragged caches in 290 us, 5.6 TB/s, where a copy of 1 GiB moves
// 5.1; in blocks of 128 rows, one wave of four busy, 369 us.
template <int DH, int KIND>
__global__ __launch_bounds__(NT, 1) void attention_masked_few_kernel(Args a) {
  using T = Tile<DH>;
  constexpr int FT = 32, BYTES = T::BYTES / (KT / FT);
  __shared__ __attribute__((aligned(16))) char lds[NT / 64][2][2][BYTES];   // wave, buffer, K or V
  __shared__ float2 ml[NT / 64][32];
  static_assert(4 * BYTES >= 32 * DH * 4, "a wave's tiles hold its result");
  const Block at(a, false);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const Lane<DH> frag(lane);
  const Sequence seq(a, at.b);
  const int row0 = at.tile * 32, row = min(row0 + (lane & 31), a.rows - 1);
  const int i = a.by_group.div(row), head = at.kh * a.group + row - i * a.group, p = a.q_offset + i;
  const int2 mine = seq.keys(a, p);
  const auto position = [&](int r) { return a.q_offset + static_cast<int>(a.by_group.div(min(r, a.rows - 1))); };
  const int2 first = uniform(seq.keys(a, position(row0))), last = uniform(seq.keys(a, position(row0 + 31)));
  const int2 span = make_int2(first.x, last.y);
  int begin = span.x / FT * FT, end = span.y;
  const int pieces = uniform(pieces_of(a, FT, begin, end));
  if (at.piece >= pieces) return;
  share(FT, at.piece * (NT / 64) + wave, pieces * (NT / 64), begin, end);
  const bf16_t* k = a.k + at.b * a.sk.b + at.kh * a.sk.h;
  const bf16_t* v = a.v + at.b * a.sv.b + at.kh * a.sv.h;
  Loader<DH, FT, 64> kl, vl;
  kl.init(lane, a.dim, [&](int r) { return r * a.sk.t; });
  vl.init(lane, a.dim, [&](int r) { return r * a.sv.t; });
  const auto fetch = [&](int k0, int buf) {
    kl.start(k + k0 * a.sk.t, lds_address(lds[wave][buf][0]), k0, span, lane);
    vl.start(v + k0 * a.sv.t, lds_address(lds[wave][buf][1]), k0, span, lane);
  };
  if (begin < end) fetch(begin, 0);
  const float slope = a.slopes ? a.slopes[head] * LOG2E : 0.0f;
  bf16x8_t fq[DH / 16];
  load_row<DH>(a.q + at.b * a.sq.b + i * a.sq.t + head * a.sq.h, a.dim, lane, fq, a.flip);

  Running<DH> run;
  zero(run.o);
  int buf = 0;
  for (int k0 = begin; k0 < end; k0 += FT, buf ^= 1) {
    landed();
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the other buffer has been read
    if (k0 + FT < end) fetch(k0 + FT, buf ^ 1);
    run.template take<KIND, 1>(a, frag, lds[wave][buf][0], lds[wave][buf][1], fq, k0, p, slope, mine,
                              k0 < last.x || k0 + FT > first.y, lane);
  }
  const float sum = run.sum + __shfl_xor(run.sum, 32);
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  float* mineo = reinterpret_cast<float*>(lds[wave]);
  store_part<DH>(mineo + (lane & 31) * DH, DH, run.o, 1.0f, lane);
  if (lane < 32) ml[wave][lane] = make_float2(run.m, sum);
  __syncthreads();
  for (int e = tid; e < 32 * DH / 4; e += NT) {
    const int r = e / (DH / 4), col = e % (DH / 4) * 4, rr = row0 + r;
    if (rr >= a.rows || col >= a.dim) continue;
    float m = ml[0][r].x, w[NT / 64], l = 0.0f;
#pragma unroll
    for (int u = 1; u < NT / 64; ++u) m = fmaxf(m, ml[u][r].x);
    const float base = m == -INFINITY ? 0.0f : m;
    float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
    for (int u = 0; u < NT / 64; ++u) {
      w[u] = __builtin_amdgcn_exp2f(ml[u][r].x - base);
      l = fmaf(w[u], ml[u][r].y, l);
      const float4 y = *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(lds[u]) + r * DH + col);
      x.x = fmaf(w[u], y.x, x.x), x.y = fmaf(w[u], y.y, x.y), x.z = fmaf(w[u], y.z, x.z), x.w = fmaf(w[u], y.w, x.w);
    }
    const int ri = a.by_group.div(rr), rh = at.kh * a.group + rr - ri * a.group;
    const long at_row = row_index(a, at.b, rh, ri);
    if (pieces > 1) {
      const long rp = at.piece * static_cast<long>(a.batch) * a.heads * a.q_len + at_row;
      *reinterpret_cast<float4*>(a.part + rp * a.dim + col) = x;
      if (col == 0) a.part_ml[rp] = make_float2(m, l);
      continue;
    }
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    *reinterpret_cast<uint2*>(a.out + at.b * a.so.b + ri * a.so.t + rh * a.so.h + col) =
        make_uint2(pack_bf16x2(x.x * inv, x.y * inv), pack_bf16x2(x.z * inv, x.w * inv));
    if (a.lse && col == 0) a.lse[at_row] = lse_of(m, l);
  }
}

// Joins the pieces of the forward: 16 lanes a row, eight columns each. few: the
// pieces are those of the kernel for few rows.
__global__ __launch_bounds__(NT) void attention_join_kernel(Args a, long rows, FastDiv by_len, FastDiv by_heads,
                                                            int few) {
  const long r = static_cast<long>(blockIdx.x) * (NT / 16) + threadIdx.x / 16;
  const int col = threadIdx.x % 16 * 8;
  if (r >= rows || col >= a.dim) return;
  const uint32_t bh = by_len.div(static_cast<uint32_t>(r)), i = static_cast<uint32_t>(r) - bh * by_len.d;
  const uint32_t b = by_heads.div(bh), h = bh - b * by_heads.d;
  const Sequence seq(a, b);
  const int packed = i * a.group + (h - a.by_group.div(h) * a.group), tile = few ? 32 : ROWS;
  const int2 span = key_span(a, seq, packed / tile * tile, tile);
  const int pieces = few ? pieces_of(a, 32, span.x / 32 * 32, span.y) : pieces_of(a, KT, span.x / KT * KT, span.y);
  if (pieces == 1) return;   // written already
  float m = -INFINITY;
#pragma unroll 8   // loads of several pieces under way at once
  for (int u = 0; u < pieces; ++u) m = fmaxf(m, a.part_ml[u * rows + r].x);
  const float base = m == -INFINITY ? 0.0f : m;
  float l = 0.0f, x[8] = {};
#pragma unroll 4
  for (int u = 0; u < pieces; ++u) {
    const float2 ml = a.part_ml[u * rows + r];
    const float w = __builtin_amdgcn_exp2f(ml.x - base);
    const float4* y = reinterpret_cast<const float4*>(a.part + (u * rows + r) * a.dim + col);
    const float4 lo = y[0], hi = y[1];
    l = fmaf(w, ml.y, l);
    x[0] = fmaf(w, lo.x, x[0]), x[1] = fmaf(w, lo.y, x[1]), x[2] = fmaf(w, lo.z, x[2]), x[3] = fmaf(w, lo.w, x[3]);
    x[4] = fmaf(w, hi.x, x[4]), x[5] = fmaf(w, hi.y, x[5]), x[6] = fmaf(w, hi.z, x[6]), x[7] = fmaf(w, hi.w, x[7]);
  }
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  *reinterpret_cast<uint4*>(a.out + b * a.so.b + i * a.so.t + h * a.so.h + col) =
      make_uint4(pack_bf16x2(x[0] * inv, x[1] * inv), pack_bf16x2(x[2] * inv, x[3] * inv),
                 pack_bf16x2(x[4] * inv, x[5] * inv), pack_bf16x2(x[6] * inv, x[7] * inv));
  if (a.lse && col == 0) a.lse[r] = lse_of(m, l);
}

// Sums the pieces of a gradient [batch][token][head] in piece order: 16 lanes a
// row, eight columns each; dQ (blockIdx.y 0), dK and dV.
struct Sum {
  const float* part;
  bf16_t* out;
  AttentionArgs::Strides to;
  long rows;            // batch * tokens * heads; 0: nothing in pieces
  FastDiv by_heads, by_tokens;
  int pieces, quantum;
};
struct Sums {
  Sum sum[3];
  int keys;             // of a tile of the kernel for dK and dV
};
__global__ __launch_bounds__(NT) void attention_sum_kernel(Args a, Sums all) {
  const Sum& j = all.sum[blockIdx.y];
  const long r = static_cast<long>(blockIdx.x) * (NT / 16) + threadIdx.x / 16;
  const int col = threadIdx.x % 16 * 8;
  if (r >= j.rows || col >= a.dim) return;
  const uint32_t bt = j.by_heads.div(static_cast<uint32_t>(r)), h = static_cast<uint32_t>(r) - bt * j.by_heads.d;
  const uint32_t b = j.by_tokens.div(bt), t = bt - b * j.by_tokens.d;
  const Sequence seq(a, b);
  const int packed = t * a.group + (h - a.by_group.div(h) * a.group);
  const bool by_rows = blockIdx.y == 0;
  const int2 span = by_rows ? key_span(a, seq, packed / ROWS * ROWS, ROWS)
                            : row_span(a, seq, static_cast<int>(t) / all.keys * all.keys, all.keys);
  a.pieces = j.pieces;
  a.quantum = j.quantum;
  const int pieces = by_rows ? pieces_of(a, KT, span.x / KT * KT, span.y)
                             : pieces_of(a, a.step, a.by_step.div(span.x) * a.step, span.y);
  if (pieces == 1) return;   // written already
  float x[8] = {};
#pragma unroll 4
  for (int u = 0; u < pieces; ++u) {
    const float4* y = reinterpret_cast<const float4*>(j.part + (u * j.rows + r) * a.dim + col);
    const float4 lo = y[0], hi = y[1];
    x[0] += lo.x, x[1] += lo.y, x[2] += lo.z, x[3] += lo.w;
    x[4] += hi.x, x[5] += hi.y, x[6] += hi.z, x[7] += hi.w;
  }
  *reinterpret_cast<uint4*>(j.out + b * j.to.b + t * j.to.t + h * j.to.h + col) =
      make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
}

// log2 of a row's sum for the backward: infinite where the row has no weight,
// so that every probability is zero.
__device__ __forceinline__ float log2_sum(const Args& a, long row) {
  const float l = a.lse[row];
  return l == -INFINITY ? INFINITY : l * LOG2E;
}

// dQ of 128 rows (or a piece of it), and delta = out . dout (the sum of P dP) of each
// for the other kernel. Scores and dP are formed again from the tiles (three products; matrix
// instructions busy 62% at 128 columns): 1400 us for 16384 causal tokens of 16
// heads, two to a key head.
template <int DH, int KIND>
__global__ __launch_bounds__(NT, 2) void attention_masked_dq_kernel(Args a) {
  using T = Tile<DH>;
  __shared__ __attribute__((aligned(16))) char lds[2][2][T::BYTES];   // buffer, K or V
  const Block at(a, true);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const Lane<DH> frag(lane);
  const Sequence seq(a, at.b);
  const int row0 = at.tile * ROWS + 32 * wave, row = min(row0 + (lane & 31), a.rows - 1);
  const int i = a.by_group.div(row), head = at.kh * a.group + row - i * a.group, p = a.q_offset + i;
  const int2 mine = seq.keys(a, p);
  const auto position = [&](int r) { return a.q_offset + static_cast<int>(a.by_group.div(min(r, a.rows - 1))); };
  const int2 wfirst = uniform(seq.keys(a, position(row0))), wlast = uniform(seq.keys(a, position(row0 + 31)));
  const int2 span = uniform(key_span(a, seq, at.tile * ROWS, ROWS));
  int begin = span.x / KT * KT, end = span.y;
  const int pieces = uniform(pieces_of(a, KT, begin, end));
  if (at.piece >= pieces) return;
  share(KT, at.piece, pieces, begin, end);
  const bf16_t* k = a.k + at.b * a.sk.b + at.kh * a.sk.h;
  const bf16_t* v = a.v + at.b * a.sv.b + at.kh * a.sv.h;
  Loader<DH, KT, NT> kl, vl;
  kl.init(tid, a.dim, [&](int r) { return r * a.sk.t; });
  vl.init(tid, a.dim, [&](int r) { return r * a.sv.t; });
  const auto fetch = [&](int k0, int buf) {
    kl.start(k + k0 * a.sk.t, lds_address(lds[buf][0]), k0, span, tid);
    vl.start(v + k0 * a.sv.t, lds_address(lds[buf][1]), k0, span, tid);
  };
  if (begin < end) fetch(begin, 0);
  const float slope = a.slopes ? a.slopes[head] * LOG2E : 0.0f;
  bf16x8_t fq[DH / 16], fo[DH / 16];
  load_row<DH>(a.q + at.b * a.sq.b + i * a.sq.t + head * a.sq.h, a.dim, lane, fq, a.flip);
  load_row<DH>(a.dout + at.b * a.sdo.b + i * a.sdo.t + head * a.sdo.h, a.dim, lane, fo);
  const long at_row = row_index(a, at.b, head, i);
  const float lsum = log2_sum(a, at_row);
  // One key in sight: its probability is 1 whatever the score (dP and delta
  // would differ by their rounding). Such a row's tile is always cut.
  const bool alone = mine.y - mine.x <= 1;
  // P (dP - delta), by the cap's slope too, of columns 32 n .. of the tile at k0.
  const auto gradients = [&](int k0, int n, const char* Ks, const char* Vs, float delta, bool by_slope) {
    f32x16_t s = product<DH>(fq, Ks, 32 * n, frag);
    const f32x16_t dp = product<DH>(fo, Vs, 32 * n, frag);
    if (KIND == PLAIN) {
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], a.c1, -lsum)) * (dp[r] - delta);
    } else {
      f32x16_t dz = dp;
#pragma unroll
      for (int r = 0; r < 16; ++r) dz[r] -= delta;
      scores<KIND>(a, s, [&](int r, float t) {
        if (by_slope) dz[r] *= fmaf(-t, t, 1.0f);
      });
      if (a.slopes) {
        const float far = static_cast<float>(p - k0 - 32 * n - col_of(0, lane));
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] -= slope * fabsf(far - static_cast<float>(col_of(r, 0)));
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(s[r] - lsum) * dz[r];
    }
    if (k0 < wlast.x || k0 + KT > wfirst.y) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int j = k0 + 32 * n + col_of(r, lane);
        if (j < mine.x || j >= mine.y || alone) s[r] = 0.0f;
      }
    }
    return s;
  };
  const auto unseen = [&](int k0) { return k0 >= wlast.y || k0 + KT <= wfirst.x; };

  // delta = out . dout carries the rounding of out, the same for all of a row's
  // scores, and the fewer they are the more of the gradient that is: dQ and dK off
  // by 0.0042 of their norm with 2 tokens, 0.0030 with 16, 0.0026 with 256. A walk of
  // few tiles is made twice, first for the sum of P dP: 0.0024 with any number. Two
  // tiles stay in their buffers meanwhile (a backward of 64 x 8 heads of 64 columns, 128
  // tokens 31.3 -> 32.9 us, 256 tokens 66.9 -> 68.8). Longer walks take the rounded
  // out: 0.0024 to 0.0026 where many keys have weight, 0.0028 where a bias leaves few
  // of them; two walks there too would be 0.0024 for a fifth of the backward (6 x 1013
  // tokens of 12 heads of 80, capped, biased: 164 -> 199 us).
  float delta = 0.0f;
  int buf = 0;
  const int walk = (end - begin + KT - 1) / KT;
  const bool twice = pieces == 1 && walk <= 3, resident = twice && walk <= 2;
  if (twice) {
    for (int k0 = begin; k0 < end; k0 += KT, buf ^= 1) {
      landed();
      __syncthreads();
      if (k0 + KT < end) fetch(k0 + KT, buf ^ 1);
      else if (!resident) fetch(begin, buf ^ 1);
      if (unseen(k0)) continue;
#pragma unroll
      for (int n = 0; n < KT / 32; ++n) {
        const f32x16_t s = gradients(k0, n, lds[buf][0], lds[buf][1], 0.0f, false);
#pragma unroll
        for (int r = 0; r < 16; ++r) delta += s[r];
      }
    }
    if (resident) buf = 0;
  } else {
    bf16x8_t f[DH / 16];
    load_row<DH>(a.out + at.b * a.so.b + i * a.so.t + head * a.so.h, a.dim, lane, f);
#pragma unroll
    for (int q = 0; q < DH / 16; ++q) {
      const u16x8_t x = __builtin_bit_cast(u16x8_t, f[q]), y = __builtin_bit_cast(u16x8_t, fo[q]);
#pragma unroll
      for (int e = 0; e < 8; ++e) delta = fmaf(bf16_to_f32(x[e]), bf16_to_f32(y[e]), delta);
    }
  }
  delta += __shfl_xor(delta, 32);
  if (at.piece == 0 && lane < 32 && row0 + lane < a.rows) a.delta[at_row] = delta;

  f32x16_t o[DH / 32];
  zero(o);
  for (int k0 = begin; k0 < end; k0 += KT, buf ^= 1) {
    landed();
    __syncthreads();
    if (k0 + KT < end && !resident) fetch(k0 + KT, buf ^ 1);
    if (unseen(k0)) continue;
    const char *Ks = lds[buf][0], *Vs = lds[buf][1];
#pragma unroll
    for (int n = 0; n < KT / 32; ++n) accumulate<DH>(gradients(k0, n, Ks, Vs, delta, true), Ks, 32 * n, frag, o);
  }
  if (row0 + (lane & 31) >= a.rows) return;
  if (pieces > 1) {
    const long r = ((static_cast<long>(at.piece) * a.batch + at.b) * a.q_len + i) * a.heads + head;
    store_part<DH>(a.part + r * a.dim, a.dim, o, a.scale, lane);
    return;
  }
  store_row<DH>(a.dq + at.b * a.sdq.b + i * a.sdq.t + head * a.sdq.h, a.dim, o, a.scale, lane);
}

// What dK and dV need of a staged row: minus log2 of its sum (PLAIN: over c1),
// minus delta, slope, position and keys.
struct RowInfo {
  float sum[KT], delta[KT], slope[KT];
  int position[KT], lo[KT], hi[KT];
};

// dK and dV of WAVES * 32 keys: the wave's own 32 are keys, the walked columns
// rows (four products). At 128 columns the two results and the fragments of K and
// V would fill the registers of two waves a SIMD (30 spilled, 2469 us for 16384
// causal tokens of 16 heads, two to a key head); eight waves, which share a staged
// tile and leave LDS for it, keep V there instead (2183 us; with V in registers
// 2372). Heads that share a key head are walked by one block, so their sum needs
// no atomics and has one order.
template <int DH, int KIND, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 2) void attention_masked_dkv_kernel(Args a) {
  using T = Tile<DH>;
  __shared__ __attribute__((aligned(16))) char lds[2][2][T::BYTES];   // buffer, Q or dO
  __shared__ __attribute__((aligned(16))) RowInfo info[2];
  constexpr bool V_IN_LDS = DH == 128 && WAVES == 8;
  __shared__ __attribute__((aligned(16))) char own_v[V_IN_LDS ? WAVES : 1][V_IN_LDS ? T::BYTES / 2 : 16];
  constexpr int THREADS = 64 * WAVES, KEYS = 32 * WAVES;
  const Block at(a, false);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const Lane<DH> frag(lane);
  const Sequence seq(a, at.b);
  const int key0 = at.tile * KEYS, wkey0 = key0 + 32 * wave, key = wkey0 + (lane & 31);
  const int valid = min(seq.limit, key0 + KEYS);
  const bf16_t* q = a.q + at.b * a.sq.b + at.kh * a.group * a.sq.h;
  const bf16_t* dout = a.dout + at.b * a.sdo.b + at.kh * a.group * a.sdo.h;
  const int2 span = uniform(row_span(a, seq, key0, KEYS));
  int begin = uniform(a.by_step.div(span.x) * a.step), end = span.y;
  const int pieces = uniform(pieces_of(a, a.step, begin, end));
  if (at.piece >= pieces) return;
  share(a.step, at.piece, pieces, begin, end);
  // Row r of the tile at r0 is query (r0 + r) / group of head (r0 + r) % group. A
  // step is a whole number of queries, so a row's offset from the tile's first
  // query is the same for every tile; with a group past a tile it is worked out
  // for each.
  const auto offset = [&](const AttentionArgs::Strides& st, int r0, int r) {
    const int i = a.by_group.div(r0 + r);
    return r < a.step ? (i - static_cast<int>(a.by_group.div(r0))) * st.t + (r0 + r - i * a.group) * st.h
                      : static_cast<long>(OUTSIDE / 2);
  };
  const bool regular = a.group <= KT;
  Loader<DH, KT, THREADS> ql, dol;
  ql.init(tid, a.dim, [&](int r) { return offset(a.sq, 0, r); });
  dol.init(tid, a.dim, [&](int r) { return offset(a.sdo, 0, r); });
  const auto fetch = [&](int r0, int buf) {
    const int i0 = a.by_group.div(r0);
    const bf16_t *qb = q + i0 * a.sq.t, *ob = dout + i0 * a.sdo.t;
    if (regular) {
      ql.start(qb, lds_address(lds[buf][0]), r0, span, tid, a.step);
      dol.start(ob, lds_address(lds[buf][1]), r0, span, tid, a.step);
      return;
    }
    Loader<DH, KT, THREADS> l;
    l.init(tid, a.dim, [&](int r) { return offset(a.sq, r0, r); });
    l.start(qb, lds_address(lds[buf][0]), r0, span, tid);
    l.init(tid, a.dim, [&](int r) { return offset(a.sdo, r0, r); });
    l.start(ob, lds_address(lds[buf][1]), r0, span, tid);
  };
  // The staged rows' statistics: loaded as the tile is (nothing waits for them
  // there), worked out and stored in LDS after the products of the tile before.
  float rl = 0.0f, rd = 0.0f, rs = 0.0f;
  int2 rdoc = make_int2(0, 0x7fffffff);
  const auto look = [&](int r0) {
    if (tid < a.step && r0 + tid < a.rows) {
      const int i = a.by_group.div(r0 + tid), head = at.kh * a.group + r0 + tid - i * a.group;
      const long at_row = row_index(a, at.b, head, i);
      rl = a.lse[at_row];
      rd = a.delta[at_row];
      if (seq.doc) rdoc = seq.doc[a.q_offset + i];
      if (a.slopes) rs = a.slopes[head];
    }
  };
  const auto note = [&](int r0, int buf) {
    if (tid < KT) {
      RowInfo& w = info[buf];
      const bool row = tid < a.step && r0 + tid < a.rows;   // else it weighs zero
      const int p = a.q_offset + static_cast<int>(a.by_group.div(r0 + tid));
      const int2 keys = seq.clip(a, p, rdoc);
      // also where the row has no weight
      w.sum[tid] = row && rl != -INFINITY ? -rl * (KIND == PLAIN ? LOG2E / a.c1 : LOG2E) : -INFINITY;
      w.delta[tid] = row ? -rd : 0.0f;
      w.slope[tid] = rs * LOG2E;
      w.position[tid] = p;
      w.lo[tid] = row ? keys.x : 0;
      w.hi[tid] = row ? keys.y : 0;
    }
  };
  if (begin < end) {
    fetch(begin, 0);
    look(begin);
    note(begin, 0);
  }
  bf16x8_t fk[DH / 16], fv[V_IN_LDS ? 1 : DH / 16];
  f32x16_t dk[DH / 32], dv[DH / 32];
  const int kc = min(key, a.kv_len - 1), dim = kc < seq.limit ? a.dim : 0;
  load_row<DH>(a.k + at.b * a.sk.b + kc * a.sk.t + at.kh * a.sk.h, dim, lane, fk, a.flip);
  const bf16_t* v = a.v + at.b * a.sv.b + at.kh * a.sv.h;
  const char* my_v = own_v[V_IN_LDS ? uniform(wave) : 0];
  if constexpr (V_IN_LDS) {
    Loader<DH, 32, 64> l;
    l.init(lane, a.dim, [&](int r) { return r * a.sv.t; });
    const int first_key = uniform(wkey0);
    l.start(v + first_key * a.sv.t, lds_address(my_v), first_key, make_int2(0, seq.limit), lane);
  } else {
    load_row<DH>(v + kc * a.sv.t, dim, lane, fv);
  }
  zero(dk);
  zero(dv);
  int buf = 0;
  for (int r0 = begin; r0 < end; r0 += a.step, buf ^= 1) {
    landed();
    __syncthreads();
    const bool more = r0 + a.step < end;
    if (more) {
      fetch(r0 + a.step, buf ^ 1);
      look(r0 + a.step);
    }
    const RowInfo& w = info[buf];
    const int tail = min(a.step, a.rows - r0) - 1;
    if (wkey0 < valid && wkey0 < w.hi[tail] && wkey0 + 32 > w.lo[0]) {
      const char *Qs = lds[buf][0], *Os = lds[buf][1];
      const bool cut = wkey0 < w.lo[tail] || wkey0 + 32 > w.hi[0];
#pragma unroll(DH <= 64 ? 2 : 1)
      for (int n = 0; n < KT / 32; ++n) {
        const Lane<DH> lf = frag.here();
        // PLAIN: the rows' statistics are what the products start from, so that
        // they cost no registers of their own and nothing waits for them
        f32x16_t s, dp;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const float4 z = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
          const int c = 32 * n + col_of(4 * g, lane);
          const float4 su = KIND == PLAIN ? *reinterpret_cast<const float4*>(w.sum + c) : z;
          const float4 de = *reinterpret_cast<const float4*>(w.delta + c);
          s[4 * g] = su.x, s[4 * g + 1] = su.y, s[4 * g + 2] = su.z, s[4 * g + 3] = su.w;
          dp[4 * g] = de.x, dp[4 * g + 1] = de.y, dp[4 * g + 2] = de.z, dp[4 * g + 3] = de.w;
        }
#pragma unroll
        for (int q = 0; q < DH / 16; ++q) s = mfma(lf.row_frag(Qs, 32 * n, q), fk[q], s);
#pragma unroll
        for (int q = 0; q < DH / 16; ++q) {
          if constexpr (V_IN_LDS) dp = mfma(lf.row_frag(Os, 32 * n, q), lf.row_frag(my_v, 0, q), dp);
          else dp = mfma(lf.row_frag(Os, 32 * n, q), fv[q], dp);
        }
        if (KIND == PLAIN) {
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            s[r] = __builtin_amdgcn_exp2f(s[r] * a.c1);
            dp[r] *= s[r];
          }
        } else {
          scores<KIND>(a, s, [&](int r, float t) { dp[r] *= fmaf(-t, t, 1.0f); });
          if (a.slopes) {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
              const int c = 32 * n + col_of(r, lane);
              s[r] -= w.slope[c] * fabsf(static_cast<float>(w.position[c] - key));
            }
          }
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            __builtin_amdgcn_sched_barrier(0);   // one group's statistics at a time: registers
            const float4 u = *reinterpret_cast<const float4*>(w.sum + 32 * n + col_of(4 * g, lane));
            const float su[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int r = 4 * g + e;
              s[r] = __builtin_amdgcn_exp2f(s[r] + su[e]);
              dp[r] *= s[r];
            }
          }
        }
        if (cut) {   // both, also where dP is not finite
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int c = 32 * n + col_of(r, lane);
            const int lo = w.lo[c], hi = w.hi[c];
            if (key < lo || key >= hi) s[r] = dp[r] = 0.0f;
            if (hi - lo <= 1) dp[r] = 0.0f;   // one key in sight: no gradient, as for dQ
          }
        }
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const bf16x8_t fp = pack8(s, c), fd = pack8(dp, c);
#pragma unroll
          for (int j = 0; j < DH / 32; ++j) dv[j] = mfma(lf.col_frag(Os, 32 * n + 16 * c, j), fp, dv[j]);
#pragma unroll
          for (int j = 0; j < DH / 32; ++j) dk[j] = mfma(lf.col_frag(Qs, 32 * n + 16 * c, j), fd, dk[j]);
        }
      }
    }
    if (more) note(r0 + a.step, buf ^ 1);
  }
  if (key >= a.kv_len) return;
  if (pieces > 1) {
    const long r = ((static_cast<long>(at.piece) * a.batch + at.b) * a.kv_len + key) * a.kv_heads + at.kh;
    store_part<DH>(a.part + r * a.dim, a.dim, dk, a.scale, lane);
    store_part<DH>(a.part2 + r * a.dim, a.dim, dv, 1.0f, lane);
    return;
  }
  store_row<DH>(a.dk + at.b * a.sdk.b + key * a.sdk.t + at.kh * a.sdk.h, a.dim, dk, a.scale, lane);
  store_row<DH>(a.dv + at.b * a.sdv.b + key * a.sdv.t + at.kh * a.sdv.h, a.dim, dv, 1.0f, lane);
}

size_t round256(size_t n) { return (n + 255) & ~static_cast<size_t>(255); }
size_t doc_bytes(const AttentionArgs& a) { return round256(static_cast<size_t>(a.batch) * a.kv_len * sizeof(int2)); }
size_t q_rows(const AttentionArgs& a) { return static_cast<size_t>(a.batch) * a.heads * a.q_len; }
size_t k_rows(const AttentionArgs& a) { return static_cast<size_t>(a.batch) * a.kv_heads * a.kv_len; }

// How the walks of a kernel's blocks are cut: up to `want` blocks fill the chip,
// and fewer of a long walk leave CUs idle (a backward of 8 heads of 4096 causal
// tokens, 128 columns, 327 us whole and 215 in pieces; of 6 x 1013 tokens, 12 heads
// of 80 on 4, 157 and 109). A piece has at least `least` steps, so that a partial
// result's write and read stay small beside its products.
struct Cut {
  int pieces = 1, quantum = 1;   // as in Args
};
Cut cut(long blocks, long steps, long want, long least) {
  Cut c;
  if (blocks <= 0 || steps <= 0) return c;
  c.pieces = static_cast<int>(std::max(1L, std::min({want / blocks, steps / least, 128L})));
  c.quantum = static_cast<int>(least);
  return c;
}

struct Plan {
  bool few;                      // forward by the kernel for few rows
  bool wide;                     // dK and dV by blocks of 256 keys, else of 128
  Cut fwd, dq, dkv;
};
Plan plan(const AttentionArgs& a) {
  Plan p;
  const long bh = static_cast<long>(a.batch) * a.kv_heads;
  const long row_tiles = (a.rows + ROWS - 1L) / ROWS;
  // Rows of one wave go to the kernel whose waves share out the keys: 4 rows of 16
  // x 8 key heads over 32768 keys take 371 us there and 377 in tiles of 128 rows, of
  // 32 x 8 over 4096 keys (one head to a row) 95 and 106, 8 rows of 32 x 8 over 2048
  // keys 45 and 49; 64 rows would read the keys twice (4 x 8 over 8192 39 us and 34).
  // One block a CU: more gain little and have to be joined (4 x 8 heads of 8192 keys
  // 30 us in 256 blocks, 35 in 512, 45 in 1024; 16 x 8 of 32768 371, 368, 367).
  p.few = a.rows <= 32;
  p.fwd = p.few ? cut(bh, (a.kv_len + 31L) / 32, 256, 8)
                : cut(bh * row_tiles, (a.kv_len + KT - 1L) / KT, 512, 8);   // two blocks a CU
  p.dq = cut(bh * row_tiles, (a.kv_len + KT - 1L) / KT, 512, 8);
  // A backward with eight waves and with four: 4 x 16 heads of 1024 causal tokens 132
  // us and 141, 64 x 8 of 256 117 and 119, 2 x 16 of 4096 485 and 527 (2 x 8 of 1024
  // 72 and 68). At 128 keys half of the eight have none: 63 and 56.
  p.wide = a.dim > 96 && a.kv_len > 128;
  // Two rounds of blocks (of four waves two fit a CU, of eight one) even out walks of
  // unlike length: 12 heads of 4096 causal tokens, 192 blocks of eight, 264 us of a
  // backward and in one round 340, 8 heads 215 and 223; but 16 heads of 2048, 128
  // blocks, 148 and 136.
  const long step = a.group <= KT ? KT / a.group * a.group : KT;
  p.dkv = cut(bh * (p.wide ? (a.kv_len + 255L) / 256 : (a.kv_len + 127L) / 128), (a.rows + step - 1) / step,
              p.wide ? 512 : 1024, 8);
  return p;
}
size_t part_bytes(const Cut& c, size_t rows, int dim) {
  return c.pieces > 1 ? round256(static_cast<size_t>(c.pieces) * rows * dim * sizeof(float)) : 0;
}

// Launch-independent values, and the document runs if there are documents.
hipError_t prepare(const AttentionArgs& in, Args& a, hipStream_t s) {
  static_cast<AttentionArgs&>(a) = in;
  a.by_group = FastDiv(in.group);
  a.by_bh = FastDiv(in.batch * in.kv_heads);
  a.by_kv = FastDiv(in.kv_heads);
  const float scale = std::fabs(in.scale);
  a.c1 = scale * LOG2E;
  a.c2 = in.cap * LOG2E;
  if (in.cap > 0.0f) {
    a.c3 = 1.0f / a.c2;   // FAR_CAP only
    a.c4 = 2.0f * scale / in.cap * LOG2E;
  }
  a.flip = in.scale < 0.0f;
  a.step = in.group <= KT ? KT / in.group * in.group : KT;
  a.by_step = FastDiv(a.step);
  if (!in.documents || in.kv_len == 0) return hipSuccess;
  int2* runs = reinterpret_cast<int2*>(in.ws);
  a.doc = runs;
  const int threads = std::min((in.kv_len + 63) / 64 * 64, 1024);
  const unsigned chunks = (in.kv_len + threads - 1) / threads;
  hipLaunchKernelGGL(document_runs_kernel, dim3(chunks * in.batch), dim3(threads), 0, s, in.documents, in.kv_len,
                     FastDiv(chunks), runs);
  return hipGetLastError();
}

// Calls f with the smallest compiled head width that holds dim, and how scores
// are formed (not PLAIN with a vanishing scale: it divides by it, and hides columns
// before they are multiplied).
template <typename F>
void with_width(const Args& a, F&& f) {
  auto pick = [&](auto width) {
    if (a.cap > NEAR_CAP) f(width, std::integral_constant<int, FAR_CAP>{});
    else if (a.cap > 0.0f || a.slopes || a.c1 < 0x1p-60f) f(width, std::integral_constant<int, GENERAL>{});
    else f(width, std::integral_constant<int, PLAIN>{});
  };
  const int dim = a.dim;
  if (dim <= 32) pick(std::integral_constant<int, 32>{});
  else if (dim <= 64) pick(std::integral_constant<int, 64>{});
  else if (dim <= 96) pick(std::integral_constant<int, 96>{});
  else pick(std::integral_constant<int, 128>{});
}

template <typename K>
hipError_t launch(K* kernel, int threads, Args& a, long length, int tile, const Cut& c, hipStream_t s) {
  a.tiles = static_cast<int>((length + tile - 1) / tile);
  a.pieces = c.pieces;
  a.quantum = c.quantum;
  a.by_tiles = FastDiv(a.tiles);

  hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(a.tiles) * a.pieces * a.batch * a.kv_heads), dim3(threads), 0, s,
                     a);
  return hipGetLastError();
}

}  // namespace

size_t attention_ws_bytes(const AttentionArgs& a, bool backward) {
  const Plan p = plan(a);
  const size_t forward = doc_bytes(a) + part_bytes(p.fwd, q_rows(a), a.dim) +
                         (p.fwd.pieces > 1 ? round256(p.fwd.pieces * q_rows(a) * sizeof(float2)) : 0);
  if (!backward) return forward;
  return std::max(forward, doc_bytes(a) + round256(q_rows(a) * sizeof(float)) + part_bytes(p.dq, q_rows(a), a.dim) +
                               2 * part_bytes(p.dkv, k_rows(a), a.dim));
}

hipError_t attention_masked_fwd(const AttentionArgs& in, hipStream_t s) {
  if (in.batch == 0 || in.q_len == 0) return hipSuccess;
  Args a;
  hipError_t e = prepare(in, a, s);
  if (e != hipSuccess) return e;
  const Plan p = plan(in);
  a.part = reinterpret_cast<float*>(in.ws + doc_bytes(in));
  a.part_ml = reinterpret_cast<float2*>(in.ws + doc_bytes(in) + part_bytes(p.fwd, q_rows(in), in.dim));
  with_width(a, [&](auto width, auto kind) {
    e = p.few ? launch(attention_masked_few_kernel<width(), kind()>, NT, a, a.rows, 32, p.fwd, s)
              : launch(attention_masked_fwd_kernel<width(), kind()>, NT, a, a.rows, ROWS, p.fwd, s);
  });
  if (e != hipSuccess || p.fwd.pieces == 1) return e;
  const long rows = static_cast<long>(q_rows(in));
  hipLaunchKernelGGL(attention_join_kernel, dim3(static_cast<unsigned>((rows + NT / 16 - 1) / (NT / 16))), dim3(NT), 0,
                     s, a, rows, FastDiv(a.q_len), FastDiv(a.heads), p.few ? 1 : 0);
  return hipGetLastError();
}

hipError_t attention_masked_bwd(const AttentionArgs& in, hipStream_t s) {
  if (in.batch == 0 || (in.q_len == 0 && in.kv_len == 0)) return hipSuccess;
  Args a;
  hipError_t e = prepare(in, a, s);
  if (e != hipSuccess) return e;
  const Plan p = plan(in);
  char* ws = in.ws + doc_bytes(in);
  a.delta = reinterpret_cast<float*>(ws);
  ws += round256(q_rows(in) * sizeof(float));
  float* part_q = reinterpret_cast<float*>(ws);
  ws += part_bytes(p.dq, q_rows(in), in.dim);
  float* part_k = reinterpret_cast<float*>(ws);
  float* part_v = reinterpret_cast<float*>(ws + part_bytes(p.dkv, k_rows(in), in.dim));
  Sums sums{};
  sums.keys = p.wide ? 256 : 128;
  long most = 0;
  const auto sum = [&](int at, const float* part, bf16_t* out, const AttentionArgs::Strides& to, size_t rows, int heads,
                       int tokens, const Cut& c) {
    if (c.pieces == 1) return;
    sums.sum[at] = {part, out, to, static_cast<long>(rows), FastDiv(heads), FastDiv(tokens), c.pieces, c.quantum};
    most = std::max(most, static_cast<long>(rows));
  };
  with_width(a, [&](auto width, auto kind) {
    if (a.q_len > 0) {
      a.part = part_q;
      e = launch(attention_masked_dq_kernel<width(), kind()>, NT, a, a.rows, ROWS, p.dq, s);
      if (e != hipSuccess) return;
      sum(0, part_q, a.dq, a.sdq, q_rows(in), a.heads, a.q_len, p.dq);
    }
    if (a.kv_len == 0) return;
    a.part = part_k;
    a.part2 = part_v;
    constexpr bool kWide = width() == 128;
    if constexpr (kWide) {
      if (p.wide) e = launch(attention_masked_dkv_kernel<width(), kind(), 8>, 512, a, a.kv_len, 256, p.dkv, s);
    }
    if (!kWide || !p.wide)
      e = launch(attention_masked_dkv_kernel<width(), kind(), 4>, 256, a, a.kv_len, 128, p.dkv, s);
    if (e != hipSuccess) return;
    sum(1, part_k, a.dk, a.sdk, k_rows(in), a.kv_heads, a.kv_len, p.dkv);
    sum(2, part_v, a.dv, a.sdv, k_rows(in), a.kv_heads, a.kv_len, p.dkv);
  });
  if (e != hipSuccess || most == 0) return e;
  hipLaunchKernelGGL(attention_sum_kernel, dim3(static_cast<unsigned>((most + NT / 16 - 1) / (NT / 16)), 3), dim3(NT), 0,
                     s, a, sums);
  return hipGetLastError();
}

}  // namespace spx
