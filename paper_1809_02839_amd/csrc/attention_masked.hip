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
#include <algorithm>
#include <type_traits>

#include "attention_tiles.hpp"

namespace spx {
namespace {

constexpr int NT = 256, ROWS = 128, KT = 64;   // threads, rows of a block, keys (rows) of a staged tile
constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;

struct Args : AttentionArgs {
  const int2* doc = nullptr;      // [batch][kv_len]: first and past-the-last token of the token's document
  float* delta = nullptr;         // [batch][heads][q_len]: out . dout (backward)
  float c1 = 0.0f;                // uncapped: scale log2(e); capped: 2 scale / cap log2(e)
  float c2 = 0.0f;                // capped: cap log2(e)
  FastDiv by_group, by_bh, by_kv, by_pieces;
  int tiles = 0;
  int pieces = 1;                 // blocks that share a tile's walk, each writing a partial result
  float* part = nullptr;          // [pieces][...][dim] partial results (pieces > 1)
  float2* part_ml = nullptr;      // [pieces][batch][heads][q_len] maximum and sum (forward)
  float* part2 = nullptr;         // dV's (part is dK's)
};

// The piece'th of `pieces` equal shares of the tiles of width W in [begin, end).
template <int W>
__device__ __forceinline__ void share(int piece, int pieces, int& begin, int& end) {
  if (pieces == 1) return;
  const long n = max(0, (end - begin + W - 1) / W);
  const int b = begin;
  begin = b + static_cast<int>(n * piece / pieces) * W;
  end = min(end, b + static_cast<int>(n * (piece + 1) / pieces) * W);
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
    int lo = 0, hi = limit;
    if (a.causal) hi = min(hi, max(p + 1, prefix));
    if (doc) {
      const int2 d = doc[p];
      lo = d.x;
      hi = min(hi, d.y);
    }
    return make_int2(lo, hi);
  }
};

// Score of one product in units of log2: s * log2(e), and tanh(z / cap).
template <bool CAP>
__device__ __forceinline__ float score(const Args& a, float acc, float& t) {
  if constexpr (CAP) {
    t = 1.0f - 2.0f * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(acc * a.c1));
    return t * a.c2;
  } else {
    return acc * a.c1;
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

__device__ uint4 zero16;   // what rows and columns outside a tensor are staged from

// Direct load into LDS: the 16 bytes at lane l's address land at LDS byte
// address lds + 16 l (lds wave-uniform, passed in M0). Issued through inline
// assembly so that the compiler, which cannot tell the two buffers apart, does
// not wait for the next tile before each read of this one; landed() waits for
// the wave's own loads, and the barrier after it for the others'.
__device__ __forceinline__ void direct16(const void* g, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(g) : "memory", "m0");
}
__device__ __forceinline__ void landed() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
__device__ __forceinline__ uint32_t lds_address(const void* p) {
  return static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const char*)p));
}

// Starts the copy of rows first .. first + KT - 1 (zero from `limit` on and from
// column `dim` on); address(row) is a row's first element.
template <int DH, typename F>
__device__ __forceinline__ void stage(uint32_t lds, int first, int limit, int dim, int tid, F&& address) {
  using T = Tile<DH>;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(tid >> 6);
#pragma unroll
  for (int i = 0; i < T::V; ++i) {
    const int e = tid + NT * i, r = e / T::C, row = first + r, col = ((e % T::C) ^ T::swizzle(r)) * 8;
    const void* g = &zero16;
    if (row < limit && col < dim) g = address(row) + col;
    direct16(g, lds + 16 * (64 * wave + NT * i));
  }
}

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
__device__ __forceinline__ void load_row(const bf16_t* row, int dim, int lane, bf16x8_t (&f)[DH / 16]) {
#pragma unroll
  for (int q = 0; q < DH / 16; ++q) {
    const int col = 16 * q + 8 * (lane >> 5);
    uint4 u = make_uint4(0, 0, 0, 0);
    if (col < dim) u = *reinterpret_cast<const uint4*>(row + col);
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

// Documents: each token's run of equal numbers. A block owns 1024 tokens; runs
// that cross its ends are followed outwards, a block's width at a time.
constexpr int DT = 1024;
__global__ __launch_bounds__(DT) void document_runs_kernel(const int32_t* ids, int len, FastDiv chunks, int2* runs) {
  __shared__ int scan[2][DT];
  __shared__ int edge[2];
  const int b = chunks.div(blockIdx.x);
  const int tid = threadIdx.x, first = (blockIdx.x - b * chunks.d) * DT, j = first + tid;
  const int last = min(first + DT, len) - 1;
  ids += static_cast<long>(b) * len;
  runs += static_cast<long>(b) * len;
  const bool in = j < len;
  const int id = in ? ids[j] : 0;
  // start of the first token's run: the first of the tokens before it that are all equal
  int start = first;
  for (int to = first; to > 0;) {
    const int w = min(DT, to), base = to - w;
    if (tid == 0) edge[0] = -1;
    __syncthreads();
    if (tid < w && ids[base + tid] != ids[first]) atomicMax(&edge[0], base + tid);
    __syncthreads();
    const int found = edge[0];
    __syncthreads();
    start = found < 0 ? base : found + 1;
    if (found >= 0) break;
    to = base;
  }
  int end = last + 1;
  for (int from = last + 1; from < len;) {
    const int w = min(DT, len - from);
    if (tid == 0) edge[1] = 0x7fffffff;
    __syncthreads();
    if (tid < w && ids[from + tid] != ids[last]) atomicMin(&edge[1], from + tid);
    __syncthreads();
    const int found = edge[1];
    __syncthreads();
    end = found == 0x7fffffff ? from + w : found;
    if (found != 0x7fffffff) break;
    from += w;
  }
  // inside the block: the last start at or before a token, the first end after it
  scan[0][tid] = tid == 0 ? start : (in && ids[j - 1] != id ? j : -1);
  scan[1][tid] = j == last ? end : (in && j < last && ids[j + 1] != id ? j + 1 : 0x7fffffff);
  __syncthreads();
  for (int step = 1; step < DT; step *= 2) {
    const int s = tid >= step ? scan[0][tid - step] : -1;
    const int e = tid + step < DT ? scan[1][tid + step] : 0x7fffffff;
    __syncthreads();
    scan[0][tid] = max(scan[0][tid], s);
    scan[1][tid] = min(scan[1][tid], e);
    __syncthreads();
  }
  if (in) runs[j] = make_int2(scan[0][tid], scan[1][tid]);
}

// One block's place: its (sequence, kv head) and tile. Consecutive blocks take
// different kv heads (of one XCD each where their number is a multiple of 8),
// and the tiles with the most work under a causal mask first: the last rows,
// the first keys.
struct Block {
  int b, kh, tile, piece;
  __device__ __forceinline__ Block(const Args& a, bool last_first) {
    const uint32_t x = blockIdx.x, tp = a.by_bh.div(x), bh = x - tp * a.by_bh.d, t = a.by_pieces.div(tp);
    piece = tp - t * a.by_pieces.d;
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
  template <bool CAP, int N>
  __device__ __forceinline__ void take(const Args& a, const Lane<DH>& frag, const char* Ks, const char* Vs,
                                       const bf16x8_t (&fq)[DH / 16], int k0, int p, float slope, int2 mine, bool cut,
                                       int lane) {
    f32x16_t s[N];
    float t;
#pragma unroll
    for (int n = 0; n < N; ++n) {
      s[n] = product<DH>(fq, Ks, 32 * n, frag);
#pragma unroll
      for (int r = 0; r < 16; ++r) s[n][r] = score<CAP>(a, s[n][r], t);
    }
    if (a.slopes) {
#pragma unroll
      for (int n = 0; n < N; ++n)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          s[n][r] -= slope * fabsf(static_cast<float>(p - (k0 + 32 * n + col_of(r, lane))));
    }
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
    top = fmaxf(top, __shfl_xor(top, 32));
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
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[n][r] = __builtin_amdgcn_exp2f(s[n][r] - base);
        sum += s[n][r];
      }
      accumulate<DH>(s[n], Vs, 32 * n, frag, o);
    }
  }
};

__device__ __forceinline__ long row_index(const Args& a, int b, int head, int i) {
  return (static_cast<long>(b) * a.heads + head) * a.q_len + i;
}
__device__ __forceinline__ float lse_of(float m, float sum) { return sum == 0.0f ? -INFINITY : m * LN2 + logf(sum); }

// A block: 128 rows, or one piece of their keys.
template <int DH, bool CAP>
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
  const int2 wfirst = seq.keys(a, position(row0)), wlast = seq.keys(a, position(row0 + 31));
  int begin = seq.keys(a, position(at.tile * ROWS)).x / KT * KT;
  int end = seq.keys(a, position(at.tile * ROWS + ROWS - 1)).y;
  share<KT>(at.piece, a.pieces, begin, end);
  const bf16_t* k = a.k + at.b * a.sk.b + at.kh * a.sk.h;
  const bf16_t* v = a.v + at.b * a.sv.b + at.kh * a.sv.h;
  const auto fetch = [&](int k0, int buf) {
    stage<DH>(lds_address(lds[buf][0]), k0, seq.limit, a.dim, tid, [&](int j) { return k + j * a.sk.t; });
    stage<DH>(lds_address(lds[buf][1]), k0, seq.limit, a.dim, tid, [&](int j) { return v + j * a.sv.t; });
  };
  if (begin < end) fetch(begin, 0);
  const float slope = a.slopes ? a.slopes[head] * LOG2E : 0.0f;
  bf16x8_t fq[DH / 16];
  load_row<DH>(a.q + at.b * a.sq.b + i * a.sq.t + head * a.sq.h, a.dim, lane, fq);

  Running<DH> run;
  zero(run.o);
  int buf = 0;
  for (int k0 = begin; k0 < end; k0 += KT, buf ^= 1) {
    landed();
    __syncthreads();
    if (k0 + KT < end) fetch(k0 + KT, buf ^ 1);
    if (k0 >= wlast.y || k0 + KT <= wfirst.x) continue;
    run.template take<CAP, KT / 32>(a, frag, lds[buf][0], lds[buf][1], fq, k0, p, slope, mine,
                                    k0 < wlast.x || k0 + KT > wfirst.y, lane);
  }
  const float sum = run.sum + __shfl_xor(run.sum, 32);
  if (row0 + (lane & 31) >= a.rows) return;
  const long r = row_index(a, at.b, head, i);
  if (a.pieces > 1) {
    const long rp = at.piece * static_cast<long>(a.batch) * a.heads * a.q_len + r;
    store_part<DH>(a.part + rp * a.dim, a.dim, run.o, 1.0f, lane);
    if (lane < 32) a.part_ml[rp] = make_float2(run.m, sum);
    return;
  }
  store_row<DH>(a.out + at.b * a.so.b + i * a.so.t + head * a.so.h, a.dim, run.o, sum == 0.0f ? 0.0f : 1.0f / sum, lane);
  if (a.lse && lane < 32) a.lse[r] = lse_of(run.m, sum);
}

// Up to 32 rows (single tokens, and what little a group makes of a few): bound
// by reading the keys and values once, so the block's waves share out the keys,
// each with tiles of 32 of its own that no other wave waits for, and join their
// sums at the end.
template <int DH, bool CAP>
__global__ __launch_bounds__(NT, 1) void attention_masked_few_kernel(Args a) {
  using T = Tile<DH>;
  constexpr int FT = 32, BYTES = T::BYTES / (KT / FT), V = FT * T::C / 64;
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
  const int2 first = seq.keys(a, position(row0)), last = seq.keys(a, position(row0 + 31));
  int begin = first.x / FT * FT, end = last.y;
  share<FT>(at.piece * (NT / 64) + wave, a.pieces * (NT / 64), begin, end);
  const bf16_t* k = a.k + at.b * a.sk.b + at.kh * a.sk.h;
  const bf16_t* v = a.v + at.b * a.sv.b + at.kh * a.sv.h;
  const auto fetch = [&](int k0, int buf) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const uint32_t to = lds_address(lds[wave][buf][t]);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const int c = lane + 64 * e, r = c / T::C, j = k0 + r, col = ((c % T::C) ^ T::swizzle(r)) * 8;
        const void* g = &zero16;
        if (j < seq.limit && col < a.dim) g = (t == 0 ? k + j * a.sk.t : v + j * a.sv.t) + col;
        direct16(g, to + 1024 * e);
      }
    }
  };
  if (begin < end) fetch(begin, 0);
  const float slope = a.slopes ? a.slopes[head] * LOG2E : 0.0f;
  bf16x8_t fq[DH / 16];
  load_row<DH>(a.q + at.b * a.sq.b + i * a.sq.t + head * a.sq.h, a.dim, lane, fq);

  Running<DH> run;
  zero(run.o);
  int buf = 0;
  for (int k0 = begin; k0 < end; k0 += FT, buf ^= 1) {
    landed();
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the other buffer has been read
    if (k0 + FT < end) fetch(k0 + FT, buf ^ 1);
    run.template take<CAP, 1>(a, frag, lds[wave][buf][0], lds[wave][buf][1], fq, k0, p, slope, mine,
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
    if (a.pieces > 1) {
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

// Joins the pieces of the forward: 16 lanes a row, eight columns each.
__global__ __launch_bounds__(NT) void attention_join_kernel(Args a, long rows, FastDiv by_len, FastDiv by_heads) {
  const long r = static_cast<long>(blockIdx.x) * (NT / 16) + threadIdx.x / 16;
  const int col = threadIdx.x % 16 * 8;
  if (r >= rows || col >= a.dim) return;
  float m = -INFINITY;
  for (int u = 0; u < a.pieces; ++u) m = fmaxf(m, a.part_ml[u * rows + r].x);
  const float base = m == -INFINITY ? 0.0f : m;
  float l = 0.0f, x[8] = {};
  for (int u = 0; u < a.pieces; ++u) {
    const float2 ml = a.part_ml[u * rows + r];
    const float w = __builtin_amdgcn_exp2f(ml.x - base);
    const float4* y = reinterpret_cast<const float4*>(a.part + (u * rows + r) * a.dim + col);
    const float4 lo = y[0], hi = y[1];
    l = fmaf(w, ml.y, l);
    x[0] = fmaf(w, lo.x, x[0]), x[1] = fmaf(w, lo.y, x[1]), x[2] = fmaf(w, lo.z, x[2]), x[3] = fmaf(w, lo.w, x[3]);
    x[4] = fmaf(w, hi.x, x[4]), x[5] = fmaf(w, hi.y, x[5]), x[6] = fmaf(w, hi.z, x[6]), x[7] = fmaf(w, hi.w, x[7]);
  }
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  const uint32_t bh = by_len.div(static_cast<uint32_t>(r)), i = static_cast<uint32_t>(r) - bh * by_len.d;
  const uint32_t b = by_heads.div(bh), h = bh - b * by_heads.d;
  *reinterpret_cast<uint4*>(a.out + b * a.so.b + i * a.so.t + h * a.so.h + col) =
      make_uint4(pack_bf16x2(x[0] * inv, x[1] * inv), pack_bf16x2(x[2] * inv, x[3] * inv),
                 pack_bf16x2(x[4] * inv, x[5] * inv), pack_bf16x2(x[6] * inv, x[7] * inv));
  if (a.lse && col == 0) a.lse[r] = lse_of(m, l);
}

// Sums the pieces of a gradient [batch][token][head] in piece order: 16 lanes a
// row, eight columns each; up to three gradients by blockIdx.y.
struct Sum {
  const float* part;
  bf16_t* out;
  AttentionArgs::Strides to;
  long rows;            // batch * tokens * heads
  FastDiv by_heads, by_tokens;
  int pieces;
};
struct Sums {
  Sum sum[3];
  int dim;
};
__global__ __launch_bounds__(NT) void attention_sum_kernel(Sums all) {
  const Sum& j = all.sum[blockIdx.y];
  const long r = static_cast<long>(blockIdx.x) * (NT / 16) + threadIdx.x / 16;
  const int col = threadIdx.x % 16 * 8;
  if (r >= j.rows || col >= all.dim) return;
  float x[8] = {};
  for (int u = 0; u < j.pieces; ++u) {
    const float4* y = reinterpret_cast<const float4*>(j.part + (u * j.rows + r) * all.dim + col);
    const float4 lo = y[0], hi = y[1];
    x[0] += lo.x, x[1] += lo.y, x[2] += lo.z, x[3] += lo.w;
    x[4] += hi.x, x[5] += hi.y, x[6] += hi.z, x[7] += hi.w;
  }
  const uint32_t bt = j.by_heads.div(static_cast<uint32_t>(r)), h = static_cast<uint32_t>(r) - bt * j.by_heads.d;
  const uint32_t b = j.by_tokens.div(bt), t = bt - b * j.by_tokens.d;
  *reinterpret_cast<uint4*>(j.out + b * j.to.b + t * j.to.t + h * j.to.h + col) =
      make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
}

// delta = out . dout of every row, 16 lanes a row.
__global__ __launch_bounds__(NT) void attention_delta_kernel(Args a, long rows, FastDiv by_heads, FastDiv by_len) {
  const long r = static_cast<long>(blockIdx.x) * (NT / 16) + threadIdx.x / 16;
  if (r >= rows) return;   // whole 16-lane groups leave
  const uint32_t t = by_heads.div(static_cast<uint32_t>(r)), h = static_cast<uint32_t>(r) - t * by_heads.d;
  const uint32_t b = by_len.div(t), i = t - b * by_len.d;
  const int col = (threadIdx.x % 16) * 8;
  float s = 0.0f;
  if (col < a.dim) {
    const u16x8_t o = *reinterpret_cast<const u16x8_t*>(a.out + b * a.so.b + i * a.so.t + h * a.so.h + col);
    const u16x8_t d = *reinterpret_cast<const u16x8_t*>(a.dout + b * a.sdo.b + i * a.sdo.t + h * a.sdo.h + col);
#pragma unroll
    for (int e = 0; e < 8; ++e) s = fmaf(bf16_to_f32(o[e]), bf16_to_f32(d[e]), s);
  }
#pragma unroll
  for (int w = 8; w >= 1; w /= 2) s += __shfl_xor(s, w);
  if (threadIdx.x % 16 == 0) a.delta[(static_cast<long>(b) * a.heads + h) * a.q_len + i] = s;
}

// A row's statistics for the backward: log2 of its sum (infinite where the row
// has no weight, so every probability is zero) and delta.
__device__ __forceinline__ float2 row_stats(const Args& a, int b, int head, int i) {
  const long at = (static_cast<long>(b) * a.heads + head) * a.q_len + i;
  const float l = a.lse[at];
  return make_float2(l == -INFINITY ? INFINITY : l * LOG2E, a.delta[at]);
}

template <int DH, bool CAP>
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
  const int2 wfirst = seq.keys(a, position(row0)), wlast = seq.keys(a, position(row0 + 31));
  int begin = seq.keys(a, position(at.tile * ROWS)).x / KT * KT;
  int end = seq.keys(a, position(at.tile * ROWS + ROWS - 1)).y;
  share<KT>(at.piece, a.pieces, begin, end);
  const bf16_t* k = a.k + at.b * a.sk.b + at.kh * a.sk.h;
  const bf16_t* v = a.v + at.b * a.sv.b + at.kh * a.sv.h;
  const auto fetch = [&](int k0, int buf) {
    stage<DH>(lds_address(lds[buf][0]), k0, seq.limit, a.dim, tid, [&](int j) { return k + j * a.sk.t; });
    stage<DH>(lds_address(lds[buf][1]), k0, seq.limit, a.dim, tid, [&](int j) { return v + j * a.sv.t; });
  };
  if (begin < end) fetch(begin, 0);
  const float slope = a.slopes ? a.slopes[head] * LOG2E : 0.0f;
  bf16x8_t fq[DH / 16], fo[DH / 16];
  load_row<DH>(a.q + at.b * a.sq.b + i * a.sq.t + head * a.sq.h, a.dim, lane, fq);
  load_row<DH>(a.dout + at.b * a.sdo.b + i * a.sdo.t + head * a.sdo.h, a.dim, lane, fo);
  const float2 st = row_stats(a, at.b, head, i);

  f32x16_t o[DH / 32];
  zero(o);
  int buf = 0;
  for (int k0 = begin; k0 < end; k0 += KT, buf ^= 1) {
    landed();
    __syncthreads();
    if (k0 + KT < end) fetch(k0 + KT, buf ^ 1);
    if (k0 >= wlast.y || k0 + KT <= wfirst.x) continue;
    const char *Ks = lds[buf][0], *Vs = lds[buf][1];
    const bool cut = k0 < wlast.x || k0 + KT > wfirst.y;
#pragma unroll
    for (int n = 0; n < KT / 32; ++n) {
      f32x16_t s = product<DH>(fq, Ks, 32 * n, frag);
      const f32x16_t dp = product<DH>(fo, Vs, 32 * n, frag);
      f32x16_t t;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        float tr;
        s[r] = score<CAP>(a, s[r], tr);
        if (CAP) t[r] = tr;
      }
      if (a.slopes) {
#pragma unroll
        for (int r = 0; r < 16; ++r)
          s[r] -= slope * fabsf(static_cast<float>(p - (k0 + 32 * n + col_of(r, lane))));
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[r] = __builtin_amdgcn_exp2f(s[r] - st.x) * (dp[r] - st.y);
        if (CAP) s[r] *= 1.0f - t[r] * t[r];
      }
      if (cut) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int j = k0 + 32 * n + col_of(r, lane);
          if (j < mine.x || j >= mine.y) s[r] = 0.0f;
        }
      }
      accumulate<DH>(s, Ks, 32 * n, frag, o);
    }
  }
  if (row0 + (lane & 31) >= a.rows) return;
  if (a.pieces > 1) {
    const long r = ((static_cast<long>(at.piece) * a.batch + at.b) * a.q_len + i) * a.heads + head;
    store_part<DH>(a.part + r * a.dim, a.dim, o, a.scale, lane);
    return;
  }
  store_row<DH>(a.dq + at.b * a.sdq.b + i * a.sdq.t + head * a.sdq.h, a.dim, o, a.scale, lane);
}

// What dK and dV need of a staged row: log2 of its sum, delta, slope, position
// and keys.
struct RowInfo {
  float sum[KT], delta[KT], slope[KT];
  int position[KT], lo[KT], hi[KT];
};

// dK and dV of 128 keys: the wave's own 32 are keys, the walked columns rows.
template <int DH, bool CAP>
__global__ __launch_bounds__(NT, 2) void attention_masked_dkv_kernel(Args a) {
  using T = Tile<DH>;
  __shared__ __attribute__((aligned(16))) char lds[2][2][T::BYTES];   // buffer, Q or dO
  __shared__ __attribute__((aligned(16))) RowInfo info[2];
  const Block at(a, false);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const Lane<DH> frag(lane);
  const Sequence seq(a, at.b);
  const int key0 = at.tile * ROWS, wkey0 = key0 + 32 * wave, key = wkey0 + (lane & 31);
  const int valid = min(seq.limit, key0 + ROWS);
  const bf16_t* q = a.q + at.b * a.sq.b + at.kh * a.group * a.sq.h;
  const bf16_t* dout = a.dout + at.b * a.sdo.b + at.kh * a.group * a.sdo.h;
  // rows that see one of the block's keys: positions [pa, pb)
  int pa = -(1 << 30), pb = 0x7fffffff;
  if (a.causal && key0 >= seq.prefix) pa = key0;
  if (seq.doc && key0 < valid) {
    pa = max(pa, seq.doc[key0].x);
    pb = seq.doc[valid - 1].y;
  }
  const long first = max(0L, static_cast<long>(pa) - a.q_offset) * a.group;
  int begin = static_cast<int>(min(first, static_cast<long>(a.rows))) / KT * KT;
  int end = key0 < valid ? static_cast<int>(min(max(static_cast<long>(pb) - a.q_offset, 0L) * a.group,
                                                static_cast<long>(a.rows)))
                         : 0;
  share<KT>(at.piece, a.pieces, begin, end);
  const auto fetch = [&](int r0, int buf) {
    int here = tid;
    asm volatile("" : "+v"(here));   // as Lane::here
    stage<DH>(lds_address(lds[buf][0]), r0, a.rows, a.dim, here, [&](int r) {
      const int i = a.by_group.div(r);
      return q + i * a.sq.t + (r - i * a.group) * a.sq.h;
    });
    stage<DH>(lds_address(lds[buf][1]), r0, a.rows, a.dim, here, [&](int r) {
      const int i = a.by_group.div(r);
      return dout + i * a.sdo.t + (r - i * a.group) * a.sdo.h;
    });
  };
  // rows past the last have an infinite sum: they weigh zero
  float sm = INFINITY, sd = 0.0f, ss = 0.0f;
  int2 sk = make_int2(0, 0);
  int sp = 0;
  const auto look = [&](int r0) {
    sm = INFINITY, sd = 0.0f, ss = 0.0f, sk = make_int2(0, 0), sp = 0;
    if (tid < KT && r0 + tid < a.rows) {
      const int i = a.by_group.div(r0 + tid), head = at.kh * a.group + r0 + tid - i * a.group;
      const float2 st = row_stats(a, at.b, head, i);
      sm = st.x, sd = st.y, sp = a.q_offset + i;
      sk = seq.keys(a, sp);
      if (a.slopes) ss = a.slopes[head] * LOG2E;
    }
  };
  const auto note = [&](int buf) {
    if (tid < KT) {
      RowInfo& w = info[buf];
      w.sum[tid] = sm, w.delta[tid] = sd, w.slope[tid] = ss;
      w.position[tid] = sp, w.lo[tid] = sk.x, w.hi[tid] = sk.y;
    }
  };
  if (begin < end) {
    fetch(begin, 0);
    look(begin);
    note(0);
  }
  bf16x8_t fk[DH / 16], fv[DH / 16];
  f32x16_t dk[DH / 32], dv[DH / 32];
  const int kc = min(key, a.kv_len - 1), dim = kc < seq.limit ? a.dim : 0;
  load_row<DH>(a.k + at.b * a.sk.b + kc * a.sk.t + at.kh * a.sk.h, dim, lane, fk);
  load_row<DH>(a.v + at.b * a.sv.b + kc * a.sv.t + at.kh * a.sv.h, dim, lane, fv);
  zero(dk);
  zero(dv);
  int buf = 0;
  for (int r0 = begin; r0 < end; r0 += KT, buf ^= 1) {
    landed();
    __syncthreads();
    const bool more = r0 + KT < end;
    if (more) {
      fetch(r0 + KT, buf ^ 1);
      look(r0 + KT);
    }
    const RowInfo& w = info[buf];
    const int tail = min(KT, a.rows - r0) - 1;
    if (wkey0 < valid && wkey0 < w.hi[tail] && wkey0 + 32 > w.lo[0]) {
      const char *Qs = lds[buf][0], *Os = lds[buf][1];
      const bool cut = wkey0 < w.lo[tail] || wkey0 + 32 > w.hi[0];
#pragma unroll 1
      for (int n = 0; n < KT / 32; ++n) {
        const Lane<DH> lf = frag.here();
        f32x16_t s = product<DH>(fk, Qs, 32 * n, lf);
        f32x16_t dp = product<DH>(fv, Os, 32 * n, lf);
        f32x16_t t;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          float tr;
          s[r] = score<CAP>(a, s[r], tr);
          if (CAP) t[r] = tr;
        }
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
          const int c = 32 * n + col_of(4 * g, lane);
          const float4 su = *reinterpret_cast<const float4*>(w.sum + c);
          const float4 de = *reinterpret_cast<const float4*>(w.delta + c);
          const float sus[4] = {su.x, su.y, su.z, su.w}, des[4] = {de.x, de.y, de.z, de.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int r = 4 * g + e;
            s[r] = __builtin_amdgcn_exp2f(s[r] - sus[e]);
            dp[r] = s[r] * (dp[r] - des[e]);
            if (CAP) dp[r] *= 1.0f - t[r] * t[r];
          }
        }
        if (cut) {   // both, also where dP is not finite
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int c = 32 * n + col_of(r, lane);
            if (key < w.lo[c] || key >= w.hi[c]) s[r] = dp[r] = 0.0f;
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
    if (more) note(buf ^ 1);
  }
  if (key >= a.kv_len) return;
  if (a.pieces > 1) {
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

// Into how many pieces the walk of each of `blocks` tiles is cut: few blocks of
// a long walk leave CUs idle, and a causal walk ends in its longest block. At
// least `least` steps stay in a piece, so that a partial result's write and
// read stay small beside its products.
int pieces_for(long blocks, long steps, long want, long least) {
  if (blocks <= 0 || steps <= 0) return 1;
  return static_cast<int>(std::max(1L, std::min({(want + blocks - 1) / blocks, steps / least, 128L})));
}

struct Plan {
  bool few;                      // forward by the kernel for few rows
  int fwd, dq, dkv;              // pieces
};
Plan plan(const AttentionArgs& a) {
  Plan p;
  const long bh = static_cast<long>(a.batch) * a.kv_heads;
  const long row_tiles = (a.rows + ROWS - 1L) / ROWS, key_tiles = (a.kv_len + ROWS - 1L) / ROWS;
  p.few = a.rows <= 64;
  p.fwd = p.few ? pieces_for(bh * ((a.rows + 31) / 32), (a.kv_len + 127L) / 128, 1024, 2)
                : pieces_for(bh * row_tiles, (a.kv_len + KT - 1L) / KT, 768, 8);
  p.dq = pieces_for(bh * row_tiles, (a.kv_len + KT - 1L) / KT, 768, 8);
  p.dkv = pieces_for(bh * key_tiles, (a.rows + KT - 1L) / KT, 1024, 8);
  return p;
}
size_t part_bytes(int pieces, size_t rows, int dim) {
  return pieces > 1 ? round256(static_cast<size_t>(pieces) * rows * dim * sizeof(float)) : 0;
}

// Launch-independent values, and the document runs if there are documents.
hipError_t prepare(const AttentionArgs& in, Args& a, hipStream_t s) {
  static_cast<AttentionArgs&>(a) = in;
  a.by_group = FastDiv(in.group);
  a.by_bh = FastDiv(in.batch * in.kv_heads);
  a.by_kv = FastDiv(in.kv_heads);
  a.c1 = in.cap > 0.0f ? 2.0f * in.scale / in.cap * LOG2E : in.scale * LOG2E;
  a.c2 = in.cap * LOG2E;
  if (!in.documents || in.kv_len == 0) return hipSuccess;
  int2* runs = reinterpret_cast<int2*>(in.ws);
  a.doc = runs;
  const unsigned chunks = (in.kv_len + DT - 1) / DT;
  hipLaunchKernelGGL(document_runs_kernel, dim3(chunks * in.batch), dim3(DT), 0, s, in.documents, in.kv_len,
                     FastDiv(chunks), runs);
  return hipGetLastError();
}

// Calls f with the smallest compiled head width that holds dim, and the cap.
template <typename F>
void with_width(int dim, bool cap, F&& f) {
  auto pick = [&](auto width) {
    if (cap) f(width, std::true_type{});
    else f(width, std::false_type{});
  };
  if (dim <= 32) pick(std::integral_constant<int, 32>{});
  else if (dim <= 64) pick(std::integral_constant<int, 64>{});
  else if (dim <= 96) pick(std::integral_constant<int, 96>{});
  else pick(std::integral_constant<int, 128>{});
}

template <typename K>
hipError_t launch(K* kernel, Args& a, long length, int tile, int pieces, hipStream_t s) {
  a.tiles = static_cast<int>((length + tile - 1) / tile);
  a.pieces = pieces;
  a.by_pieces = FastDiv(pieces);
  hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(a.tiles) * pieces * a.batch * a.kv_heads), dim3(NT), 0, s, a);
  return hipGetLastError();
}

}  // namespace

size_t attention_ws_bytes(const AttentionArgs& a, bool backward) {
  const Plan p = plan(a);
  const size_t forward = doc_bytes(a) + part_bytes(p.fwd, q_rows(a), a.dim) +
                         (p.fwd > 1 ? round256(p.fwd * q_rows(a) * sizeof(float2)) : 0);
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
  with_width(a.dim, a.cap > 0.0f, [&](auto width, auto cap) {
    e = p.few ? launch(attention_masked_few_kernel<width(), cap()>, a, a.rows, 32, p.fwd, s)
              : launch(attention_masked_fwd_kernel<width(), cap()>, a, a.rows, ROWS, p.fwd, s);
  });
  if (e != hipSuccess || p.fwd == 1) return e;
  const long rows = static_cast<long>(q_rows(in));
  hipLaunchKernelGGL(attention_join_kernel, dim3(static_cast<unsigned>((rows + NT / 16 - 1) / (NT / 16))), dim3(NT), 0,
                     s, a, rows, FastDiv(a.q_len), FastDiv(a.heads));
  return hipGetLastError();
}

hipError_t attention_masked_bwd(const AttentionArgs& in, hipStream_t s) {
  if (in.batch == 0) return hipSuccess;
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
  Sums sums;
  sums.dim = a.dim;
  int nsums = 0;
  long most = 0;
  const auto sum = [&](const float* part, bf16_t* out, const AttentionArgs::Strides& to, size_t rows, int heads,
                       int tokens, int pieces) {
    sums.sum[nsums++] = {part, out, to, static_cast<long>(rows), FastDiv(heads), FastDiv(tokens), pieces};
    most = std::max(most, static_cast<long>(rows));
  };
  if (a.q_len > 0) {
    const long rows = static_cast<long>(q_rows(in));
    hipLaunchKernelGGL(attention_delta_kernel, dim3(static_cast<unsigned>((rows + NT / 16 - 1) / (NT / 16))), dim3(NT),
                       0, s, a, rows, FastDiv(a.heads), FastDiv(a.q_len));
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  with_width(a.dim, a.cap > 0.0f, [&](auto width, auto cap) {
    if (a.q_len > 0) {
      a.part = part_q;
      e = launch(attention_masked_dq_kernel<width(), cap()>, a, a.rows, ROWS, p.dq, s);
      if (e != hipSuccess) return;
      if (p.dq > 1) sum(part_q, a.dq, a.sdq, q_rows(in), a.heads, a.q_len, p.dq);
    }
    if (a.kv_len == 0) return;
    a.part = part_k;
    a.part2 = part_v;
    e = launch(attention_masked_dkv_kernel<width(), cap()>, a, a.kv_len, ROWS, p.dkv, s);
    if (e != hipSuccess) return;
    if (p.dkv > 1) {
      sum(part_k, a.dk, a.sdk, k_rows(in), a.kv_heads, a.kv_len, p.dkv);
      sum(part_v, a.dv, a.sdv, k_rows(in), a.kv_heads, a.kv_len, p.dkv);
    }
  });
  if (e != hipSuccess || nsums == 0) return e;
  hipLaunchKernelGGL(attention_sum_kernel, dim3(static_cast<unsigned>((most + NT / 16 - 1) / (NT / 16)), nsums),
                     dim3(NT), 0, s, sums);
  return hipGetLastError();
}

}  // namespace spx
