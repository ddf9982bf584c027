// Argument checks of the stand-alone operators, and the quantities their
// kernels take that depend on the arguments alone.
#include "operators.hpp"

#include <algorithm>
#include <cmath>

namespace spx {
namespace {

void fail(const std::string& m) { throw StageError(SPECTRAIN_EINVAL, m); }

bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

constexpr int64_t MAX_STRIDE = int64_t{1} << 40;   // elements; keeps every offset inside 63 bits

void check_strides(const spectrain_strides& st, int multiple, const char* what) {
  for (int64_t v : {st.batch, st.token, st.head}) {
    if (v < 0 || v > MAX_STRIDE) fail(std::string(what) + " strides must lie in [0, 2^40]");
    if (v % multiple) fail(std::string(what) + " strides must be multiples of " + std::to_string(multiple));
  }
}

// A written tensor's elements are distinct: each dimension steps over all that
// the closer-strided ones span.
void check_written(const spectrain_strides& st, int64_t batch, int64_t tokens, int64_t heads, int64_t dim,
                   const char* what) {
  if (batch == 0 || tokens == 0 || heads == 0) return;
  std::pair<int64_t, int64_t> d[3] = {{st.batch, batch}, {st.token, tokens}, {st.head, heads}};
  std::sort(d, d + 3);
  long double span = static_cast<long double>(dim);
  for (const auto& [stride, size] : d) {
    if (size < 2) continue;
    if (static_cast<long double>(stride) < span) fail(std::string(what) + " strides make its elements overlap");
    span += static_cast<long double>(stride) * (size - 1);
  }
}

}  // namespace

// ----------------------------------------------------------------- rotary ----
void run_rotary(const spectrain_rotary_desc* desc, const void* x, const int32_t* positions, int inverse, void* out,
                hipStream_t s) {
  if (!desc) fail("desc is NULL");
  const spectrain_rotary_desc& d = *desc;
  if (d.abi_version != SPECTRAIN_ABI_VERSION) fail("abi_version mismatch");
  if (d.dtype != SPECTRAIN_FP32 && d.dtype != SPECTRAIN_BF16) fail("unknown dtype");
  if (d.batch < 0 || d.tokens < 0 || d.heads < 0) fail("batch, tokens and heads must be >= 0");
  if (d.head_dim < 2 || d.head_dim > 256) fail("head_dim must lie in [2, 256]");
  if (d.rotary_dim < 2 || d.rotary_dim > d.head_dim || d.rotary_dim % 2)
    fail("rotary_dim must be even and lie in [2, head_dim]");
  if (d.layout != SPECTRAIN_ROTARY_HALF && d.layout != SPECTRAIN_ROTARY_INTERLEAVED) fail("unknown rotary layout");
  if (d.scaling < SPECTRAIN_ROTARY_UNSCALED || d.scaling > SPECTRAIN_ROTARY_PARTS) fail("unknown rotary scaling");
  if (d.reserved != 0) fail("reserved must be 0");
  if (!(d.base > 1.0) || !std::isfinite(d.base)) fail("base must be finite and > 1");
  if (d.scaling != SPECTRAIN_ROTARY_UNSCALED && (!(d.factor >= 1.0) || !std::isfinite(d.factor)))
    fail("factor must be finite and >= 1");
  if (d.scaling == SPECTRAIN_ROTARY_PARTS && d.original_length < 1) fail("original_length must be >= 1");
  check_strides(d.x, 1, "x");
  check_strides(d.out, 1, "out");
  const int64_t rows = static_cast<int64_t>(d.batch) * d.tokens;
  if (rows >= 1 << 24 || d.heads > 65535) fail("batch * tokens must be below 2^24 and heads below 2^16");
  if (rows == 0 || d.heads == 0) return;
  if (!x || !out) fail("x and out must not be NULL");
  check_written(d.out, d.batch, d.tokens, d.heads, d.head_dim, "out");
  const size_t esz = d.dtype == SPECTRAIN_BF16 ? 2 : 4;
  if (!aligned(x, esz) || !aligned(out, esz) || !aligned(positions, 4)) fail("a tensor is not aligned to its elements");
  if (x == out && (d.x.batch != d.out.batch || d.x.token != d.out.token || d.x.head != d.out.head))
    fail("in place, x and out must have the same strides");

  RotaryArgs a;
  a.x = x;
  a.out = out;
  a.positions = positions;
  a.first = positions ? 0 : d.first_position;
  a.tokens = d.tokens;
  a.rows = static_cast<int>(rows);
  a.heads = d.heads;
  a.dim = d.head_dim;
  a.rot = d.rotary_dim;
  a.xb = d.x.batch;
  a.xt = d.x.token;
  a.xh = d.x.head;
  a.ob = d.out.batch;
  a.ot = d.out.token;
  a.oh = d.out.head;
  a.interleaved = d.layout == SPECTRAIN_ROTARY_INTERLEAVED;
  a.sign = inverse ? -1.0f : 1.0f;
  a.magnitude = d.scaling == SPECTRAIN_ROTARY_PARTS ? static_cast<float>(0.1 * std::log(d.factor) + 1.0) : 1.0f;
  const double tau = 6.283185307179586476925;
  double base = d.base;
  if (d.scaling == SPECTRAIN_ROTARY_NTK && d.rotary_dim > 2)
    base *= std::pow(d.factor, static_cast<double>(d.rotary_dim) / (d.rotary_dim - 2));
  // powers by repeated multiplication: off by at most 128 x 2^-53, 2^-26 of a
  // turn at position 2^20, and a call's 128 std::pow would take longer than its launch
  const double ratio = std::pow(base, -2.0 / d.rotary_dim);
  double power = 1.0;
  for (int i = 0; i < d.rotary_dim / 2; ++i, power *= ratio) {
    double w = power;
    if (d.scaling == SPECTRAIN_ROTARY_LINEAR) w /= d.factor;
    if (d.scaling == SPECTRAIN_ROTARY_PARTS) {
      const double turns = d.original_length * w / tau;
      const double keep = std::min(std::max((turns - 1.0) / 31.0, 0.0), 1.0);
      w *= keep + (1.0 - keep) / d.factor;
    }
    a.turns[i] = w / tau;   // turns per position
  }
  hip_check(rotary(a, d.dtype, s), "rotary");
}

// -------------------------------------------------------------- attention ----
namespace {

// layout: whether strides are looked at (they do not change the workspace).
AttentionArgs attention_args(const spectrain_attention_desc* desc, bool backward, bool layout = true) {
  if (!desc) fail("desc is NULL");
  const spectrain_attention_desc& d = *desc;
  if (d.abi_version != SPECTRAIN_ABI_VERSION) fail("abi_version mismatch");
  if (d.dtype != SPECTRAIN_BF16) fail("attention runs in bf16 only");
  if (d.batch < 0 || d.q_len < 0 || d.kv_len < 0) fail("batch, q_len and kv_len must be >= 0");
  if (d.heads < 1 || d.kv_heads < 1 || d.heads % d.kv_heads) fail("heads must be a positive multiple of kv_heads");
  if (d.head_dim < 8 || d.head_dim > 128 || d.head_dim % 8) fail("head_dim must be a multiple of 8 up to 128");
  if (d.causal != 0 && d.causal != 1) fail("causal must be 0 or 1");
  if (!std::isfinite(d.scale)) fail("scale must be finite");
  if (!(d.cap >= 0.0f) || !std::isfinite(d.cap)) fail("cap must be finite and >= 0");
  // scores and the factors that form them stay finite
  constexpr float LARGEST = 1.2676506e30f;   // 2^100
  if (std::fabs(d.scale) > LARGEST || (d.cap > 0.0f && (d.cap > LARGEST || std::fabs(d.scale) > d.cap * LARGEST)))
    fail("|scale|, cap and |scale| / cap must be at most 2^100");
  constexpr int MAX_LEN = 1 << 30;   // positions and tile ends stay inside 32 bits
  if (d.q_len > MAX_LEN || d.kv_len > MAX_LEN || d.q_offset > MAX_LEN || d.q_offset < -MAX_LEN)
    fail("q_len, kv_len and |q_offset| must be at most 2^30");
  const int64_t rows = static_cast<int64_t>(d.q_len) * (d.heads / d.kv_heads);
  if (rows > MAX_LEN) fail("q_len * heads / kv_heads must be at most 2^30");
  const int64_t bh = static_cast<int64_t>(d.batch) * d.heads;
  // grids of up to 2^32 - 1 threads
  if (bh * ((d.q_len + 31) / 32) >= 1 << 23 || bh * ((d.kv_len + 31) / 32) >= 1 << 23)
    fail("batch * heads * length / 32 must be below 2^23");
  if (layout) {
    check_strides(d.q, 8, "q");
    check_strides(d.k, 8, "k");
    check_strides(d.v, 8, "v");
    check_strides(d.out, 8, "out");
    check_written(d.out, d.batch, d.q_len, d.heads, d.head_dim, "out");
    if (backward) {
      check_written(d.dq, d.batch, d.q_len, d.heads, d.head_dim, "dq");
      check_written(d.dk, d.batch, d.kv_len, d.kv_heads, d.head_dim, "dk");
      check_written(d.dv, d.batch, d.kv_len, d.kv_heads, d.head_dim, "dv");
      check_strides(d.dout, 8, "dout");
      check_strides(d.dq, 8, "dq");
      check_strides(d.dk, 8, "dk");
      check_strides(d.dv, 8, "dv");
    }
  }
  if (layout) {   // byte offsets inside a tile of 64 rows are 32 bits wide
    const int64_t g = d.heads / d.kv_heads, q = std::min<int64_t>(d.q_len, 64 / g + 2), k = std::min(d.kv_len, 64);
    const auto span = [&](const spectrain_strides& st, int64_t tokens, int64_t heads, const char* what) {
      if (std::max<int64_t>(tokens - 1, 0) * st.token + (heads - 1) * st.head >= int64_t{1} << 29)
        fail(std::string(what) + ": 64 tokens, and the heads of a group, may span at most 2^29 elements");
    };
    span(d.q, q, g, "q");
    span(d.k, k, 1, "k");
    span(d.v, k, 1, "v");
    if (backward) span(d.dout, q, g, "dout");
  }
  AttentionArgs a;
  a.batch = d.batch;
  a.heads = d.heads;
  a.kv_heads = d.kv_heads;
  a.group = d.heads / d.kv_heads;
  a.dim = d.head_dim;
  a.q_len = d.q_len;
  a.kv_len = d.kv_len;
  a.q_offset = d.q_offset;
  a.rows = static_cast<int>(rows);
  a.causal = d.causal;
  a.scale = d.scale;
  a.cap = d.cap;
  a.sq = {d.q.batch, d.q.token, d.q.head};
  a.sk = {d.k.batch, d.k.token, d.k.head};
  a.sv = {d.v.batch, d.v.token, d.v.head};
  a.so = {d.out.batch, d.out.token, d.out.head};
  a.sdo = {d.dout.batch, d.dout.token, d.dout.head};
  a.sdq = {d.dq.batch, d.dq.token, d.dq.head};
  a.sdk = {d.dk.batch, d.dk.token, d.dk.head};
  a.sdv = {d.dv.batch, d.dv.token, d.dv.head};
  return a;
}

void attention_masks(AttentionArgs& a, const spectrain_attention_masks* m) {
  if (m) {
    a.documents = m->documents;
    a.prefix = m->prefix;
    a.kv_lengths = m->kv_lengths;
    a.slopes = m->slopes;
    for (const void* p : {static_cast<const void*>(m->documents), static_cast<const void*>(m->prefix),
                          static_cast<const void*>(m->kv_lengths), static_cast<const void*>(m->slopes)})
      if (!aligned(p, 4)) fail("a mask is not 4-byte aligned");
  }
  if (a.prefix && !a.causal) fail("prefix needs causal");
  if (a.documents && (a.q_offset < 0 || a.q_offset + static_cast<int64_t>(a.q_len) > a.kv_len))
    fail("documents need 0 <= q_offset and q_offset + q_len <= kv_len");
  if (a.documents && static_cast<int64_t>(a.batch) * ((a.kv_len + 1023) / 1024) >= 1 << 22)
    fail("documents need batch * kv_len / 1024 below 2^22");
}

void check_workspace(const void* ws, size_t ws_bytes, size_t need) {
  if (need && (!ws || ws_bytes < need))
    fail("workspace of " + std::to_string(ws_bytes) + " bytes is smaller than the " + std::to_string(need) +
         " bytes needed");
  if (!aligned(ws, 256)) fail("workspace must be 256-byte aligned");
}

void check_tensor(const void* p, int64_t elements, const char* what) {
  if (elements && !p) fail(std::string(what) + " is NULL");
  if (!aligned(p, 16)) fail(std::string(what) + " must be 16-byte aligned");
}

}  // namespace

size_t attention_workspace(const spectrain_attention_desc* desc, bool backward) {
  const AttentionArgs a = attention_args(desc, backward, false);
  return attention_ws_bytes(a, backward);
}

void check_attention_masks(const spectrain_attention_desc* desc, const spectrain_attention_masks* masks) {
  AttentionArgs a = attention_args(desc, false, false);
  attention_masks(a, masks);
}

void run_attention_forward(const spectrain_attention_desc* desc, const spectrain_attention_masks* masks, const void* q,
                           const void* k, const void* v, void* out, float* lse, void* ws, size_t ws_bytes,
                           hipStream_t s) {
  AttentionArgs a = attention_args(desc, false);
  attention_masks(a, masks);
  check_workspace(ws, ws_bytes, attention_ws_bytes(a, false));
  const int64_t nq = static_cast<int64_t>(a.batch) * a.q_len, nk = static_cast<int64_t>(a.batch) * a.kv_len;
  check_tensor(q, nq, "q");
  check_tensor(k, nk, "k");
  check_tensor(v, nk, "v");
  check_tensor(out, nq, "out");
  if (!aligned(lse, 4)) fail("lse must be 4-byte aligned");
  if (nq && (out == q || out == k || out == v)) fail("out must not be an input");
  a.q = static_cast<const bf16_t*>(q);
  a.k = static_cast<const bf16_t*>(k);
  a.v = static_cast<const bf16_t*>(v);
  a.out = static_cast<bf16_t*>(out);
  a.lse = lse;
  a.ws = static_cast<char*>(ws);
  hip_check(attention_masked_fwd(a, s), "attention_masked");
}

void run_attention_backward(const spectrain_attention_desc* desc, const spectrain_attention_masks* masks, const void* q,
                            const void* k, const void* v, const void* out, const float* lse, const void* dout,
                            void* dq, void* dk, void* dv, void* ws, size_t ws_bytes, hipStream_t s) {
  AttentionArgs a = attention_args(desc, true);
  attention_masks(a, masks);
  check_workspace(ws, ws_bytes, attention_ws_bytes(a, true));
  const int64_t nq = static_cast<int64_t>(a.batch) * a.q_len, nk = static_cast<int64_t>(a.batch) * a.kv_len;
  check_tensor(q, nq, "q");
  check_tensor(k, nk, "k");
  check_tensor(v, nk, "v");
  check_tensor(out, nq, "out");
  check_tensor(dout, nq, "dout");
  check_tensor(dq, nq, "dq");
  check_tensor(dk, nk, "dk");
  check_tensor(dv, nk, "dv");
  if (nq && !lse) fail("lse is NULL");
  if (!aligned(lse, 4)) fail("lse must be 4-byte aligned");
  for (const void* g : {static_cast<const void*>(dq), static_cast<const void*>(dk), static_cast<const void*>(dv)})
    for (const void* in : {q, k, v, out, dout})
      if (g && g == in) fail("a gradient must not be an input");
  if (dq && (dq == dk || dq == dv)) fail("the gradients must not overlap");
  if (dk && dk == dv) fail("the gradients must not overlap");
  a.q = static_cast<const bf16_t*>(q);
  a.k = static_cast<const bf16_t*>(k);
  a.v = static_cast<const bf16_t*>(v);
  a.out = const_cast<bf16_t*>(static_cast<const bf16_t*>(out));
  a.lse = const_cast<float*>(lse);
  a.dout = static_cast<const bf16_t*>(dout);
  a.dq = static_cast<bf16_t*>(dq);
  a.dk = static_cast<bf16_t*>(dk);
  a.dv = static_cast<bf16_t*>(dv);
  a.ws = static_cast<char*>(ws);
  hip_check(attention_masked_bwd(a, s), "attention_masked_bwd");
}

// ------------------------------------------------------------- checkpoint ----
void run_checkpoint(int dtype, int64_t rows, int64_t cols, const void* x, int64_t ld, uint8_t* codes, uint8_t* scales,
                    void* out, hipStream_t s) {
  if (dtype != SPECTRAIN_FP32 && dtype != SPECTRAIN_BF16) fail("unknown dtype");
  if (rows < 0 || cols < 0) fail("rows and cols must be >= 0");
  if (ld < cols || ld > MAX_STRIDE) fail("ld must lie in [cols, 2^40]");
  if (rows == 0 || cols == 0) return;
  // grids of up to 2^32 - 1 threads, four to a group of values
  if (cols >= 1 << 30 || rows >= 1 << 30 || rows * ((cols + 31) / 32) > (1 << 30) - 64)
    fail("cols must be below 2^30 and rows * ceil(cols / 32) at most 2^30 - 64");
  if ((!x && !out) || !codes || !scales) fail("a tensor is NULL");
  if (!aligned(x, dtype == SPECTRAIN_BF16 ? 2 : 4) || !aligned(out, dtype == SPECTRAIN_BF16 ? 2 : 4))
    fail("a tensor is not aligned to its elements");
  CheckpointArgs a;
  a.x = x;
  a.out = out;
  a.codes = codes;
  a.scales = scales;
  a.rows = rows;
  a.cols = cols;
  a.ld = ld;
  hip_check(x ? checkpoint_pack(&a, 1, dtype, s) : checkpoint_restore(&a, 1, dtype, s), x ? "checkpoint_pack"
                                                                                  : "checkpoint_restore");
}

}  // namespace spx
