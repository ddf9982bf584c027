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

// --------------------------------------------------- linear layers in 8 bits ----
namespace {

constexpr int64_t MAX_CODES_LD = int64_t{1} << 22;   // byte offsets inside a tile of 256 rows stay below 2^30

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

void check_version(uint32_t v) {
  if (v != SPECTRAIN_ABI_VERSION) fail("abi_version mismatch");
}

void check_dtype(int dtype, const char* what) {
  if (dtype != SPECTRAIN_FP32 && dtype != SPECTRAIN_BF16) fail(std::string("unknown ") + what);
}

size_t bytes_of(int dtype) { return dtype == SPECTRAIN_BF16 ? 2 : 4; }

// Elements between rows of a matrix.
void check_ld(int64_t ld, int64_t cols, const char* what) {
  if (ld < cols || ld > MAX_STRIDE) fail(std::string(what) + " must lie in [" + std::to_string(cols) + ", 2^40]");
}

void check_elements(const void* p, int dtype, const char* what) {
  if (!aligned(p, bytes_of(dtype))) fail(std::string(what) + " is not aligned to its elements");
}

// Lines of codes or scale bytes.
void check_lines(const void* p, int64_t ld, int64_t bytes, int64_t most, const char* what) {
  if (ld < bytes || ld > most || ld % 16)
    fail(std::string(what) + "_ld must be a multiple of 16 in [" + std::to_string(bytes) + ", " +
         std::to_string(most) + "]");
  if (!aligned(p, 16)) fail(std::string(what) + " must be 16-byte aligned");
}

void check_blocks(const void* codes, const void* scales, int64_t rows, int64_t cols, int64_t codes_ld,
                  int64_t scales_ld, const char* what) {
  if (!codes != !scales) fail(std::string(what) + " go with their scales");
  if (!codes) return;
  check_lines(codes, codes_ld, cols, MAX_CODES_LD, what);
  check_lines(scales, scales_ld, rows, MAX_STRIDE, (std::string(what) + " scales").c_str());
  if (codes == scales) fail(std::string(what) + " and their scales overlap");
}

BlocksArgs blocks_args(const spectrain_blocks_desc* desc) {
  if (!desc) fail("desc is NULL");
  const spectrain_blocks_desc& d = *desc;
  check_version(d.abi_version);
  check_dtype(d.dtype, "dtype");
  if (d.reserved != 0) fail("reserved must be 0");
  if (d.rows < 0 || d.cols < 0) fail("rows and cols must be >= 0");
  if (d.rows >= int64_t{1} << 31 || d.cols >= int64_t{1} << 31) fail("rows and cols must be below 2^31");
  if (ceil_div(d.rows, 128) * ceil_div(d.cols, 128) > 1 << 23)
    fail("ceil(rows / 128) * ceil(cols / 128) must be at most 2^23");
  check_ld(d.ld, d.cols, "ld");
  BlocksArgs a;
  a.rows = d.rows;
  a.cols = d.cols;
  a.ld = d.ld;
  a.codes_ld = d.codes_ld;
  a.scales_ld = d.scales_ld;
  a.t_ld = d.transposed_ld;
  a.t_scales_ld = d.transposed_scales_ld;
  return a;
}

}  // namespace

void run_blocks_pack(const spectrain_blocks_desc* desc, const void* x, uint8_t* codes, uint8_t* scales, uint8_t* t_codes,
                     uint8_t* t_scales, hipStream_t s) {
  BlocksArgs a = blocks_args(desc);
  if (desc->shape != SPECTRAIN_BLOCKS_ROWS && desc->shape != SPECTRAIN_BLOCKS_TILES) fail("unknown shape");
  check_blocks(codes, scales, a.rows, a.cols, a.codes_ld, a.scales_ld, "codes");
  check_blocks(t_codes, t_scales, a.cols, a.rows, a.t_ld, a.t_scales_ld, "transposed");
  if (a.rows == 0 || a.cols == 0) return;
  if (!x || (!codes && !t_codes)) fail("a tensor is NULL");
  check_elements(x, desc->dtype, "x");
  if (codes && t_codes && (t_codes == codes || t_codes == scales || t_scales == codes || t_scales == scales))
    fail("the outputs must not overlap");
  for (const void* p : {static_cast<const void*>(codes), static_cast<const void*>(scales),
                        static_cast<const void*>(t_codes), static_cast<const void*>(t_scales)})
    if (p == x) fail("an output must not be x");
  a.x = x;
  a.codes = codes;
  a.scales = scales;
  a.t_codes = t_codes;
  a.t_scales = t_scales;
  a.tiles = desc->shape == SPECTRAIN_BLOCKS_TILES;
  hip_check(blocks_pack(a, desc->dtype, s), "blocks_pack");
}

void run_blocks_restore(const spectrain_blocks_desc* desc, const uint8_t* codes, const uint8_t* scales, void* out,
                        hipStream_t s) {
  BlocksArgs a = blocks_args(desc);
  check_blocks(codes, scales, a.rows, a.cols, a.codes_ld, a.scales_ld, "codes");
  if (a.rows == 0 || a.cols == 0) return;
  if (!codes || !out) fail("a tensor is NULL");
  check_elements(out, desc->dtype, "out");
  if (out == codes || out == scales) fail("out must not be an input");
  a.codes = const_cast<uint8_t*>(codes);
  a.scales = const_cast<uint8_t*>(scales);
  a.out = out;
  hip_check(blocks_restore(a, desc->dtype, s), "blocks_restore");
}

// --------------------------------------------------------------- rms norm ----
namespace {

RmsNormArgs rms_norm_args(const spectrain_rms_norm_desc* desc) {
  if (!desc) fail("desc is NULL");
  const spectrain_rms_norm_desc& d = *desc;
  check_version(d.abi_version);
  check_dtype(d.dtype, "dtype");
  check_dtype(d.out_dtype, "out_dtype");
  check_dtype(d.weight_dtype, "weight_dtype");
  if (d.out_dtype != d.dtype && d.out_dtype != SPECTRAIN_BF16) fail("out_dtype must be dtype or bf16");
  if (d.reserved != 0) fail("reserved must be 0");
  if (!(d.eps > 0.0f) || !std::isfinite(d.eps)) fail("eps must be finite and > 0");
  if (d.rows < 0 || d.rows >= int64_t{1} << 31) fail("rows must lie in [0, 2^31)");
  if (d.cols < 1 || d.cols > RMS_NORM_COLS) fail("cols must lie in [1, 32768]");
  RmsNormArgs a;
  a.rows = d.rows;
  a.cols = d.cols;
  a.dtype = d.dtype;
  a.out_dtype = d.out_dtype;
  a.weight_dtype = d.weight_dtype;
  a.eps = d.eps;
  return a;
}

// A matrix that may be absent: its ld is looked at only where it is given.
long given_ld(const void* p, int64_t ld, int64_t cols, int dtype, const char* what) {
  if (!p) return 0;
  check_ld(ld, cols, (std::string(what) + "_ld").c_str());
  check_elements(p, dtype, what);
  return ld;
}

}  // namespace

void run_rms_norm_forward(const spectrain_rms_norm_desc* desc, const void* x, const void* residual, const void* weight,
                          void* sum, void* y, uint8_t* codes, uint8_t* scales, float* rstd, hipStream_t s) {
  RmsNormArgs a = rms_norm_args(desc);
  const spectrain_rms_norm_desc& d = *desc;
  a.x_ld = given_ld(x, d.x_ld, a.cols, d.dtype, "x");
  a.residual_ld = given_ld(residual, d.residual_ld, a.cols, d.dtype, "residual");
  a.sum_ld = given_ld(sum, d.sum_ld, a.cols, d.dtype, "sum");
  a.y_ld = given_ld(y, d.y_ld, a.cols, d.out_dtype, "y");
  check_elements(weight, d.weight_dtype, "weight");
  check_blocks(codes, scales, a.rows, a.cols, d.codes_ld, d.scales_ld, "codes");
  if (!aligned(rstd, 4)) fail("rstd must be 4-byte aligned");
  if (sum && !residual) fail("sum goes with a residual");
  if (a.rows == 0) return;
  if (!x || !weight || (!y && !codes)) fail("a tensor is NULL");
  if (sum && ((sum == x && a.sum_ld != a.x_ld) || (sum == residual && a.sum_ld != a.residual_ld)))
    fail("in place, sum must have the same ld");
  for (const void* o : {static_cast<const void*>(y), static_cast<const void*>(codes), static_cast<const void*>(scales),
                        static_cast<const void*>(rstd)})
    if (o && (o == x || o == residual || o == weight || o == sum)) fail("an output must not be an input or the sum");
  if (sum && sum == weight) fail("an output must not be an input or the sum");
  if (codes && (codes == y || scales == y)) fail("the outputs must not overlap");
  a.x = x;
  a.residual = residual;
  a.weight = weight;
  a.sum = sum;
  a.y = y;
  a.codes = codes;
  a.scales = scales;
  a.codes_ld = d.codes_ld;
  a.scales_ld = d.scales_ld;
  a.rstd = rstd;
  hip_check(rms_norm_fwd(a, s), "rms_norm");
}

size_t rms_norm_workspace(const spectrain_rms_norm_desc* desc) {
  const RmsNormArgs a = rms_norm_args(desc);
  return rms_norm_ws_bytes(a.rows, a.cols);
}

void run_rms_norm_backward(const spectrain_rms_norm_desc* desc, const void* dy, const void* h, const void* weight,
                           const float* rstd, const void* dsum, void* dx, float* dweight, void* ws, size_t ws_bytes,
                           hipStream_t s) {
  RmsNormArgs a = rms_norm_args(desc);
  const spectrain_rms_norm_desc& d = *desc;
  check_workspace(ws, ws_bytes, rms_norm_ws_bytes(a.rows, a.cols));
  a.dy_ld = given_ld(dy, d.dy_ld, a.cols, d.out_dtype, "dy");
  a.sum_ld = given_ld(h, d.sum_ld, a.cols, d.dtype, "sum");
  a.dsum_ld = given_ld(dsum, d.dsum_ld, a.cols, d.dtype, "dsum");
  a.dx_ld = given_ld(dx, d.dx_ld, a.cols, d.dtype, "dx");
  check_elements(weight, d.weight_dtype, "weight");
  if (!aligned(rstd, 4) || !aligned(dweight, 4)) fail("rstd and dweight must be 4-byte aligned");
  if (!dweight) fail("dweight is NULL");
  if (a.rows && (!dy || !h || !weight || !rstd || !dx)) fail("a tensor is NULL");
  if (dx && (dx == h || dx == weight || dx == rstd || dx == dweight)) fail("dx must not be h, weight, rstd or dweight");
  for (const void* p : {dy, h, weight, static_cast<const void*>(rstd), dsum})
    if (p == dweight) fail("dweight must not be an input");
  if (dx && dx == dsum && a.dx_ld != a.dsum_ld) fail("in place, dx must have the same ld");
  if (dx && dx == dy && (a.dx_ld != a.dy_ld || d.dtype != d.out_dtype)) fail("in place, dx must have the same ld and type");
  a.dy = dy;
  a.x = h;
  a.weight = weight;
  a.rstd = const_cast<float*>(rstd);
  a.dsum = dsum;
  a.dx = dx;
  a.dweight = dweight;
  a.ws = static_cast<float*>(ws);
  hip_check(rms_norm_bwd(a, s), "rms_norm_bwd");
}

// ---------------------------------------------------------------- product ----
namespace {

ProductArgs product_args(const spectrain_product_desc* desc) {
  if (!desc) fail("desc is NULL");
  const spectrain_product_desc& d = *desc;
  check_version(d.abi_version);
  check_dtype(d.out_dtype, "out_dtype");
  check_dtype(d.bias_dtype, "bias_dtype");
  if ((d.relu != 0 && d.relu != 1) || (d.accumulate != 0 && d.accumulate != 1)) fail("relu and accumulate must be 0 or 1");
  if (d.accumulate && d.out_dtype != SPECTRAIN_FP32) fail("accumulate needs a float32 out");
  if (d.reserved != 0) fail("reserved must be 0");
  if (d.m < 0 || d.n < 0 || d.k < 0) fail("m, n and k must be >= 0");
  if (d.m >= int64_t{1} << 31 || d.n >= int64_t{1} << 31 || d.k > MAX_CODES_LD)
    fail("m and n must be below 2^31 and k at most 2^22");
  if (ceil_div(d.m, 64) * ceil_div(d.n, 64) > 1 << 22) fail("ceil(m / 64) * ceil(n / 64) must be at most 2^22");
  ProductArgs a;
  a.m = d.m;
  a.n = d.n;
  a.k = d.k;
  a.out_dtype = d.out_dtype;
  a.bias_dtype = d.bias_dtype;
  a.relu = d.relu;
  a.accumulate = d.accumulate;
  return a;
}

}  // namespace

size_t product_workspace(const spectrain_product_desc* desc) {
  const ProductArgs a = product_args(desc);
  return product_ws_bytes(a.m, a.n, a.k);
}

void run_product(const spectrain_product_desc* desc, const uint8_t* a_codes, const uint8_t* a_scales,
                 const uint8_t* b_codes, const uint8_t* b_scales, const void* bias, const void* mask, void* out,
                 void* ws, size_t ws_bytes, hipStream_t s) {
  ProductArgs a = product_args(desc);
  const spectrain_product_desc& d = *desc;
  check_workspace(ws, ws_bytes, product_ws_bytes(a.m, a.n, a.k));
  check_blocks(a_codes, a_scales, a.m, a.k, d.a_ld, d.a_scales_ld, "a");
  check_blocks(b_codes, b_scales, a.n, a.k, d.b_ld, d.b_scales_ld, "b");
  const int64_t blocks = ceil_div(a.k, 128);
  if (blocks && std::max(d.a_scales_ld, d.b_scales_ld) > ((int64_t{1} << 31) - 1) / blocks)
    fail("scales_ld * ceil(k / 128) must be below 2^31");
  a.out_ld = given_ld(out, d.out_ld, a.n, d.out_dtype, "out");
  a.mask_ld = given_ld(mask, d.mask_ld, a.n, d.out_dtype, "mask");
  check_elements(bias, d.bias_dtype, "bias");
  if (a.m == 0 || a.n == 0) return;
  if (!out || (a.k && (!a_codes || !b_codes))) fail("a tensor is NULL");
  for (const void* p : {static_cast<const void*>(a_codes), static_cast<const void*>(a_scales),
                        static_cast<const void*>(b_codes), static_cast<const void*>(b_scales), bias, mask})
    if (out == p) fail("out must not be an input");
  a.a = a_codes;
  a.a_scales = a_scales;
  a.b = b_codes;
  a.b_scales = b_scales;
  a.a_ld = d.a_ld;
  a.a_scales_ld = d.a_scales_ld;
  a.b_ld = d.b_ld;
  a.b_scales_ld = d.b_scales_ld;
  a.bias = bias;
  a.mask = mask;
  a.out = out;
  a.ws = static_cast<float*>(ws);
  hip_check(product(a, s), "product");
}

}  // namespace spx
