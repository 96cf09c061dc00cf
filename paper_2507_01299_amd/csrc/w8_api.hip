// C ABI of the operators on 8-bit floating-point weights and of the log probabilities: argument checks, workspace carving, launches.
#include "../../include/larosa.h"

#include <hip/hip_runtime.h>

#include <cmath>

#include "kernels.hpp"
#include "w8.hpp"

using namespace larosa;

namespace {

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
inline hipStream_t stream_of(void* s) { return static_cast<hipStream_t>(s); }
inline int status_of(hipError_t e) { return e == hipSuccess ? LAROSA_OK : LAROSA_EHIP; }
inline bool type16(larosa_dtype t) { return t == LAROSA_F16 || t == LAROSA_BF16; }
inline size_t round_up(size_t v, size_t a) { return (v + a - 1) / a * a; }

int check_held(const void* codes, const void* scales) {
  return !codes || !scales || !aligned(codes, 16) || !aligned(scales, 4) ? LAROSA_EINVAL : LAROSA_OK;
}

int check_width(int d_in) {
  if (d_in < 8 || d_in % 8) return LAROSA_EINVAL;
  return d_in > kWidthMax8 ? LAROSA_EUNSUPPORTED : LAROSA_OK;
}

int check_rows(const void* x, int ld_x, int n_rows, int d, const void* rms) {
  if (!x || !aligned(x, 16) || !aligned(rms, 16) || n_rows < 1 || ld_x < d || ld_x % 8) return LAROSA_EINVAL;
  return n_rows > kRowsMax8 ? LAROSA_EUNSUPPORTED : LAROSA_OK;
}

// A product of n rows of x: the rows to 8 bits at `codes` and `scales`, unless the product takes them as they are, then the product.
int run_product(Product8Args a, const Product8Plan& plan, const void* x, int ld_x, const void* rms, float rms_eps, larosa_dtype t,
                uint8_t* codes, uint8_t* scales, hipStream_t s) {
  const uint16_t* const rows = static_cast<const uint16_t*>(x);
  if (rms_eps < 0.f && takes_rows16(plan, a.n_rows, a.d_in)) {
    a.x16 = rows;
    a.ld_x = ld_x;
    a.x_bf16 = t == LAROSA_BF16;
  } else {
    a.tiled = plan.kind != 0;
    if (hipError_t e = launch_quantize_rows8(rows, ld_x, a.n_rows, a.d_in, static_cast<const uint16_t*>(rms), rms_eps, codes, scales, a.tiled,
                                             t == LAROSA_BF16, s))
      return status_of(e);
  }
  return status_of(launch_product8(a, plan, s));
}

// Sizes of a product; d_out need not be a multiple of 8 here.
int check_product(int n_rows, int d_in, int d_out) {
  if (n_rows < 1 || d_out < 1) return LAROSA_EINVAL;
  if (int rc = check_width(d_in)) return rc;
  if (n_rows > kRowsMax8 || d_out > kOutMax8) return LAROSA_EUNSUPPORTED;
  return plans_product8(n_rows, d_out) ? LAROSA_OK : LAROSA_EUNSUPPORTED;
}

// Workspace: arrival counters, then the pieces in this order, each from a multiple of 256 bytes on.
struct Carver {
  size_t at = kCounterBytes;
  size_t take(size_t bytes) {
    const size_t here = at;
    at += round_up(bytes, 256);
    return here;
  }
};

// What the queries answer: the most that any number of rows up to n_rows asks for (fewer rows go in more parts or slices), so that a workspace for
// the largest batch serves the smaller ones.  A call itself looks at its own need only.
size_t partial_up_to(int n_rows, int d_in, int d_out) {
  size_t most = 0;
  for (int n = 64; n - 64 < n_rows && n <= kRowsOfParts8; n += 64) {
    const size_t here = plan_product8(n < n_rows ? n : n_rows, d_in, d_out).partial_floats;
    if (here > most) most = here;
  }
  return most;
}

struct RowsSpace { size_t codes, scales; };
RowsSpace take_rows(Carver& c, int n_rows, int d) {
  const size_t codes = c.take(tiled_bytes8(n_rows, d));
  return {codes, c.take(static_cast<size_t>(n_rows) * scale_pitch8(d))};
}

int check_logprobs(int n_rows, int n_vocab, float scale, const void* given, int n_given, const void* logp, const void* entropy,
                   int n_top, const void* top_id, const void* top_logp) {
  if (n_rows < 1 || n_vocab < 1 || n_given < 0 || n_top < 0 || n_top > n_vocab) return LAROSA_EINVAL;
  if (!(scale > 0.f) || !std::isfinite(scale)) return LAROSA_EINVAL;
  if (n_given > 0 && (!given || !logp)) return LAROSA_EINVAL;
  if (n_top > 0 && !top_id) return LAROSA_EINVAL;
  if (!aligned(given, 4) || !aligned(logp, 4) || !aligned(entropy, 4) || !aligned(top_id, 4) || !aligned(top_logp, 4)) return LAROSA_EINVAL;
  if (n_rows > kRowsMax8 || n_vocab > kVocabMax || n_top > kTopMax || scale > kLogitScaleMax) return LAROSA_EUNSUPPORTED;
  return LAROSA_OK;
}

// Rows that one launch of the log probabilities takes: a counter word and a place in the workspace for each, and fewer than 2^24 workgroups.
int rows_at_once(const LogprobsPlan& p) {
  const size_t per_row = p.sums_bytes + p.best_bytes;
  long n = kCounterWords;
  if (per_row && static_cast<long>((size_t{128} << 20) / per_row) < n) n = static_cast<long>((size_t{128} << 20) / per_row);
  if (((1L << 24) - 1) / p.slices < n) n = ((1L << 24) - 1) / p.slices;
  return n > 1 ? static_cast<int>(n) : 1;
}

size_t logprobs_space(const LogprobsPlan& p, int n_rows) {
  const int n = rows_at_once(p) < n_rows ? rows_at_once(p) : n_rows;
  return round_up(p.sums_bytes * n, 256) + round_up(p.best_bytes * n, 256);
}

size_t logprobs_space_up_to(int n_rows, int n_vocab, int n_top) {
  size_t most = logprobs_space(plan_logprobs(n_rows, n_vocab, n_top), n_rows);
  for (int n = 1; n < n_rows && n <= kWorkgroupsOfFew; ++n) {
    const size_t here = logprobs_space(plan_logprobs(n, n_vocab, n_top), n);
    if (here > most) most = here;
  }
  return most;
}

int run_logprobs(LogprobsArgs a, int n_rows, int type, const LogprobsPlan& p, unsigned* counters, char* space, hipStream_t s) {
  const int at_once = rows_at_once(p) < n_rows ? rows_at_once(p) : n_rows;
  const int size = type == kLogitsF32 ? 4 : 2;
  a.slices = p.slices;
  a.slice_len = p.slice_len;
  a.counters = counters;
  a.sums = reinterpret_cast<float*>(space);
  a.best = reinterpret_cast<unsigned long long*>(space + round_up(p.sums_bytes * at_once, 256));
  for (int row = 0; row < n_rows; row += at_once) {
    LogprobsArgs b = a;
    b.n_rows = n_rows - row < at_once ? n_rows - row : at_once;
    b.logits = static_cast<const char*>(a.logits) + row * a.ld * size;
    if (a.n_given) {
      b.given = a.given + static_cast<size_t>(row) * a.n_given;
      b.logp = a.logp + static_cast<size_t>(row) * a.n_given;
    }
    if (a.entropy) b.entropy = a.entropy + row;
    if (a.n_top) b.top_id = a.top_id + static_cast<size_t>(row) * a.n_top;
    if (a.top_logp) b.top_logp = a.top_logp + static_cast<size_t>(row) * a.n_top;
    if (hipError_t e = launch_logprobs(b, type, s)) return status_of(e);
  }
  return LAROSA_OK;
}

// Rows whose logits lie in the workspace at once: 128 MiB, which stay in the memory-side cache; a multiple of 256 where there are as many, and 16
// of the largest vocabulary (kOutMax8).
int score_rows(int n_rows, int n_vocab) {
  const long ld = static_cast<long>(round_up(n_vocab, 16));
  long n = (128L << 20) / (ld * 4);
  if (n >= 256) n = n / 256 * 256;
  return n < n_rows ? static_cast<int>(n) : n_rows;
}

struct ScoreSpace { RowsSpace rows; size_t partial, logits, logprobs, end; int at_once; long ld; };
ScoreSpace score_space(int n_rows, int d_in, int n_vocab, int n_top, bool up_to = false) {
  ScoreSpace s{};
  Carver c;
  s.at_once = score_rows(n_rows, n_vocab);
  s.ld = static_cast<long>(round_up(n_vocab, 16));
  const int tail = n_rows % s.at_once;
  s.rows = take_rows(c, s.at_once, d_in);
  size_t partial, probs;
  if (up_to) {
    partial = partial_up_to(s.at_once, d_in, n_vocab);
    probs = logprobs_space_up_to(s.at_once, n_vocab, n_top);
  } else {
    partial = plan_product8(s.at_once, d_in, n_vocab).partial_floats;
    probs = logprobs_space(plan_logprobs(s.at_once, n_vocab, n_top), s.at_once);
    if (tail) {                                  // the last part may be divided otherwise
      const size_t p = plan_product8(tail, d_in, n_vocab).partial_floats;
      const size_t q = logprobs_space(plan_logprobs(tail, n_vocab, n_top), tail);
      if (p > partial) partial = p;
      if (q > probs) probs = q;
    }
  }
  s.partial = c.take(partial * sizeof(float));
  s.logits = c.take(static_cast<size_t>(s.at_once) * s.ld * sizeof(float));
  s.logprobs = c.take(probs);
  s.end = c.at;
  return s;
}

Product8Args product_args(const void* w_codes, const void* w_scales, const void* x_codes, const void* x_scales, void* y, long ld_y,
                          int n_rows, int d_in, int d_out, int out, void* ws, size_t partial) {
  Product8Args a{};
  a.w = {static_cast<const uint8_t*>(w_codes), static_cast<const uint8_t*>(w_scales)};
  a.x = {static_cast<const uint8_t*>(x_codes), static_cast<const uint8_t*>(x_scales)};
  a.y = y;
  a.ld_y = ld_y;
  a.n_rows = n_rows;
  a.d_in = d_in;
  a.d_out = d_out;
  a.out = out;
  a.counters = static_cast<unsigned*>(ws);
  a.partial = reinterpret_cast<float*>(static_cast<char*>(ws) + partial);
  return a;
}

}  // namespace

extern "C" {

int larosa_quantize_w8(const void* W, int d_in, int d_out, larosa_dtype t, void* codes, void* scales, void* stream) {
  if (!W || !aligned(W, 16) || !type16(t) || d_out < 8 || d_out % 8) return LAROSA_EINVAL;
  if (int rc = check_held(codes, scales)) return rc;
  if (int rc = check_width(d_in)) return rc;
  if (d_out > kOutMax8) return LAROSA_EUNSUPPORTED;
  return status_of(launch_quantize_w8(static_cast<const uint16_t*>(W), d_in, d_out, static_cast<uint8_t*>(codes),
                                      static_cast<uint8_t*>(scales), t == LAROSA_BF16, stream_of(stream)));
}

int larosa_quantize_rows8(const void* x, int ld_x, int n_rows, int d, const void* rms, float rms_eps, larosa_dtype t, void* codes,
                          void* scales, void* stream) {
  if (!type16(t) || std::isnan(rms_eps)) return LAROSA_EINVAL;
  if (int rc = check_held(codes, scales)) return rc;
  if (int rc = check_width(d)) return rc;
  if (int rc = check_rows(x, ld_x, n_rows, d, rms)) return rc;
  return status_of(launch_quantize_rows8(static_cast<const uint16_t*>(x), ld_x, n_rows, d, static_cast<const uint16_t*>(rms), rms_eps,
                                         static_cast<uint8_t*>(codes), static_cast<uint8_t*>(scales), false, t == LAROSA_BF16,
                                         stream_of(stream)));
}

size_t larosa_product8_workspace_bytes(int n_rows, int d_in, int d_out) {
  if (check_product(n_rows, d_in, d_out)) return 0;
  Carver c;
  c.take(partial_up_to(n_rows, d_in, d_out) * sizeof(float));
  return c.at;
}

int larosa_product8(const void* w_codes, const void* w_scales, const void* x_codes, const void* x_scales, void* y, int ld_y,
                    int n_rows, int d_in, int d_out, larosa_dtype t, void* ws, size_t ws_bytes, void* stream) {
  if (!type16(t) || !y || !aligned(y, 16) || d_out % 8 || ld_y < d_out || ld_y % 8) return LAROSA_EINVAL;
  if (int rc = check_held(w_codes, w_scales)) return rc;
  if (int rc = check_held(x_codes, x_scales)) return rc;
  if (int rc = check_product(n_rows, d_in, d_out)) return rc;
  if (ld_y > kOutMax8) return LAROSA_EUNSUPPORTED;
  const Product8Plan plan = plan_product8(n_rows, d_in, d_out);
  Carver c;
  c.take(plan.partial_floats * sizeof(float));
  if (!ws || !aligned(ws, 256) || ws_bytes < c.at) return LAROSA_EWORKSPACE;
  const Product8Args a = product_args(w_codes, w_scales, x_codes, x_scales, y, ld_y, n_rows, d_in, d_out,
                                      t == LAROSA_BF16 ? kOutBF16 : kOutF16, ws, kCounterBytes);
  return status_of(launch_product8(a, plan, stream_of(stream)));
}

size_t larosa_dense_w8_workspace_bytes(int n_rows, int d_in, int d_out) {
  if (check_product(n_rows, d_in, d_out)) return 0;
  Carver c;
  take_rows(c, n_rows, d_in);
  c.take(partial_up_to(n_rows, d_in, d_out) * sizeof(float));
  return c.at;
}

int larosa_dense_w8(const void* w_codes, const void* w_scales, const void* x, int ld_x, const void* rms, float rms_eps, void* y,
                    int ld_y, int n_rows, int d_in, int d_out, larosa_dtype t, void* ws, size_t ws_bytes, void* stream) {
  if (!type16(t) || std::isnan(rms_eps) || !y || !aligned(y, 16) || d_out % 8 || ld_y < d_out || ld_y % 8) return LAROSA_EINVAL;
  if (int rc = check_held(w_codes, w_scales)) return rc;
  if (int rc = check_product(n_rows, d_in, d_out)) return rc;
  if (int rc = check_rows(x, ld_x, n_rows, d_in, rms)) return rc;
  if (ld_y > kOutMax8) return LAROSA_EUNSUPPORTED;
  const Product8Plan plan = plan_product8(n_rows, d_in, d_out);
  Carver c;
  const RowsSpace r = take_rows(c, n_rows, d_in);
  const size_t partial = c.take(plan.partial_floats * sizeof(float));
  if (!ws || !aligned(ws, 256) || ws_bytes < c.at) return LAROSA_EWORKSPACE;
  char* const w = static_cast<char*>(ws);
  const Product8Args a = product_args(w_codes, w_scales, w + r.codes, w + r.scales, y, ld_y, n_rows, d_in, d_out,
                                      t == LAROSA_BF16 ? kOutBF16 : kOutF16, ws, partial);
  return run_product(a, plan, x, ld_x, rms, rms_eps, t, reinterpret_cast<uint8_t*>(w + r.codes), reinterpret_cast<uint8_t*>(w + r.scales),
                     stream_of(stream));
}

size_t larosa_logprobs_workspace_bytes(int n_rows, int n_vocab, int n_top, larosa_dtype t) {
  if (!type16(t) && t != LAROSA_F32) return 0;
  if (check_logprobs(n_rows, n_vocab, 1.f, nullptr, 0, nullptr, nullptr, 0, nullptr, nullptr)) return 0;
  if (n_top < 0 || n_top > kTopMax || n_top > n_vocab) return 0;
  return kCounterBytes + logprobs_space_up_to(n_rows, n_vocab, n_top);
}

int larosa_logprobs(const void* logits, int ld, int n_rows, int n_vocab, larosa_dtype t, float scale, const int32_t* given,
                    int n_given, float* logp, float* entropy, int n_top, int32_t* top_id, float* top_logp, void* ws,
                    size_t ws_bytes, void* stream) {
  if ((!type16(t) && t != LAROSA_F32) || !logits || !aligned(logits, t == LAROSA_F32 ? 4 : 2) || ld < n_vocab) return LAROSA_EINVAL;
  if (int rc = check_logprobs(n_rows, n_vocab, scale, given, n_given, logp, entropy, n_top, top_id, top_logp)) return rc;
  const LogprobsPlan plan = plan_logprobs(n_rows, n_vocab, n_top);
  if (!ws || !aligned(ws, 256) || ws_bytes < kCounterBytes + logprobs_space(plan, n_rows)) return LAROSA_EWORKSPACE;
  LogprobsArgs a{};
  a.logits = logits;
  a.ld = ld;
  a.n_vocab = n_vocab;
  a.scale = scale;
  a.given = given; a.n_given = n_given; a.logp = logp;
  a.entropy = entropy;
  a.n_top = n_top; a.top_id = top_id; a.top_logp = top_logp;
  return run_logprobs(a, n_rows, t, plan, static_cast<unsigned*>(ws), static_cast<char*>(ws) + kCounterBytes, stream_of(stream));
}

size_t larosa_score_w8_workspace_bytes(int n_rows, int d_in, int n_vocab, int n_top) {
  if (check_product(n_rows, d_in, n_vocab) || n_top < 0 || n_top > kTopMax || n_top > n_vocab) return 0;
  return score_space(n_rows, d_in, n_vocab, n_top, true).end;
}

int larosa_score_w8(const void* w_codes, const void* w_scales, const void* x, int ld_x, const void* rms, float rms_eps, int n_rows,
                    int d_in, int n_vocab, larosa_dtype t, float scale, const int32_t* given, int n_given, float* logp,
                    float* entropy, int n_top, int32_t* top_id, float* top_logp, void* ws, size_t ws_bytes, void* stream) {
  if (!type16(t) || std::isnan(rms_eps)) return LAROSA_EINVAL;
  if (int rc = check_held(w_codes, w_scales)) return rc;
  if (int rc = check_product(n_rows, d_in, n_vocab)) return rc;
  if (int rc = check_rows(x, ld_x, n_rows, d_in, rms)) return rc;
  if (int rc = check_logprobs(n_rows, n_vocab, scale, given, n_given, logp, entropy, n_top, top_id, top_logp)) return rc;
  const ScoreSpace sp = score_space(n_rows, d_in, n_vocab, n_top);
  if (!ws || !aligned(ws, 256) || ws_bytes < sp.end) return LAROSA_EWORKSPACE;
  char* const w = static_cast<char*>(ws);
  const hipStream_t s = stream_of(stream);
  uint8_t* const codes = reinterpret_cast<uint8_t*>(w + sp.rows.codes);
  uint8_t* const scales = reinterpret_cast<uint8_t*>(w + sp.rows.scales);
  for (int row = 0; row < n_rows; row += sp.at_once) {
    const int n = n_rows - row < sp.at_once ? n_rows - row : sp.at_once;
    const Product8Args a = product_args(w_codes, w_scales, codes, scales, w + sp.logits, sp.ld, n, d_in, n_vocab, kOutF32, ws, sp.partial);
    if (int rc = run_product(a, plan_product8(n, d_in, n_vocab), static_cast<const uint16_t*>(x) + static_cast<long>(row) * ld_x, ld_x, rms, rms_eps, t, codes, scales, s)) return rc;
    LogprobsArgs b{};
    b.logits = w + sp.logits;
    b.ld = sp.ld;
    b.n_vocab = n_vocab;
    b.scale = scale;
    b.n_given = n_given;
    if (n_given) {
      b.given = given + static_cast<size_t>(row) * n_given;
      b.logp = logp + static_cast<size_t>(row) * n_given;
    }
    b.entropy = entropy ? entropy + row : nullptr;
    b.n_top = n_top;
    if (n_top) b.top_id = top_id + static_cast<size_t>(row) * n_top;
    if (n_top && top_logp) b.top_logp = top_logp + static_cast<size_t>(row) * n_top;
    if (int rc = run_logprobs(b, n, kLogitsF32, plan_logprobs(n, n_vocab, n_top), static_cast<unsigned*>(ws),
                              w + sp.logprobs, s))
      return rc;
  }
  return LAROSA_OK;
}

}  // extern "C"
