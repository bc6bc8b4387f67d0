// C ABI of the operators around a block in a training or serving step (declared in
// include/jarq.h): argument checks and dispatch to the kernels' launchers.
#include <algorithm>
#include <cmath>
#include <initializer_list>
#include <vector>

#include "jarq.h"
#include "jarq_internal.h"

using namespace jarq;

namespace {

constexpr int64_t kMaxTokens = 1 << 22;
constexpr int32_t kMaxChannels = 1 << 20;

bool aligned(const void* ptr, size_t a) { return ptr != nullptr && ((uintptr_t)ptr % a) == 0; }
bool aligned_or_null(const void* ptr, size_t a) { return ptr == nullptr || aligned(ptr, a); }

bool is_dtype(int32_t dtype) { return dtype >= JARQ_F32 && dtype <= JARQ_BF16; }
bool is_16bit(int32_t dtype) { return dtype == JARQ_F16 || dtype == JARQ_BF16; }
size_t bytes_of(int32_t dtype) { return dtype == JARQ_F32 ? 4 : 2; }

bool valid_norm_size(int64_t tokens, int32_t cols) {
  return tokens >= 0 && tokens <= kMaxTokens && cols >= 1 && cols <= kMaxChannels;
}
bool valid_norm(int32_t dtype, int32_t gain_dtype, int64_t tokens, int32_t cols, const void* gain,
                float eps) {
  return is_dtype(dtype) && (gain_dtype == dtype || gain_dtype == JARQ_F32) &&
         valid_norm_size(tokens, cols) && aligned(gain, bytes_of(gain_dtype)) &&
         eps >= 0x1p-126f && std::isfinite(eps);
}
// X, and the residual and H both or neither
bool valid_rows(int32_t dtype, const void* X, const void* residual, const void* H) {
  const size_t a = bytes_of(dtype);
  return aligned(X, a) && (residual == nullptr) == (H == nullptr) && aligned_or_null(residual, a) &&
         aligned_or_null(H, a);
}

bool valid_linlog(int64_t tokens, int32_t d, int32_t vocab) {
  return tokens >= 0 && tokens <= kMaxTokens && d >= 8 && d <= kMaxChannels && d % 8 == 0 &&
         vocab >= 1 && vocab <= (1 << 22);
}

jarq_status check(const void* ws, size_t bytes, size_t need) {
  return ws == nullptr || (uintptr_t)ws % 256 != 0 || bytes < need ? JARQ_EWORKSPACE : JARQ_OK;
}
jarq_status status_of(hipError_t e) { return e == hipSuccess ? JARQ_OK : JARQ_EHIP; }

size_t pad256(size_t n) { return (n + 255) & ~(size_t)255; }

// An array in memory.
struct Span {
  uintptr_t from, to;
};
Span span(const void* p, size_t bytes) { return Span{(uintptr_t)p, (uintptr_t)p + bytes}; }
bool before(const Span& a, const Span& b) { return a.from < b.from; }
// Sorts; whether none overlaps another.
bool apart(std::vector<Span>& s) {
  if (!std::is_sorted(s.begin(), s.end(), before)) std::sort(s.begin(), s.end(), before);
  for (size_t k = 1; k < s.size(); ++k)
    if (s[k].from < s[k - 1].to) return false;
  return true;
}
// Whether r overlaps one of the sorted, disjoint spans.
bool meets(const std::vector<Span>& s, const Span& r) {
  const auto at = std::upper_bound(s.begin(), s.end(), r, before);
  return (at != s.end() && at->from < r.to) || (at != s.begin() && (at - 1)->to > r.from);
}

// Whether two arrays share bytes (an empty one and a null pointer share none).
bool overlap(const Span& a, const Span& b) {
  return a.from != 0 && b.from != 0 && std::max(a.from, b.from) < std::min(a.to, b.to);
}
// Whether what is written lies where it may: over one of `over` as a whole or apart from it (row by
// row the same), and apart from `others`.
bool fits(const Span& out, std::initializer_list<Span> over, std::initializer_list<Span> others) {
  for (const Span& s : over)
    if (s.from != out.from && overlap(out, s)) return false;
  for (const Span& s : others)
    if (overlap(out, s)) return false;
  return true;
}

}  // namespace

extern "C" {

jarq_status jarq_rms_norm(int32_t dtype, int32_t gain_dtype, int64_t tokens, int32_t cols,
                          const void* X, const void* residual, const void* gain, float eps,
                          void* H, void* Y, void* stream) {
  if (!valid_norm(dtype, gain_dtype, tokens, cols, gain, eps)) return JARQ_EINVAL;
  if (tokens == 0) return JARQ_OK;
  if (!valid_rows(dtype, X, residual, H) || !aligned(Y, bytes_of(dtype))) return JARQ_EINVAL;
  // (a row is read before it is written)
  const size_t rows = bytes_of(dtype) * (size_t)tokens * cols;
  const Span x = span(X, rows), r = span(residual, rows), h = span(H, rows), y = span(Y, rows);
  const Span g = span(gain, bytes_of(gain_dtype) * (size_t)cols);
  if (!fits(h, {x, r}, {g, y}) || !fits(y, {x, r}, {g})) return JARQ_EINVAL;
  return status_of(launch_rms_norm((hipStream_t)stream, dtype, gain_dtype, X, residual, gain, eps,
                                   (int)tokens, cols, H, Y));
}

jarq_status jarq_rms_norm_i8(int32_t dtype, int32_t gain_dtype, int64_t tokens, int32_t cols,
                             const void* X, const void* residual, const void* gain, float eps,
                             void* H, int8_t* Q, float* scale, void* stream) {
  if (!valid_norm(dtype, gain_dtype, tokens, cols, gain, eps) || cols % 16 != 0 || cols > 131056)
    return JARQ_EINVAL;
  if (tokens == 0) return JARQ_OK;
  if (!valid_rows(dtype, X, residual, H) || !aligned(Q, 16) || !aligned(scale, 4))
    return JARQ_EINVAL;
  const size_t rows = bytes_of(dtype) * (size_t)tokens * cols;
  const Span x = span(X, rows), r = span(residual, rows), h = span(H, rows);
  const Span q = span(Q, (size_t)tokens * cols), s = span(scale, 4 * (size_t)tokens);
  const Span g = span(gain, bytes_of(gain_dtype) * (size_t)cols);
  if (!fits(h, {x, r}, {g, q, s}) || !fits(q, {}, {x, r, g, s}) || !fits(s, {}, {x, r, g}))
    return JARQ_EINVAL;
  return status_of(launch_rms_norm_i8((hipStream_t)stream, dtype, gain_dtype, X, residual, gain,
                                      eps, (int)tokens, cols, H, Q, scale));
}

size_t jarq_rms_norm_workspace_bytes(int64_t tokens, int32_t cols) {
  return valid_norm_size(tokens, cols) ? pad256(rms_norm_workspace_bytes((int)tokens, cols)) : 0;
}

jarq_status jarq_rms_norm_backward(int32_t dtype, int32_t gain_dtype, int64_t tokens,
                                   int32_t cols, const void* H, const void* gain, const void* dY,
                                   const void* dH, float eps, void* dX, void* dgain,
                                   void* workspace, size_t workspace_bytes, void* stream) {
  if (!valid_norm(dtype, gain_dtype, tokens, cols, gain, eps) ||
      !aligned_or_null(dgain, bytes_of(gain_dtype)))
    return JARQ_EINVAL;
  const size_t a = bytes_of(dtype);
  if (tokens > 0 &&
      (!aligned(H, a) || !aligned(dY, a) || !aligned_or_null(dH, a) || !aligned_or_null(dX, a)))
    return JARQ_EINVAL;
  const jarq_status s =
      check(workspace, workspace_bytes, jarq_rms_norm_workspace_bytes(tokens, cols));
  if (s != JARQ_OK) return s;
  const size_t rows = a * (size_t)tokens * cols;
  const Span h = span(H, rows), y = span(dY, rows), d = span(dH, rows);
  const Span g = span(gain, bytes_of(gain_dtype) * (size_t)cols), x = span(dX, rows);
  const Span dg = span(dgain, bytes_of(gain_dtype) * (size_t)cols);
  const Span ws = span(workspace, jarq_rms_norm_workspace_bytes(tokens, cols));
  if (!fits(x, {y, d}, {h, g, dg, ws}) || !fits(dg, {}, {h, y, d, g, ws}) ||
      !fits(ws, {}, {h, y, d, g}))
    return JARQ_EINVAL;
  return status_of(launch_rms_norm_backward((hipStream_t)stream, dtype, gain_dtype, H, gain, dY,
                                            dH, eps, (int)tokens, cols, dX, dgain,
                                            (char*)workspace));
}

size_t jarq_linear_logprobs_workspace_bytes(int64_t tokens, int32_t d, int32_t vocab) {
  if (!valid_linlog(tokens, d, vocab)) return 0;
  return tokens == 0 ? 256 : pad256(linear_logprobs_workspace_bytes((int)tokens, d, vocab));
}

jarq_status jarq_linear_logprobs(int32_t dtype, int64_t tokens, int32_t d, int32_t vocab,
                                 const void* X, const void* W, const int64_t* targets,
                                 float* logprob, float* lse, float* lse_rest, void* workspace,
                                 size_t workspace_bytes, void* stream) {
  if (!is_16bit(dtype) || !valid_linlog(tokens, d, vocab) || !aligned(W, 16)) return JARQ_EINVAL;
  if (tokens == 0) return JARQ_OK;
  if (!aligned(X, 16) || !aligned(targets, 8) || !aligned(logprob, 4) || !aligned(lse, 4) ||
      !aligned(lse_rest, 4))
    return JARQ_EINVAL;
  const jarq_status s =
      check(workspace, workspace_bytes, jarq_linear_logprobs_workspace_bytes(tokens, d, vocab));
  if (s != JARQ_OK) return s;
  return status_of(launch_linear_logprobs((hipStream_t)stream, dtype, (int)tokens, d, vocab, X, W,
                                          targets, logprob, lse, lse_rest, (char*)workspace));
}

size_t jarq_linear_logprobs_backward_workspace_bytes(int64_t tokens, int32_t d, int32_t vocab) {
  if (!valid_linlog(tokens, d, vocab)) return 0;
  return tokens == 0 ? 256
                     : pad256(linear_logprobs_backward_workspace_bytes((int)tokens, d, vocab));
}

jarq_status jarq_linear_logprobs_backward(int32_t dtype, int64_t tokens, int32_t d, int32_t vocab,
                                          const void* X, const void* W, const int64_t* targets,
                                          const float* logprob, const float* lse,
                                          const float* lse_rest, const float* d_logprob,
                                          const float* d_lse, void* dX, void* dW,
                                          void* workspace, size_t workspace_bytes, void* stream) {
  if (!is_16bit(dtype) || !valid_linlog(tokens, d, vocab) || !aligned(W, 16) ||
      !aligned_or_null(dX, 16) || !aligned_or_null(dW, 16))
    return JARQ_EINVAL;
  if (tokens > 0 && (!aligned(X, 16) || !aligned(targets, 8) || !aligned(logprob, 4) ||
                     !aligned(lse, 4) || !aligned(lse_rest, 4) || !aligned(d_logprob, 4) ||
                     !aligned_or_null(d_lse, 4)))
    return JARQ_EINVAL;
  const jarq_status s = check(workspace, workspace_bytes,
                              jarq_linear_logprobs_backward_workspace_bytes(tokens, d, vocab));
  if (s != JARQ_OK) return s;
  return status_of(launch_linear_logprobs_backward((hipStream_t)stream, dtype, (int)tokens, d,
                                                   vocab, X, W, targets, logprob, lse, lse_rest,
                                                   d_logprob, d_lse, dX, dW, (char*)workspace));
}

int64_t jarq_adamw_state_length(int32_t count, const int64_t* numel) {
  if (count < 0 || (count > 0 && numel == nullptr)) return -1;
  int64_t n = 0;
  for (int32_t k = 0; k < count; ++k) {
    if (numel[k] < 0 || numel[k] > ((int64_t)1 << 40)) return -1;
    n += (numel[k] + 127) / 128 * 128;
    if (n > ((int64_t)1 << 44)) return -1;
  }
  return n;
}

jarq_status jarq_adamw_step(int32_t dtype, int32_t bits, int32_t count,
                            const jarq_adamw_tensor* tensors, const jarq_adamw_state* in,
                            const jarq_adamw_state* out, const jarq_adamw_options* options,
                            void* stream) try {
  if (!is_dtype(dtype) || (bits != 8 && bits != 32) || count < 0 ||
      (count > 0 && tensors == nullptr) || in == nullptr || out == nullptr || options == nullptr)
    return JARQ_EINVAL;
  const jarq_adamw_options& o = *options;
  if (!(o.lr >= 0.0) || !std::isfinite(o.lr) || !(o.beta1 >= 0.0 && o.beta1 < 1.0) ||
      !(o.beta2 >= 0.0 && o.beta2 < 1.0) || !((float)o.eps >= 0x1p-126f) ||
      !std::isfinite((float)o.eps) || !(o.weight_decay >= 0.0) || !std::isfinite(o.weight_decay) ||
      o.step < 1 || !aligned_or_null(o.lr_at, 4) || !aligned_or_null(o.step_at, 8) ||
      !aligned_or_null(o.grad_mul, 4))
    return JARQ_EINVAL;
  const size_t e = bytes_of(dtype);
  const bool same = in->m == out->m;
  int64_t n = 0;
  for (int32_t k = 0; k < count; ++k) {
    const jarq_adamw_tensor& t = tensors[k];
    if (t.numel < 0 || t.numel > ((int64_t)1 << 40)) return JARQ_EINVAL;
    if (t.numel == 0) continue;
    n += (t.numel + 127) / 128 * 128;
    if (n > ((int64_t)1 << 44) || !aligned_or_null(t.grad, e) || !aligned(t.param, e) ||
        !aligned(t.param_out, e) || (t.param == t.param_out) != same ||
        (t.grad == nullptr && !same))
      return JARQ_EINVAL;
  }
  if (n == 0) return JARQ_OK;
  // the state's arrays: master, m, v, and their blocks' exponents
  const size_t each[5] = {dtype == JARQ_F32 ? 0 : 4 * (size_t)n, (size_t)n * (bits / 8),
                          (size_t)n * (bits / 8), bits == 8 ? (size_t)n / 128 : 0,
                          bits == 8 ? (size_t)n / 128 : 0};
  const void* const read[5] = {in->master, in->m, in->v, in->m_exp, in->v_exp};
  const void* const written[5] = {out->master, out->m, out->v, out->m_exp, out->v_exp};
  std::vector<Span> to;
  to.reserve((size_t)count + 5);
  for (int32_t k = 0; k < count; ++k)
    if (tensors[k].numel > 0) to.push_back(span(tensors[k].param_out, e * (size_t)tensors[k].numel));
  for (int k = 0; k < 5; ++k) {
    if (each[k] == 0) continue;
    const size_t a = k < 3 ? 16 : 1;
    if (!aligned(read[k], a) || !aligned(written[k], a) || (read[k] == written[k]) != same)
      return JARQ_EINVAL;
    to.push_back(span(written[k], each[k]));
  }
  if (!apart(to)) return JARQ_EINVAL;
  for (int32_t k = 0; k < count; ++k) {
    const size_t bytes = e * (size_t)tensors[k].numel;
    if (bytes == 0) continue;
    if ((tensors[k].grad && meets(to, span(tensors[k].grad, bytes))) ||
        (!same && meets(to, span(tensors[k].param, bytes))))
      return JARQ_EINVAL;
  }
  for (int k = 0; k < 5; ++k)
    if (!same && each[k] != 0 && meets(to, span(read[k], each[k]))) return JARQ_EINVAL;
  for (const Span& s : {span(o.lr_at, 4), span(o.step_at, 8), span(o.grad_mul, 4)})
    if (s.from != 0 && meets(to, s)) return JARQ_EINVAL;
  return status_of(launch_adamw((hipStream_t)stream, dtype, bits, count, tensors, *in, *out, o));
} catch (...) {
  return JARQ_EHIP;   // (no host memory)
}

}  // extern "C"
