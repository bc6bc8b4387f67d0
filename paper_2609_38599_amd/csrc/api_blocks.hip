// C ABI of the operators that run, train and evaluate refined layers (declared in
// include/jarq.h): argument checks and dispatch to the kernels' launchers.
#include "jarq.h"
#include "jarq_internal.h"

using namespace jarq;

namespace {

constexpr int64_t kMaxTokens = 1 << 22;
constexpr int32_t kMaxChannels = 1 << 20;

bool aligned(const void* ptr, size_t a) { return ptr != nullptr && ((uintptr_t)ptr % a) == 0; }

bool is_dtype(int32_t dtype) { return dtype >= JARQ_F32 && dtype <= JARQ_BF16; }
bool is_16bit(int32_t dtype) { return dtype == JARQ_F16 || dtype == JARQ_BF16; }
size_t bytes_of(int32_t dtype) { return dtype == JARQ_F32 ? 4 : 2; }

bool valid_gated(int32_t dtype, int32_t act, int64_t tokens, int32_t d, int32_t f) {
  return is_16bit(dtype) && act >= JARQ_ACT_SILU && act <= JARQ_ACT_GELU_TANH && tokens >= 0 &&
         tokens <= kMaxTokens && d >= 8 && d <= kMaxChannels && d % 8 == 0 && f >= 8 &&
         f <= kMaxChannels && f % 8 == 0;
}

bool valid_i8(int64_t tokens, int32_t n, int32_t k, int32_t group) {
  if (tokens < 0 || tokens > kMaxTokens || n < 1 || n > (1 << 22) || k < 16 || k > 131056 ||
      k % 16 != 0)
    return false;
  return group == 0 || ((group == 32 || group == 64 || group == 128) && k % group == 0);
}

bool valid_logits(int32_t dtype, const void* logits, int64_t ld, int64_t tokens, int32_t vocab) {
  return is_dtype(dtype) && tokens >= 0 && tokens <= kMaxTokens && vocab >= 1 &&
         vocab <= (1 << 30) && ld >= vocab && ld <= ((int64_t)1 << 31) &&
         (tokens == 0 || aligned(logits, bytes_of(dtype)));
}

jarq_status check(const void* ws, size_t bytes, size_t need) {
  return ws == nullptr || (uintptr_t)ws % 256 != 0 || bytes < need ? JARQ_EWORKSPACE : JARQ_OK;
}
jarq_status status_of(hipError_t e) { return e == hipSuccess ? JARQ_OK : JARQ_EHIP; }

size_t pad256(size_t n) { return (n + 255) & ~(size_t)255; }

}  // namespace

extern "C" {

jarq_status jarq_gated_forward(int32_t dtype, int32_t act, int64_t tokens, int32_t d, int32_t f,
                               const void* X, const void* Wg, const void* Wu, void* Y, float* pre,
                               void* stream) {
  if (!valid_gated(dtype, act, tokens, d, f) || !aligned(Wg, 16) || !aligned(Wu, 16))
    return JARQ_EINVAL;
  if (tokens == 0) return JARQ_OK;
  if (!aligned(X, 16) || !aligned(Y, 16) || (pre != nullptr && !aligned(pre, 16)))
    return JARQ_EINVAL;
  return status_of(launch_gated_forward((hipStream_t)stream, dtype, act, (int)tokens, d, f, X, Wg,
                                        Wu, Y, pre));
}

size_t jarq_gated_workspace_bytes(int64_t tokens, int32_t d, int32_t f) {
  if (!valid_gated(JARQ_BF16, JARQ_ACT_SILU, tokens, d, f)) return 0;
  return tokens == 0 ? 256 : gated_workspace_bytes((int)tokens, d, f);
}

jarq_status jarq_gated_backward(int32_t dtype, int32_t act, int64_t tokens, int32_t d, int32_t f,
                                const void* X, const void* Wg, const void* Wu, const void* dY,
                                const float* pre, void* dX, void* dWg, void* dWu, void* workspace,
                                size_t workspace_bytes, void* stream) {
  if (!valid_gated(dtype, act, tokens, d, f) || !aligned(Wg, 16) || !aligned(Wu, 16) ||
      (dX != nullptr && !aligned(dX, 16)) || (dWg != nullptr && !aligned(dWg, 16)) ||
      (dWu != nullptr && !aligned(dWu, 16)))
    return JARQ_EINVAL;
  if (tokens > 0 && (!aligned(X, 16) || !aligned(dY, 16) || !aligned(pre, 16))) return JARQ_EINVAL;
  const jarq_status s =
      check(workspace, workspace_bytes, jarq_gated_workspace_bytes(tokens, d, f));
  if (s != JARQ_OK) return s;
  return status_of(launch_gated_backward((hipStream_t)stream, dtype, act, (int)tokens, d, f, X, Wg,
                                         Wu, dY, pre, dX, dWg, dWu, (char*)workspace));
}

jarq_status jarq_quant_rows_i8(int32_t dtype, const void* X, int64_t rows, int32_t cols, int8_t* Q,
                               float* scale, void* stream) {
  if (!is_dtype(dtype) || !valid_i8(rows, 1, cols, 0)) return JARQ_EINVAL;
  if (rows == 0) return JARQ_OK;
  if (!aligned(X, 16) || !aligned(Q, 16) || !aligned(scale, 4)) return JARQ_EINVAL;
  return status_of(launch_quant_rows((hipStream_t)stream, dtype, X, (int)rows, cols, Q, scale));
}

jarq_status jarq_codes_i8(const jarq_params* p, const uint8_t* codes, const int32_t* zeros,
                          int8_t* out, int32_t* flag, void* stream) {
  if (jarq_workspace_bytes(p) == 0 || !aligned(codes, 16) || !aligned(zeros, 4) ||
      !aligned(out, 16) || !aligned(flag, 4))
    return JARQ_EINVAL;
  hipStream_t st = (hipStream_t)stream;
  int32_t bad = 0;
  if (launch_codes_i8(st, codes, zeros, p->rows, p->cols, p->group_size, out, flag) !=
          hipSuccess ||
      hipMemcpyAsync(&bad, flag, sizeof(bad), hipMemcpyDeviceToHost, st) != hipSuccess ||
      hipStreamSynchronize(st) != hipSuccess)
    return JARQ_EHIP;
  return bad ? JARQ_EINVAL : JARQ_OK;
}

jarq_status jarq_matmul_i8(int32_t dtype, int64_t tokens, int32_t n, int32_t k, int32_t group,
                           const int8_t* Xq, const float* sx, const int8_t* Wq, const float* sw,
                           void* Y, void* stream) {
  if (!is_dtype(dtype) || !valid_i8(tokens, n, k, group) || !aligned(Wq, 16) || !aligned(sw, 4))
    return JARQ_EINVAL;
  if (tokens == 0) return JARQ_OK;
  if (!aligned(Xq, 16) || !aligned(sx, 4) || !aligned(Y, bytes_of(dtype))) return JARQ_EINVAL;
  return status_of(launch_matmul_i8((hipStream_t)stream, dtype, (int)tokens, n, k, group, Xq, sx,
                                    Wq, sw, Y));
}

size_t jarq_linear_i8_workspace_bytes(int64_t tokens, int32_t k) {
  if (!valid_i8(tokens, 1, k, 0)) return 0;
  return pad256((size_t)tokens * k) + pad256(4 * (size_t)tokens) + 256;
}

jarq_status jarq_linear_i8(int32_t dtype, int64_t tokens, int32_t n, int32_t k, int32_t group,
                           const void* X, const int8_t* Wq, const float* sw, void* Y,
                           void* workspace, size_t workspace_bytes, void* stream) {
  if (!is_dtype(dtype) || !valid_i8(tokens, n, k, group) || !aligned(Wq, 16) || !aligned(sw, 4))
    return JARQ_EINVAL;
  if (tokens == 0) return JARQ_OK;
  if (!aligned(X, 16) || !aligned(Y, bytes_of(dtype))) return JARQ_EINVAL;
  const jarq_status s =
      check(workspace, workspace_bytes, jarq_linear_i8_workspace_bytes(tokens, k));
  if (s != JARQ_OK) return s;
  hipStream_t st = (hipStream_t)stream;
  int8_t* q = (int8_t*)workspace;
  float* sx = (float*)((char*)workspace + pad256((size_t)tokens * k));
  return status_of(
      launch_linear_i8(st, dtype, (int)tokens, n, k, group, X, Wq, sw, Y, q, sx));
}

size_t jarq_token_logprobs_workspace_bytes(int64_t tokens, int32_t vocab, int32_t top) {
  if (tokens < 0 || tokens > kMaxTokens || vocab < 1 || vocab > (1 << 30) || top < 0 ||
      top > JARQ_MAX_TOP || top > vocab)
    return 0;
  return tokens == 0 ? 256 : pad256(logprob_workspace_bytes((int)tokens, vocab, top) + 1);
}

jarq_status jarq_token_logprobs_keep(int32_t dtype, const void* logits, int64_t ld, int64_t tokens,
                                     int32_t vocab, const int64_t* targets, int32_t top,
                                     float* logprob, float* entropy, float* lse, float* lse_rest,
                                     int32_t* top_index, float* top_logprob, void* workspace,
                                     size_t workspace_bytes, void* stream) {
  if (!valid_logits(dtype, logits, ld, tokens, vocab) || top < 0 || top > JARQ_MAX_TOP ||
      top > vocab)
    return JARQ_EINVAL;
  if (tokens == 0) return JARQ_OK;
  if (!aligned(targets, 8) || !aligned(logprob, 4) || (entropy != nullptr && !aligned(entropy, 4)) ||
      (lse != nullptr && !aligned(lse, 4)) || (lse_rest != nullptr && !aligned(lse_rest, 4)) ||
      (top > 0 && (!aligned(top_index, 4) || !aligned(top_logprob, 4))))
    return JARQ_EINVAL;
  const jarq_status s = check(workspace, workspace_bytes,
                              jarq_token_logprobs_workspace_bytes(tokens, vocab, top));
  if (s != JARQ_OK) return s;
  return status_of(launch_token_logprobs((hipStream_t)stream, dtype, logits, (size_t)ld,
                                         (int)tokens, vocab, targets, top, logprob, entropy, lse,
                                         lse_rest, top_index, top_logprob, (char*)workspace));
}

jarq_status jarq_token_logprobs(int32_t dtype, const void* logits, int64_t ld, int64_t tokens,
                                int32_t vocab, const int64_t* targets, int32_t top, float* logprob,
                                float* entropy, float* lse, int32_t* top_index, float* top_logprob,
                                void* workspace, size_t workspace_bytes, void* stream) {
  return jarq_token_logprobs_keep(dtype, logits, ld, tokens, vocab, targets, top, logprob, entropy,
                                  lse, nullptr, top_index, top_logprob, workspace, workspace_bytes,
                                  stream);
}

static jarq_status logprobs_backward(int32_t dtype, const void* logits, int64_t ld, int64_t tokens,
                                     int32_t vocab, const int64_t* targets, const float* lse,
                                     const float* lse_rest, const float* entropy,
                                     const float* d_logprob, const float* d_entropy,
                                     void* d_logits, int64_t ld_d, void* stream) {
  if (!valid_logits(dtype, logits, ld, tokens, vocab) ||
      !valid_logits(dtype, d_logits, ld_d, tokens, vocab))
    return JARQ_EINVAL;
  if (tokens == 0) return JARQ_OK;
  if (!aligned(targets, 8) || !aligned(lse, 4) || !aligned(d_logprob, 4) ||
      (d_entropy != nullptr && (!aligned(d_entropy, 4) || !aligned(entropy, 4))))
    return JARQ_EINVAL;
  return status_of(launch_token_logprobs_backward(
      (hipStream_t)stream, dtype, logits, (size_t)ld, (int)tokens, vocab, targets, lse, lse_rest,
      entropy, d_logprob, d_entropy, d_logits, (size_t)ld_d));
}

jarq_status jarq_token_logprobs_backward(int32_t dtype, const void* logits, int64_t ld,
                                         int64_t tokens, int32_t vocab, const int64_t* targets,
                                         const float* lse, const float* entropy,
                                         const float* d_logprob, const float* d_entropy,
                                         void* d_logits, int64_t ld_d, void* stream) {
  return logprobs_backward(dtype, logits, ld, tokens, vocab, targets, lse, nullptr, entropy,
                           d_logprob, d_entropy, d_logits, ld_d, stream);
}

jarq_status jarq_token_logprobs_keep_backward(int32_t dtype, const void* logits, int64_t ld,
                                              int64_t tokens, int32_t vocab,
                                              const int64_t* targets, const float* lse,
                                              const float* lse_rest, const float* entropy,
                                              const float* d_logprob, const float* d_entropy,
                                              void* d_logits, int64_t ld_d, void* stream) {
  if (tokens > 0 && !aligned(lse_rest, 4)) return JARQ_EINVAL;
  return logprobs_backward(dtype, logits, ld, tokens, vocab, targets, lse, lse_rest, entropy,
                           d_logprob, d_entropy, d_logits, ld_d, stream);
}

}  // extern "C"
