// C ABI of the vocabulary head: argument checks of its products, the distillation loss and the token log probabilities.

#include <hip/hip_runtime.h>

#include <cmath>
#include <exception>
#include <string>

#include "common.h"
#include "internal.h"

using namespace fold;

namespace {

int vfail(int code, const std::string& msg) {
  set_error(msg);
  return code;
}

// runs an entry point's body; nothing it throws leaves the library
template <class F>
int32_t guarded(F&& body) {
  try {
    clear_error();
    return body();
  } catch (const std::exception& e) {
    return vfail(FOLD_E_INVALID, std::string("internal error: ") + e.what());
  } catch (...) {
    return vfail(FOLD_E_INVALID, "internal error");
  }
}

constexpr int kMaxVocab = 1 << 30;      // columns and their keys are counted in 31 bits
constexpr int kMaxHeadVocab = 1 << 21;  // a tile of a product is addressed by 32-bit offsets (256 lines of the logits)
constexpr int64_t kMaxTiles = (1 << 24) - 8;  // workgroups of one launch, rounded up to 8: its threads fit 32 bits

bool known_type(int dtype) { return dtype == FOLD_F32 || dtype == FOLD_BF16; }
bool misaligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) != 0; }
size_t bytes_of(int dtype, int64_t rows, int width) {
  return (size_t)rows * (size_t)row_ld(width) * (dtype == FOLD_BF16 ? 2 : 4);
}

// whether an output shares memory with another buffer (NULL: no)
struct Span {
  const void* p;
  size_t bytes;
};
bool overlap(const Span& a, const Span& b) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
  return x && y && a.bytes && b.bytes && x < y + b.bytes && y < x + a.bytes;
}

int check_rows(const std::string& who, int dtype, int64_t rows, int vocab) {
  if (!known_type(dtype)) return vfail(FOLD_E_INVALID, who + ": unknown dtype");
  if (rows < 0 || rows > INT32_MAX) return vfail(FOLD_E_INVALID, who + ": rows out of range");
  if (vocab < 1 || vocab > kMaxVocab) return vfail(FOLD_E_INVALID, who + ": vocabulary size out of range (1 .. 2^30)");
  return FOLD_OK;
}

// tiles: workgroups of the call's largest launch
template <class F>
int check_product(const std::string& who, int dtype, int64_t rows, int hidden, int vocab, F&& tiles) {
  const int rc = check_rows(who, dtype, rows, vocab);
  if (rc != FOLD_OK) return rc;
  if (vocab > kMaxHeadVocab) return vfail(FOLD_E_INVALID, who + ": vocabulary size out of range (1 .. 2^21)");
  if (hidden < 1 || hidden > kMaxHidden) return vfail(FOLD_E_INVALID, who + ": hidden size out of range");
  if (vocab_tiles(rows, hidden, vocab) >= kMaxTiles && tiles(dtype, rows, hidden, vocab) >= kMaxTiles)
    return vfail(FOLD_E_INVALID, who + ": too many tiles for one launch (rows times the widths)");
  return FOLD_OK;
}

// rows in pool order against a schedule: its node order, or NULL
int check_order(const std::string& who, const fold_sched* sh, int64_t rows, const int** order) {
  *order = nullptr;
  if (!sh) return FOLD_OK;
  if (sh->s.N != rows) return vfail(FOLD_E_MISMATCH, who + ": rows differ from the schedule's nodes");
  int dev = -1;
  FOLD_HIP_CHECK(hipGetDevice(&dev));
  if (dev != sh->s.device) return vfail(FOLD_E_MISMATCH, who + ": the schedule belongs to another device");
  *order = sh->s.pos_node;
  return FOLD_OK;
}

int check_distill_sizes(const std::string& who, int dtype, int64_t rows, int vocab, int num_teacher) {
  const int rc = check_rows(who, dtype, rows, vocab);
  if (rc != FOLD_OK) return rc;
  if (num_teacher < 0 || num_teacher > kMaxTeacherTokens)
    return vfail(FOLD_E_INVALID, who + ": num_teacher must be 0 .. 256");
  return FOLD_OK;
}

int check_token_sizes(const std::string& who, int dtype, int64_t rows, int vocab, int top_k) {
  const int rc = check_rows(who, dtype, rows, vocab);
  if (rc != FOLD_OK) return rc;
  if (top_k < 0 || top_k > kMaxTopTokens) return vfail(FOLD_E_INVALID, who + ": top_k must be 0 .. 32");
  return FOLD_OK;
}

}  // namespace

extern "C" {

int32_t fold_vocab_logits(int32_t dtype, int64_t rows, int32_t hidden, int32_t vocab, const void* states,
                          const void* W, const float* bias, int32_t logits_dtype, void* logits, hipStream_t st) {
  return guarded([&]() -> int32_t {
    const std::string who("fold_vocab_logits");
    const int rc = check_product(who, dtype, rows, hidden, vocab, vocab_logits_tiles);
    if (rc != FOLD_OK) return rc;
    if (!known_type(logits_dtype) || (dtype == FOLD_F32 && logits_dtype != FOLD_F32))
      return vfail(FOLD_E_INVALID, who + ": logits are fp32, or bf16 for a bf16 head");
    if (rows == 0) return FOLD_OK;
    if (!states || !W || !logits) return vfail(FOLD_E_INVALID, who + ": NULL buffer");
    if (misaligned(states) || misaligned(W) || misaligned(logits))
      return vfail(FOLD_E_INVALID, who + ": states, W and logits must be 16-byte aligned");
    const Span out{logits, bytes_of(logits_dtype, rows, vocab)};
    if (overlap(out, {states, bytes_of(dtype, rows, hidden)}) || overlap(out, {W, bytes_of(dtype, vocab, hidden)}) ||
        overlap(out, {bias, (size_t)vocab * sizeof(float)}))
      return vfail(FOLD_E_INVALID, who + ": logits overlaps an input");
    launch_vocab_logits(dtype, rows, hidden, vocab, states, W, bias, logits_dtype, logits, st);
    FOLD_HIP_CHECK(hipGetLastError());
    return FOLD_OK;
  });
}

int32_t fold_vocab_workspace_size(int32_t dtype, int64_t rows, int32_t hidden, int32_t vocab, size_t* bytes) {
  return guarded([&]() -> int32_t {
    const std::string who("fold_vocab_workspace_size");
    if (!bytes) return vfail(FOLD_E_INVALID, who + ": NULL argument");
    const int rc = check_product(who, dtype, rows, hidden, vocab, vocab_backward_tiles);
    if (rc != FOLD_OK) return rc;
    *bytes = vocab_backward_bytes(dtype, rows, hidden, vocab);
    return FOLD_OK;
  });
}

int32_t fold_vocab_backward(int32_t dtype, int64_t rows, int32_t hidden, int32_t vocab, const void* states,
                            const void* W, const void* dlogits, float* d_states, float* dW, float* dbias,
                            int32_t flags, void* ws, size_t ws_bytes, hipStream_t st) {
  return guarded([&]() -> int32_t {
    const std::string who("fold_vocab_backward");
    const int rc = check_product(who, dtype, rows, hidden, vocab, vocab_backward_tiles);
    if (rc != FOLD_OK) return rc;
    if (flags & ~FOLD_VOCAB_ACCUMULATE) return vfail(FOLD_E_INVALID, who + ": unknown flag");
    if ((!d_states || rows == 0) && !dW && !dbias) return FOLD_OK;
    if (rows > 0 && (!dlogits || (dW && !states) || (d_states && !W)))
      return vfail(FOLD_E_INVALID, who + ": NULL buffer");
    if (misaligned(states) || misaligned(W) || misaligned(dlogits) || misaligned(d_states) || misaligned(dW) ||
        misaligned(ws))
      return vfail(FOLD_E_INVALID, who + ": buffers must be 16-byte aligned");
    const size_t need = vocab_backward_bytes(dtype, rows, hidden, vocab);
    if (need > 0 && (!ws || ws_bytes < need))
      return vfail(FOLD_E_MISMATCH, who + ": workspace smaller than fold_vocab_workspace_size");
    const Span all[] = {{d_states, bytes_of(FOLD_F32, rows, hidden)}, {dW, bytes_of(FOLD_F32, vocab, hidden)},
                        {dbias, (size_t)vocab * sizeof(float)},       {ws, need},
                        {states, bytes_of(dtype, rows, hidden)},      {W, bytes_of(dtype, vocab, hidden)},
                        {dlogits, bytes_of(dtype, rows, vocab)}};
    for (int i = 0; i < 4; ++i)
      for (int j = i + 1; j < 7; ++j)
        if (overlap(all[i], all[j])) return vfail(FOLD_E_INVALID, who + ": an output overlaps another buffer");
    launch_vocab_backward(dtype, rows, hidden, vocab, states, W, dlogits, d_states, dW, dbias,
                          flags & FOLD_VOCAB_ACCUMULATE, ws, st);
    FOLD_HIP_CHECK(hipGetLastError());
    return FOLD_OK;
  });
}

int32_t fold_distill_workspace_size(int32_t dtype, int64_t rows, int32_t vocab, int32_t num_teacher, size_t* bytes) {
  return guarded([&]() -> int32_t {
    const std::string who("fold_distill_workspace_size");
    if (!bytes) return vfail(FOLD_E_INVALID, who + ": NULL argument");
    const int rc = check_distill_sizes(who, dtype, rows, vocab, num_teacher);
    if (rc != FOLD_OK) return rc;
    *bytes = distill_workspace_bytes(dtype, rows, vocab, num_teacher);
    return FOLD_OK;
  });
}

int32_t fold_loss_distill(const fold_sched* sched, int32_t dtype, int64_t rows, int32_t vocab, const void* logits,
                          int32_t num_teacher, const int32_t* teacher_token, const float* teacher_logit,
                          const int32_t* labels, float temperature, float soft_weight, float hard_weight, float scale,
                          float* row_loss, int32_t grad_dtype, void* dlogits, void* ws, size_t ws_bytes,
                          hipStream_t st) {
  return guarded([&]() -> int32_t {
    const std::string who("fold_loss_distill");
    int rc = check_distill_sizes(who, dtype, rows, vocab, num_teacher);
    if (rc != FOLD_OK) return rc;
    if (!known_type(grad_dtype) || (dtype == FOLD_BF16 && grad_dtype != FOLD_BF16))
      return vfail(FOLD_E_INVALID, who + ": the gradient is of the logits' type, or bf16");
    if (!(temperature >= 1e-3f && temperature <= 1e3f))
      return vfail(FOLD_E_INVALID, who + ": temperature must be in [1e-3, 1e3]");
    if (!(soft_weight >= 0.f && std::isfinite(soft_weight)) || !(hard_weight >= 0.f && std::isfinite(hard_weight)) ||
        !std::isfinite(scale))
      return vfail(FOLD_E_INVALID, who + ": weights must be finite and not negative, scale finite");
    const int* order = nullptr;
    rc = check_order(who, sched, rows, &order);
    if (rc != FOLD_OK) return rc;
    if (rows == 0) return FOLD_OK;
    if (!logits || !row_loss || (num_teacher > 0 && (!teacher_token || !teacher_logit)))
      return vfail(FOLD_E_INVALID, who + ": NULL buffer");
    if (misaligned(logits) || misaligned(dlogits) || misaligned(ws))
      return vfail(FOLD_E_INVALID, who + ": logits, dlogits and the workspace must be 16-byte aligned");
    if (dlogits && !(dlogits == logits && grad_dtype == dtype)) {
      if (overlap({logits, bytes_of(dtype, rows, vocab)}, {dlogits, bytes_of(grad_dtype, rows, vocab)}))
        return vfail(FOLD_E_INVALID, who + ": dlogits overlaps logits (it may be the same buffer for the same type)");
    }
    const size_t need = distill_workspace_bytes(dtype, rows, vocab, num_teacher);
    if (need > 0 && (!ws || ws_bytes < need))
      return vfail(FOLD_E_MISMATCH, who + ": workspace smaller than fold_distill_workspace_size");
    launch_distill(dtype, order, rows, vocab, logits, num_teacher, teacher_token, teacher_logit, labels, temperature,
                   soft_weight, hard_weight, scale, row_loss, grad_dtype, dlogits, ws, st);
    FOLD_HIP_CHECK(hipGetLastError());
    return FOLD_OK;
  });
}

int32_t fold_token_workspace_size(int32_t dtype, int64_t rows, int32_t vocab, int32_t top_k, size_t* bytes) {
  return guarded([&]() -> int32_t {
    const std::string who("fold_token_workspace_size");
    if (!bytes) return vfail(FOLD_E_INVALID, who + ": NULL argument");
    const int rc = check_token_sizes(who, dtype, rows, vocab, top_k);
    if (rc != FOLD_OK) return rc;
    *bytes = token_workspace_bytes(dtype, rows, vocab, top_k);
    return FOLD_OK;
  });
}

int32_t fold_token_logprobs(const fold_sched* sched, int32_t dtype, int64_t rows, int32_t vocab, const void* logits,
                            int32_t num_tokens, const int32_t* tokens, float* logp, float* entropy, int32_t top_k,
                            int32_t* top_token, float* top_logp, void* ws, size_t ws_bytes, hipStream_t st) {
  return guarded([&]() -> int32_t {
    const std::string who("fold_token_logprobs");
    int rc = check_token_sizes(who, dtype, rows, vocab, top_k);
    if (rc != FOLD_OK) return rc;
    if (num_tokens < 0) return vfail(FOLD_E_INVALID, who + ": negative num_tokens");
    const int* order = nullptr;
    rc = check_order(who, sched, rows, &order);
    if (rc != FOLD_OK) return rc;
    if (rows == 0 || (num_tokens == 0 && top_k == 0 && !entropy)) return FOLD_OK;
    if (!logits || (num_tokens > 0 && (!tokens || !logp)) || (top_k > 0 && (!top_token || !top_logp)))
      return vfail(FOLD_E_INVALID, who + ": NULL buffer");
    if (misaligned(logits) || misaligned(ws))
      return vfail(FOLD_E_INVALID, who + ": logits and the workspace must be 16-byte aligned");
    const size_t need = token_workspace_bytes(dtype, rows, vocab, top_k);
    if (need > 0 && (!ws || ws_bytes < need))
      return vfail(FOLD_E_MISMATCH, who + ": workspace smaller than fold_token_workspace_size");
    launch_token(dtype, order, rows, vocab, logits, num_tokens, tokens, logp, entropy, top_k, top_token, top_logp, ws,
                 st);
    FOLD_HIP_CHECK(hipGetLastError());
    return FOLD_OK;
  });
}

}  // extern "C"
