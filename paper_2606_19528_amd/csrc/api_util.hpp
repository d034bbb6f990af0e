// api_util.hpp -- what the C entry points share: errors, argument checks, and
// the launch timing hook.  Internal to the library; nothing here throws.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <cstdio>

#include "../../include/lora_mi355x.h"
#include "launch.hpp"

namespace lora {

inline lora_status_t fail(lora_status_t s, const char *msg) {
  set_last_error(msg);
  return s;
}

inline lora_status_t hip_fail(hipError_t e, const char *what) {
  char text[256];
  std::snprintf(text, sizeof text, "%s: %s", what, hipGetErrorString(e));
  set_last_error(text);
  return LORA_EHIP;
}

// ----- kernel timing hook ----------------------------------------------------
enum KernelId {
  K_GEMM_FWD = 0,     // y  = x W^T + (s u) B^T
  K_GEMM_BWD_DX,      // dx = dy W + du A, with the dA / dB token reductions alongside
  K_GEMM_FROZEN_DX,   // dx = dy W (rank 0)
  K_LORA_DOWN,        // u  = x A^T (+ LoRA-step operands)
  K_LORA_DY_B,        // du = s dy B (+ LoRA-step operand)
  K_GEMM_FWD_Q,       // gemm_fwd with the quantized W dequantized on the fly
  K_GEMM_BWD_DX_Q,    // gemm_bwd_dx, quantized W
  K_GEMM_FROZEN_DX_Q, // gemm_frozen_dx, quantized W
  K_HEAD_VOCAB,       // reduced vocabulary (mark, compact, target positions)
  K_HEAD_GATHER,      // gathers of the trainable hidden rows and of the rows of J
  K_HEAD_LOGITS,      // logits GEMM with the row-statistics epilogue (+ combine)
  K_HEAD_DZ,          // logits recomputed, softmax gradient epilogue
  K_HEAD_DH,          // dh += dz W_J (fp32), then the bf16 dh rows
  K_TOPK_SIM,         // similarity GEMM with the candidate epilogue (+ row norms)
  K_TOPK_SELECT,      // per-row selection of the k best candidates
  K_EMBED_FWD,        // embedding lookup
  K_EMBED_SORT,       // tokens of the embedding gradient sorted
  K_EMBED_GRAD,       // the gradient's sums
  K_TOKEN_LOGP,       // log-probabilities of the targets
  K_POLICY_LOSS,      // policy loss and its gradient
  K_PREFERENCE_LOSS,  // preference loss and its gradient
  K_GRAD_NORM,        // norm of a list of gradients
  K_GRAD_SCALE,       // the list scaled by the clip coefficient
  K_COUNT
};

// Tag of a launch's meetings (meet.hpp).
meet_word next_tag();

// Brackets the launches of one kernel with events while the hook is enabled.
struct Timed {
  int id;
  hipStream_t st;
  hipEvent_t a = nullptr, b = nullptr;
  bool on = false;
  Timed(int id, hipStream_t st);
  void done();
};

// ----- validation helpers ------------------------------------------------------
constexpr int64_t kMaxElems = (int64_t(1) << 31) - 1;
constexpr int64_t kMaxDim = int64_t(1) << 20;  // keeps every tile's byte offsets within 32 bits

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

struct Range {
  uintptr_t lo, hi;  // [lo, hi)
  bool set;
};
inline Range rng(const void *p, int64_t bytes) {
  if (!p || bytes <= 0) return {0, 0, false};
  uintptr_t lo = reinterpret_cast<uintptr_t>(p);
  return {lo, lo + (uintptr_t)bytes, true};
}
inline bool overlap(const Range &a, const Range &b) {
  return a.set && b.set && a.lo < b.hi && b.lo < a.hi;
}
// Whether an output overlaps an input or another output.
inline bool any_overlap(const Range *outs, size_t n_outs, const Range *ins, size_t n_ins) {
  for (size_t i = 0; i < n_outs; ++i) {
    for (size_t j = 0; j < n_ins; ++j)
      if (overlap(outs[i], ins[j])) return true;
    for (size_t j = i + 1; j < n_outs; ++j)
      if (overlap(outs[i], outs[j])) return true;
  }
  return false;
}

inline size_t esize(lora_dtype_t dt) { return dt == LORA_BF16 ? 2 : 4; }
inline size_t round256(size_t b) { return (b + 255) & ~size_t(255); }

inline lora_status_t check_ws(void *ws, size_t ws_bytes, size_t need) {
  if (need == 0) return LORA_OK;
  if (!ws) return fail(LORA_EWORKSPACE, "workspace required but ws is NULL");
  if (ws_bytes < need) return fail(LORA_EWORKSPACE, "workspace too small");
  if (!aligned16(ws)) return fail(LORA_EINVAL, "workspace not 16-byte aligned");
  return LORA_OK;
}

}  // namespace lora
