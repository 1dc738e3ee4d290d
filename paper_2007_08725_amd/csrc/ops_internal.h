// Internal declarations of the word-model operators (include/lda_ops.h): the
// launchers of ops_norm.hip and ops_product.hip.  Device code targets gfx950
// (CDNA4, wave64) only.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/lda_ops.h"

namespace lda {
namespace ops {

inline int64_t round_up(int64_t a, int64_t b) { return (a + b - 1) / b * b; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Scratch of one call, cut from the caller's workspace in 256-byte steps.
// With a null base it only counts: the *_workspace calls and the launches
// walk through the same code.
struct Arena {
  char *base = nullptr;
  size_t used = 0;
  template <typename T>
  T *take(int64_t count) {
    T *p = base ? reinterpret_cast<T *>(base + used) : nullptr;
    used += (size_t(count) * sizeof(T) + 255) & ~size_t(255);
    return p;
  }
};

// Each enqueues its kernels on the stream of `a`, or, with dry = true, only
// counts the workspace in `ws`.
hipError_t norm_forward(const lda_norm_args &a);
hipError_t norm_backward(const lda_norm_args &a, Arena &ws, bool dry);
hipError_t gated_forward(const lda_gated_args &a, Arena &ws, bool dry);
hipError_t gated_backward(const lda_gated_args &a, Arena &ws, bool dry);
hipError_t xent_forward(const lda_xent_args &a, Arena &ws, bool dry);
hipError_t xent_backward(const lda_xent_args &a, Arena &ws, bool dry);

}  // namespace ops
}  // namespace lda
