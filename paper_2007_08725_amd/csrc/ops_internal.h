// Internal declarations of the word-model operators (include/lda_ops.h): the
// launchers of ops_norm.hip, ops_product.hip, ops_embed.hip and ops_recurrence.hip.  Device code targets gfx950
// (CDNA4, wave64) only.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/lda_ops.h"

namespace lda {
namespace ops {

inline int64_t round_up(int64_t a, int64_t b) { return (a + b - 1) / b * b; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Workgroups of a kernel that strides over its elements.
inline unsigned strided(int64_t workgroups) { return unsigned(workgroups < 65536 ? workgroups : 65536); }

#define OPS_TRY(expr)                      \
  do {                                     \
    hipError_t e_ = (expr);                \
    if (e_ != hipSuccess) return e_;       \
  } while (0)

// Launches fn(first row, rows) for all rows, `groups` of them to a workgroup of
// `threads`: in more than one launch where one would have 2^32 threads.
template <typename Fn>
hipError_t by_rows(int64_t rows, int64_t threads, int64_t groups, Fn fn) {
  const int64_t most = 0xffffffffll / threads * groups;
  for (int64_t first = 0; first < rows; first += most) {
    fn(first, rows - first < most ? rows - first : most);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

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
hipError_t embed_forward(const lda_embed_args &a);
hipError_t embed_backward(const lda_embed_args &a, Arena &ws, bool dry);
hipError_t recur_forward(const lda_recur_args &a, Arena &ws, bool dry);
hipError_t recur_backward(const lda_recur_args &a, Arena &ws, bool dry);
hipError_t recur_step(const lda_recur_args &a);
hipError_t distill_forward(const lda_distill_args &a, Arena &ws, bool dry);
hipError_t distill_backward(const lda_distill_args &a, Arena &ws, bool dry);

// dweight[v] = scale times the sum of the rows i of dy with words[i] = v, in one
// order (ops_embed.hip); defined for float outside that file.
template <typename T>
hipError_t sum_by_word(const int32_t *words, int64_t n, const T *dy, int64_t lddy, int width, int vocab, float scale,
                       T *dweight, Arena &ws, bool dry, hipStream_t s);

}  // namespace ops
}  // namespace lda
