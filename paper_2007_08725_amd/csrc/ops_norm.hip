// Layer norm, forward and backward (include/lda_ops.h).
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "ops_internal.h"

#pragma clang fp contract(fast)

namespace lda {
namespace ops {
namespace {

typedef __bf16 bf16;
typedef _Float16 f16;

__device__ inline float block_sum(float v, float *shared) {
  for (int x = 1; x < 64; x <<= 1) v += __shfl_xor(v, x);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = v;
  __syncthreads();
  return shared[0] + shared[1] + shared[2] + shared[3];
}

// One workgroup per row.
template <typename T>
__global__ __launch_bounds__(256) void k_norm(const T *x, int64_t ldx, const T *weight, const T *bias, int cols,
                                              float eps, T *y, int64_t ldy, float *mean, float *rstd) {
  __shared__ float shared[4];
  const T *row = x + int64_t(blockIdx.x) * ldx;
  float s = 0.0f;
  for (int c = threadIdx.x; c < cols; c += 256) s += float(row[c]);
  const float mu = block_sum(s, shared) / cols;
  float q = 0.0f;
  for (int c = threadIdx.x; c < cols; c += 256) {
    const float d = float(row[c]) - mu;
    q += d * d;
  }
  const float r = 1.0f / sqrtf(block_sum(q, shared) / cols + eps);
  T *out = y + int64_t(blockIdx.x) * ldy;
  for (int c = threadIdx.x; c < cols; c += 256) {
    const float h = (float(row[c]) - mu) * r;
    out[c] = T(weight ? h * float(weight[c]) + float(bias[c]) : h);
  }
  if (threadIdx.x == 0) {
    mean[blockIdx.x] = mu;
    rstd[blockIdx.x] = r;
  }
}

template <typename T>
__global__ __launch_bounds__(256) void k_norm_dx(const T *dy, int64_t lddy, const T *x, int64_t ldx, const T *weight,
                                                 const float *mean, const float *rstd, int cols, T *dx, int64_t lddx) {
  __shared__ float shared[4];
  const T *row = x + int64_t(blockIdx.x) * ldx, *grad = dy + int64_t(blockIdx.x) * lddy;
  const float mu = mean[blockIdx.x], r = rstd[blockIdx.x];
  float sg = 0.0f, sh = 0.0f;
  for (int c = threadIdx.x; c < cols; c += 256) {
    const float g = float(grad[c]) * (weight ? float(weight[c]) : 1.0f);
    sg += g;
    sh += g * (float(row[c]) - mu) * r;
  }
  sg = block_sum(sg, shared) / cols;
  sh = block_sum(sh, shared) / cols;
  T *out = dx + int64_t(blockIdx.x) * lddx;
  for (int c = threadIdx.x; c < cols; c += 256) {
    const float g = float(grad[c]) * (weight ? float(weight[c]) : 1.0f);
    out[c] = T(r * (g - sg - (float(row[c]) - mu) * r * sh));
  }
}

// Column sums of dy h and dy over `per` rows a workgroup: part[2][parts][cols].
template <typename T>
__global__ __launch_bounds__(256) void k_norm_dw(const T *dy, int64_t lddy, const T *x, int64_t ldx, const float *mean,
                                                 const float *rstd, int64_t rows, int cols, int64_t per, float *part) {
  const int c = blockIdx.x * 256 + threadIdx.x;
  if (c >= cols) return;
  const int64_t first = blockIdx.y * per, last = first + per < rows ? first + per : rows;
  float sw = 0.0f, sb = 0.0f;
  for (int64_t r = first; r < last; ++r) {
    const float g = float(dy[r * lddy + c]);
    sb += g;
    sw += g * (float(x[r * ldx + c]) - mean[r]) * rstd[r];
  }
  part[int64_t(blockIdx.y) * cols + c] = sw;
  part[(int64_t(gridDim.y) + blockIdx.y) * cols + c] = sb;
}

template <typename T>
__global__ __launch_bounds__(256) void k_norm_join(const float *part, int parts, int cols, T *dweight, T *dbias) {
  const int c = blockIdx.x * 256 + threadIdx.x;
  if (c >= cols) return;
  const float *p = part + int64_t(blockIdx.y) * parts * cols + c;
  float s = 0.0f;
  for (int i = 0; i < parts; ++i) s += p[int64_t(i) * cols];
  (blockIdx.y ? dbias : dweight)[c] = T(s);
}

template <typename T>
hipError_t norm_forward_t(const lda_norm_args &a) {
  if (a.rows == 0) return hipSuccess;
  k_norm<T><<<unsigned(a.rows), 256, 0, static_cast<hipStream_t>(a.stream)>>>(
      static_cast<const T *>(a.x), a.ldx, static_cast<const T *>(a.weight), static_cast<const T *>(a.bias), a.cols,
      a.eps, static_cast<T *>(a.y), a.ldy, a.mean, a.rstd);
  return hipGetLastError();
}

template <typename T>
hipError_t norm_backward_t(const lda_norm_args &a, Arena &ws, bool dry) {
  const hipStream_t s = static_cast<hipStream_t>(a.stream);
  const int64_t parts = a.rows < 64 ? (a.rows ? a.rows : 1) : 64, per = ceil_div(a.rows, parts);
  float *part = a.dweight ? ws.take<float>(2 * parts * a.cols) : nullptr;
  if (dry) return hipSuccess;
  const T *dy = static_cast<const T *>(a.dy), *x = static_cast<const T *>(a.x);
  if (a.rows) {
    k_norm_dx<T><<<unsigned(a.rows), 256, 0, s>>>(dy, a.lddy, x, a.ldx, static_cast<const T *>(a.weight), a.mean,
                                                  a.rstd, a.cols, static_cast<T *>(a.dx), a.lddx);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (!a.dweight) return hipSuccess;
  const unsigned wide = unsigned(ceil_div(a.cols, 256));
  k_norm_dw<T><<<dim3(wide, unsigned(parts)), 256, 0, s>>>(dy, a.lddy, x, a.ldx, a.mean, a.rstd, a.rows, a.cols, per,
                                                          part);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  k_norm_join<T><<<dim3(wide, 2), 256, 0, s>>>(part, int(parts), a.cols, static_cast<T *>(a.dweight),
                                               static_cast<T *>(a.dbias));
  return hipGetLastError();
}

}  // namespace

hipError_t norm_forward(const lda_norm_args &a) {
  switch (a.dtype) {
    case LDA_F32: return norm_forward_t<float>(a);
    case LDA_BF16: return norm_forward_t<bf16>(a);
    default: return norm_forward_t<f16>(a);
  }
}

hipError_t norm_backward(const lda_norm_args &a, Arena &ws, bool dry) {
  switch (a.dtype) {
    case LDA_F32: return norm_backward_t<float>(a, ws, dry);
    case LDA_BF16: return norm_backward_t<bf16>(a, ws, dry);
    default: return norm_backward_t<f16>(a, ws, dry);
  }
}

}  // namespace ops
}  // namespace lda
