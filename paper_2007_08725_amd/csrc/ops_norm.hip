// Layer norm, forward and backward (include/lda_ops.h).
//
// Both passes are bound by memory: a row is read once, kept in the registers of
// the lanes that share it, reduced across them, and written once.  The backward
// pass walks several rows with the same lanes and keeps its columns' sums of
// dweight and dbias in registers meanwhile; they are joined in a fixed order.
// Rows too wide for that are read again.
//
// Measured: 8192 x 1024 of bf16 forward 9.6 us (3.5 TB/s), backward 13.2 us (3.8
// TB/s) and 4.3 us to join the 512 parts of each sum; 4096 x 32768 of f16 forward 124 us (4.3
// TB/s), backward 112 + 180 + 12 us.
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

template <typename T>
constexpr int kChunk = 16 / int(sizeof(T));

// 16 bytes of a row as they lie in memory.
template <typename T>
struct Chunk {
  typedef T vec __attribute__((ext_vector_type(kChunk<T>)));
  vec v;
  __device__ float operator[](int e) const { return float(v[e]); }
};

// The columns of a row that a lane holds: V chunks, LANES chunks apart.  Rows
// that do not start at multiples of 16 bytes, or do not end at one, are moved
// element by element.
template <typename T, int LANES, int V, bool Aligned>
struct Cols {
  static constexpr int C = kChunk<T>;
  static __device__ int first(int v, int lane) { return (v * LANES + lane) * C; }
  static __device__ void load_one(const T *row, int cols, int lane, int v, Chunk<T> &x) {
    const int c = first(v, lane);
    if (Aligned) {
      if (c < cols) x.v = *reinterpret_cast<const typename Chunk<T>::vec *>(row + c);
      else x.v = typename Chunk<T>::vec(T(0.0f));
    } else {
#pragma unroll
      for (int e = 0; e < C; ++e) x.v[e] = c + e < cols ? row[c + e] : T(0.0f);
    }
  }
  static __device__ void load(const T *row, int cols, int lane, Chunk<T> (&x)[V]) {
#pragma unroll
    for (int v = 0; v < V; ++v) load_one(row, cols, lane, v, x[v]);
  }
  static __device__ void store(T *row, int cols, int c, typename Chunk<T>::vec x) {
    if (Aligned) {
      if (c < cols) *reinterpret_cast<typename Chunk<T>::vec *>(row + c) = x;
    } else {
#pragma unroll
      for (int e = 0; e < C; ++e)
        if (c + e < cols) row[c + e] = x[e];
    }
  }
};

// Sums over the LANES lanes that share a row; every lane gets them.
template <int LANES>
__device__ inline float2 row_sum(float2 s, float2 *shared) {
#pragma unroll
  for (int x = 1; x < (LANES < 64 ? LANES : 64); x <<= 1) {
    s.x += __shfl_xor(s.x, x);
    s.y += __shfl_xor(s.y, x);
  }
  if (LANES > 64) {
    constexpr int WAVES = LANES / 64;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = s;
    __syncthreads();
    s = shared[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) {
      s.x += shared[w].x;
      s.y += shared[w].y;
    }
  }
  return s;
}

constexpr int threads_of(int lanes) { return lanes > 256 ? lanes : 256; }

template <typename T, int LANES, int V, bool Aligned>
__global__ __launch_bounds__(threads_of(LANES)) void k_norm(const T *x, int64_t ldx, const T *weight, const T *bias,
                                                            int64_t rows, int cols, float eps, T *y, int64_t ldy,
                                                            float *mean, float *rstd) {
  typedef Cols<T, LANES, V, Aligned> At;
  constexpr int C = At::C;
  __shared__ float2 shared[16];
  const int lane = threadIdx.x % LANES;
  const int64_t row = int64_t(blockIdx.x) * (threads_of(LANES) / LANES) + threadIdx.x / LANES;
  if (LANES <= 64 && row >= rows) return;
  Chunk<T> v[V];
  At::load(x + row * ldx, cols, lane, v);
  float s = 0.0f;
#pragma unroll
  for (int i = 0; i < V; ++i)
#pragma unroll
    for (int e = 0; e < C; ++e) s += v[i][e];
  const float mu = row_sum<LANES>(make_float2(s, 0.0f), shared).x / cols;
  // the squares of the deviations, not the sum of squares: exact where a row's
  // mean is large beside its spread
  float q = 0.0f;
#pragma unroll
  for (int i = 0; i < V; ++i)
#pragma unroll
    for (int e = 0; e < C; ++e) {
      const float d = At::first(i, lane) + e < cols ? v[i][e] - mu : 0.0f;
      q += d * d;
    }
  const float r = 1.0f / sqrtf(row_sum<LANES>(make_float2(q, 0.0f), shared).x / cols + eps);
  if (lane == 0) {
    mean[row] = mu;
    rstd[row] = r;
  }
  Chunk<T> w[V], b[V];
  if (weight) {
    At::load(weight, cols, lane, w);
    At::load(bias, cols, lane, b);
  }
  T *out = y + row * ldy;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    typename Chunk<T>::vec o;
#pragma unroll
    for (int e = 0; e < C; ++e) {
      const float h = (v[i][e] - mu) * r;
      o[e] = T(weight ? h * w[i][e] + b[i][e] : h);
    }
    At::store(out, cols, At::first(i, lane), o);
  }
}

// Each group of LANES lanes takes every (gridDim.x * groups)-th row.  part
// [2][gridDim.x][cols]: the workgroup's sums of dy h and of dy by column.
template <typename T, int LANES, int V, bool Aligned>
__global__ __launch_bounds__(threads_of(LANES)) void k_norm_grad(const T *dy, int64_t lddy, const T *x, int64_t ldx,
                                                                 const T *weight, const float *mean, const float *rstd,
                                                                 int64_t rows, int cols, T *dx, int64_t lddx,
                                                                 float *part) {
  typedef Cols<T, LANES, V, Aligned> At;
  constexpr int C = At::C, THREADS = threads_of(LANES), GROUPS = THREADS / LANES;
  __shared__ float2 shared[GROUPS > 1 ? THREADS * C : 16];
  const int lane = threadIdx.x % LANES, group = threadIdx.x / LANES;
  float sw[V][C], sb[V][C];
#pragma unroll
  for (int i = 0; i < V; ++i)
#pragma unroll
    for (int e = 0; e < C; ++e) sw[i][e] = sb[i][e] = 0.0f;
  Chunk<T> w[V];
  if (weight) At::load(weight, cols, lane, w);
  // every lane of a workgroup that meets at barriers has the same rows
  for (int64_t row = int64_t(blockIdx.x) * GROUPS + group; row < rows; row += int64_t(gridDim.x) * GROUPS) {
    Chunk<T> v[V], d[V];
    At::load(x + row * ldx, cols, lane, v);
    At::load(dy + row * lddy, cols, lane, d);
    const float mu = mean[row], r = rstd[row];
    float2 s = make_float2(0.0f, 0.0f);
#pragma unroll
    for (int i = 0; i < V; ++i) {
#pragma unroll
      for (int e = 0; e < C; ++e) {
        const float h = (v[i][e] - mu) * r;
        const float g = weight ? d[i][e] * w[i][e] : d[i][e];
        // past the columns dy is 0
        s.x += g;
        s.y += g * h;
        sw[i][e] += d[i][e] * h;
        sb[i][e] += d[i][e];
      }
    }
    s = row_sum<LANES>(s, shared);
    s.x /= cols;
    s.y /= cols;
    T *out = dx + row * lddx;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      typename Chunk<T>::vec o;
#pragma unroll
      for (int e = 0; e < C; ++e) {
        const float h = (v[i][e] - mu) * r;
        const float g = weight ? d[i][e] * w[i][e] : d[i][e];
        o[e] = T(r * (g - s.x - h * s.y));
      }
      At::store(out, cols, At::first(i, lane), o);
    }
  }
  if (!part) return;
  float *pw = part + int64_t(blockIdx.x) * cols, *pb = pw + int64_t(gridDim.x) * cols;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    if (GROUPS > 1) {
      // the groups' sums, in the order of the groups
      __syncthreads();
#pragma unroll
      for (int e = 0; e < C; ++e) shared[e * THREADS + threadIdx.x] = make_float2(sw[i][e], sb[i][e]);
      __syncthreads();
      for (int at = threadIdx.x; at < LANES * C; at += THREADS) {
        const int e = at % C, l = at / C, c = At::first(i, l) + e;
        float2 t = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
          const float2 o = shared[e * THREADS + g * LANES + l];
          t.x += o.x;
          t.y += o.y;
        }
        if (c < cols) {
          pw[c] = t.x;
          pb[c] = t.y;
        }
      }
    } else {
#pragma unroll
      for (int e = 0; e < C; ++e) {
        const int c = At::first(i, lane) + e;
        if (c < cols) {
          pw[c] = sw[i][e];
          pb[c] = sb[i][e];
        }
      }
    }
  }
}

// dweight (blockIdx.y = 0) and dbias (1) from their parts: 16 columns a
// workgroup, 16 threads a column.
template <typename T>
__global__ __launch_bounds__(256) void k_norm_join(const float *part, int parts, int cols, T *dweight, T *dbias) {
  __shared__ float shared[16][17];
  const int c = blockIdx.x * 16 + (threadIdx.x & 15), way = threadIdx.x >> 4;
  float s = 0.0f;
  if (c < cols) {
    const float *p = part + int64_t(blockIdx.y) * parts * cols + c;
#pragma unroll 4
    for (int i = way; i < parts; i += 16) s += p[int64_t(i) * cols];
  }
  shared[way][threadIdx.x & 15] = s;
  __syncthreads();
  if (threadIdx.x < 16 && c < cols) {
    for (int w = 1; w < 16; ++w) s += shared[w][threadIdx.x];
    (blockIdx.y ? dbias : dweight)[c] = T(s);
  }
}

// ---------------------------------------------- rows wider than registers ---
template <typename T>
__global__ __launch_bounds__(1024) void k_norm_wide(const T *x, int64_t ldx, const T *weight, const T *bias, int cols,
                                                    float eps, T *y, int64_t ldy, float *mean, float *rstd) {
  __shared__ float2 shared[16];
  const T *row = x + int64_t(blockIdx.x) * ldx;
  float s = 0.0f;
  for (int c = threadIdx.x; c < cols; c += 1024) s += float(row[c]);
  const float mu = row_sum<1024>(make_float2(s, 0.0f), shared).x / cols;
  float q = 0.0f;
  for (int c = threadIdx.x; c < cols; c += 1024) {
    const float d = float(row[c]) - mu;
    q += d * d;
  }
  const float r = 1.0f / sqrtf(row_sum<1024>(make_float2(q, 0.0f), shared).x / cols + eps);
  T *out = y + int64_t(blockIdx.x) * ldy;
  for (int c = threadIdx.x; c < cols; c += 1024) {
    const float h = (float(row[c]) - mu) * r;
    out[c] = T(weight ? h * float(weight[c]) + float(bias[c]) : h);
  }
  if (threadIdx.x == 0) {
    mean[blockIdx.x] = mu;
    rstd[blockIdx.x] = r;
  }
}

// The backward pass in two kernels: the rows' two sums (sums [2][rows]: mean g,
// mean g h), then strips of 256 chunks of the columns over `per` rows each, which
// give dx and the parts [2][gridDim.y][cols] of dweight and dbias.  x and dy are
// read twice, but a lane keeps one chunk's sums: all columns of such a row kept
// by 512 or 1,024 lanes need more registers than there are (measured at 32,768
// columns of 16 bits: 402 to 680 us in one kernel, against 290 here).
template <typename T, bool Aligned>
__global__ __launch_bounds__(1024) void k_norm_wide_sums(const T *dy, int64_t lddy, const T *x, int64_t ldx,
                                                         const T *weight, const float *mean, const float *rstd,
                                                         int64_t rows, int cols, float *sums) {
  typedef Cols<T, 1024, 1, Aligned> At;
  constexpr int C = At::C;
  __shared__ float2 shared[16];
  const int64_t row = blockIdx.x;
  const float mu = mean[row], r = rstd[row];
  float2 s = make_float2(0.0f, 0.0f);
#pragma unroll 2
  for (int c = 0; c < cols; c += 1024 * C) {
    Chunk<T> v, d, w;
    At::load_one(x + row * ldx + c, cols - c, threadIdx.x, 0, v);
    At::load_one(dy + row * lddy + c, cols - c, threadIdx.x, 0, d);
    if (weight) At::load_one(weight + c, cols - c, threadIdx.x, 0, w);
#pragma unroll
    for (int e = 0; e < C; ++e) {
      const float g = weight ? d[e] * w[e] : d[e];
      s.x += g;
      s.y += g * ((v[e] - mu) * r);
    }
  }
  s = row_sum<1024>(s, shared);
  if (threadIdx.x == 0) {
    sums[row] = s.x / cols;
    sums[rows + row] = s.y / cols;
  }
}

template <typename T, bool Aligned>
__global__ __launch_bounds__(256) void k_norm_wide_grad(const T *dy, int64_t lddy, const T *x, int64_t ldx,
                                                        const T *weight, const float *mean, const float *rstd,
                                                        const float *sums, int64_t rows, int cols, int64_t per, T *dx,
                                                        int64_t lddx, float *part) {
  typedef Cols<T, 256, 1, Aligned> At;
  constexpr int C = At::C;
  const int first = blockIdx.x * 256 * C, mine = cols - first;  // the strip's first column, and the columns from it on
  const int lane = threadIdx.x, c = At::first(0, lane);
  Chunk<T> w;
  if (weight) At::load_one(weight + first, mine, lane, 0, w);
  float sw[C], sb[C];
#pragma unroll
  for (int e = 0; e < C; ++e) sw[e] = sb[e] = 0.0f;
  const int64_t from = blockIdx.y * per, to = from + per < rows ? from + per : rows;
#pragma unroll 4
  for (int64_t row = from; row < to; ++row) {
    Chunk<T> v, d;
    At::load_one(x + row * ldx + first, mine, lane, 0, v);
    At::load_one(dy + row * lddy + first, mine, lane, 0, d);
    const float mu = mean[row], r = rstd[row], mg = sums[row], mh = sums[rows + row];
    typename Chunk<T>::vec o;
#pragma unroll
    for (int e = 0; e < C; ++e) {
      const float h = (v[e] - mu) * r;
      const float g = weight ? d[e] * w[e] : d[e];
      sw[e] += d[e] * h;
      sb[e] += d[e];
      o[e] = T(r * (g - mg - h * mh));
    }
    At::store(dx + row * lddx + first, mine, c, o);
  }
  if (!part) return;
#pragma unroll
  for (int e = 0; e < C; ++e)
    if (c + e < mine) {
      part[int64_t(blockIdx.y) * cols + first + c + e] = sw[e];
      part[(int64_t(gridDim.y) + blockIdx.y) * cols + first + c + e] = sb[e];
    }
}

// ------------------------------------------------------------------- host ---
template <int LANES_, int V_, bool Aligned_>
struct Shape {
  static constexpr int LANES = LANES_, V = V_;
  static constexpr bool Aligned = Aligned_;
};

// Calls fn with the lanes that share a row of `chunks` 16-byte chunks and the
// chunks that each holds; false if no lanes hold them all.  A wave a row up to
// 256 chunks (of 8 lanes up to 8), then workgroups of 256 threads, then of 1,024
// in the forward pass and of 512 in the backward pass, whose lanes need more
// registers: two sums of each column.
template <bool Aligned, bool Grad, typename Fn>
bool with_lanes(int64_t chunks, Fn fn) {
  if (chunks <= 8) fn(Shape<8, 1, Aligned>());
  else if (chunks <= 64) fn(Shape<64, 1, Aligned>());
  else if (chunks <= 128) fn(Shape<64, 2, Aligned>());
  else if (chunks <= 256) fn(Shape<64, 4, Aligned>());
  else if (chunks <= 512) fn(Shape<256, 2, Aligned>());
  else if (chunks <= 1024) fn(Shape<256, 4, Aligned>());
  else if (chunks <= 2048) fn(Shape<Grad ? 512 : 1024, Grad ? 4 : 2, Aligned>());
  else {
    if constexpr (!Grad)
      if (chunks <= 4096) {
        fn(Shape<1024, 4, Aligned>());
        return true;
      }
    return false;
  }
  return true;
}

template <typename T, bool Grad, typename Fn>
bool with_shape(bool aligned, int cols, Fn fn) {
  const int64_t chunks = ceil_div(cols, kChunk<T>);
  return aligned ? with_lanes<true, Grad>(chunks, fn) : with_lanes<false, Grad>(chunks, fn);
}

template <typename T>
bool aligned16(const void *p, int64_t ld) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld % kChunk<T> == 0;
}

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

template <typename T>
hipError_t norm_forward_t(const lda_norm_args &a) {
  if (a.rows == 0) return hipSuccess;
  const hipStream_t s = static_cast<hipStream_t>(a.stream);
  const T *x = static_cast<const T *>(a.x), *w = static_cast<const T *>(a.weight), *b = static_cast<const T *>(a.bias);
  T *y = static_cast<T *>(a.y);
  const bool aligned = a.cols % kChunk<T> == 0 && aligned16<T>(x, a.ldx) && aligned16<T>(y, a.ldy) &&
                       aligned16<T>(w, 0) && aligned16<T>(b, 0);
  hipError_t e = hipSuccess;
  const bool done = with_shape<T, false>(aligned, a.cols, [&](auto shape) {
    typedef decltype(shape) S;
    constexpr int threads = threads_of(S::LANES), groups = threads / S::LANES;
    e = by_rows(a.rows, threads, groups, [&](int64_t m, int64_t rows) {
      k_norm<T, S::LANES, S::V, S::Aligned><<<unsigned(ceil_div(rows, groups)), threads, 0, s>>>(
          x + m * a.ldx, a.ldx, w, b, rows, a.cols, a.eps, y + m * a.ldy, a.ldy, a.mean + m, a.rstd + m);
    });
  });
  if (done) return e;
  return by_rows(a.rows, 1024, 1, [&](int64_t m, int64_t rows) {
    k_norm_wide<T><<<unsigned(rows), 1024, 0, s>>>(x + m * a.ldx, a.ldx, w, b, a.cols, a.eps, y + m * a.ldy, a.ldy,
                                                   a.mean + m, a.rstd + m);
  });
}

template <typename T>
hipError_t norm_backward_t(const lda_norm_args &a, Arena &ws, bool dry) {
  const hipStream_t s = static_cast<hipStream_t>(a.stream);
  const T *dy = static_cast<const T *>(a.dy), *x = static_cast<const T *>(a.x), *w = static_cast<const T *>(a.weight);
  T *dx = static_cast<T *>(a.dx);
  const bool aligned = a.cols % kChunk<T> == 0 && aligned16<T>(x, a.ldx) && aligned16<T>(dy, a.lddy) &&
                       aligned16<T>(dx, a.lddx) && aligned16<T>(w, 0);
  hipError_t e = hipSuccess;
  int64_t parts = 0;
  float *part = nullptr;
  const bool done = with_shape<T, true>(aligned, a.cols, [&](auto shape) {
    typedef decltype(shape) S;
    constexpr int threads = threads_of(S::LANES), groups = threads / S::LANES;
    // workgroups: enough to fill the device, each with several rows, so that
    // the parts stay small beside x and dy
    const int64_t most = threads == 512 ? 256 : 1024;
    parts = ceil_div(a.rows, groups * 4);
    parts = parts > most ? most : parts < 1 ? 1 : parts;
    part = a.dweight ? ws.take<float>(2 * parts * a.cols) : nullptr;
    if (dry) return;
    k_norm_grad<T, S::LANES, S::V, S::Aligned><<<unsigned(parts), threads, 0, s>>>(
        dy, a.lddy, x, a.ldx, w, a.mean, a.rstd, a.rows, a.cols, dx, a.lddx, part);
    e = hipGetLastError();
  });
  if (!done) {
    const int64_t strips = ceil_div(a.cols, 256 * kChunk<T>);
    // about 2,048 workgroups, each with at least eight rows
    const int64_t per = a.rows * strips > 16384 ? ceil_div(a.rows * strips, 2048) : 8;
    parts = a.rows ? ceil_div(a.rows, per) : 1;
    part = a.dweight ? ws.take<float>(2 * parts * a.cols) : nullptr;
    float *sums = ws.take<float>(2 * a.rows);
    if (!dry) {
      auto sum = aligned ? k_norm_wide_sums<T, true> : k_norm_wide_sums<T, false>;
      e = by_rows(a.rows, 1024, 1, [&](int64_t m, int64_t rows) {
        sum<<<unsigned(rows), 1024, 0, s>>>(dy + m * a.lddy, a.lddy, x + m * a.ldx, a.ldx, w, a.mean + m, a.rstd + m,
                                            a.rows, a.cols, sums + m);
      });
      if (e != hipSuccess) return e;
      auto kernel = aligned ? k_norm_wide_grad<T, true> : k_norm_wide_grad<T, false>;
      kernel<<<dim3(unsigned(strips), unsigned(parts)), 256, 0, s>>>(dy, a.lddy, x, a.ldx, w, a.mean, a.rstd, sums,
                                                                    a.rows, a.cols, per, dx, a.lddx, part);
      e = hipGetLastError();
    }
  }
  if (dry || !part || e != hipSuccess) return e;
  k_norm_join<T><<<dim3(unsigned(ceil_div(a.cols, 16)), 2), 256, 0, s>>>(part, int(parts), a.cols,
                                                                         static_cast<T *>(a.dweight),
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
